"""Binding of libtbn's paged key/value cache and its attention (include/tbn.h), in the manner of ``tbn.py``: argument
marshalling only, PyTorch supplies device memory and the stream, there is no CPU fallback.

    pool = kv.kv_pool(n_pages, kv_heads, dim, page, torch.bfloat16, summary=True)     # one per layer
    index = kv.kv_index(n_seqs, max_pages, n_pages, page)                             # one for all of them

    kv.tbn_kv_reserve(index, n_new) -> pairs for tbn_kv_copy_pages                    # once per step
    kv.tbn_kv_append(pool, index, k_new, v_new, cu_new, max_new)                      # per layer
    out, lse = kv.tbn_tree_attention(q, pool, index, cu_q, max_q, mask=...)
    picks = kv.tbn_block_select(q, pool, index, cu_q, max_q, n_select)
    out, lse = kv.tbn_block_attention(q, pool, index, cu_q, max_q, picks)
    out, lse = kv.tbn_window_attention(q, pool, index, cu_q, max_q, n_sink, window, mask=...)
    kv.tbn_kv_keep / tbn_kv_release / tbn_kv_fork / tbn_kv_compact / tbn_kv_copy_pages

    pool = kv.kv4_pool(n_pages, kv_heads, dim, page)                                  # in place of kv_pool: keys and values in 4 bits
    kv.tbn_kv4_append / tbn_kv4_read / tbn_kv4_keep / tbn_kv4_copy_pages
    out, lse = kv.tbn_kv4_attention(q, pool, index, cu_q, max_q, mask=..., n_sink=..., window=...)

    picks, counts, next = kv.tbn_verify(target, tokens, u, cu_q, max_q, draft=..., parents=...)   # picks and counts go to tbn_kv_keep

``KVPool``, ``KV4Pool`` and ``KVIndex`` hold the tensors and the C structs that describe them; build them once.
"""
from __future__ import annotations

import ctypes
import math
from typing import Optional, Tuple

import torch

from . import tbn
from .tbn import _call, _dev, _dt, _empty, _own, _raise, _stream, lib, TBN_OK

TBN_KV_FULL = 1
TBN_KV_INVALID = 2
MAX_SEQUENCES = 8192        # of an index, of a verification
VERIFY_MAX_TOKENS = 2048    # of a sequence


class _Pool(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("summary", ctypes.c_void_p), ("step", ctypes.c_void_p),
                ("n_pages", ctypes.c_int64), ("kv_heads", ctypes.c_int32), ("dim", ctypes.c_int32), ("page", ctypes.c_int32),
                ("dt", ctypes.c_int32)]


class _Pool4(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_exp", ctypes.c_void_p), ("v_exp", ctypes.c_void_p),
                ("n_pages", ctypes.c_int64), ("kv_heads", ctypes.c_int32), ("dim", ctypes.c_int32), ("page", ctypes.c_int32)]


class _Index(ctypes.Structure):
    _fields_ = [("table", ctypes.c_void_p), ("lens", ctypes.c_void_p), ("refs", ctypes.c_void_p), ("status", ctypes.c_void_p),
                ("n_pages", ctypes.c_int64), ("n_seqs", ctypes.c_int32), ("max_pages", ctypes.c_int32), ("page", ctypes.c_int32)]


class KVPool:
    """Pages of one layer: k (n_pages, kv_heads, page, dim), v (n_pages, kv_heads, dim, page), both float32 or bfloat16, and,
    for ``tbn_block_select``, summary int8 (n_pages, kv_heads, 2, dim) with step float32 (n_pages, kv_heads)."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, summary: Optional[torch.Tensor] = None, step: Optional[torch.Tensor] = None):
        if k.dim() != 4:
            raise ValueError("k must be (n_pages, kv_heads, page, dim)")
        n, h, p, d = k.shape
        if tuple(v.shape) != (n, h, d, p) or v.dtype != k.dtype:
            raise ValueError("v must be (n_pages, kv_heads, dim, page) with k's dtype")
        if (summary is None) != (step is None):
            raise ValueError("summary and step go together")
        if summary is not None and (tuple(summary.shape) != (n, h, 2, d) or tuple(step.shape) != (n, h)):
            raise ValueError("summary must be (n_pages, kv_heads, 2, dim), step (n_pages, kv_heads)")
        _same_device(k.device, v, summary, step)
        self.k, self.v, self.summary, self.step = k, v, summary, step
        self.n_pages, self.kv_heads, self.page, self.dim, self.dtype, self.device = n, h, p, d, k.dtype, k.device
        self._c = _Pool(_dev(k, "k"), _dev(v, "v"), None if summary is None else _dev(summary, "summary", torch.int8),
                        None if step is None else _dev(step, "step", torch.float32), n, h, d, p, _dt(k))
        self._at, self._gpu = ctypes.addressof(self._c), k.device.index


class KV4Pool:
    """Pages of one layer in 4 bits: k uint8 (n_pages, kv_heads, page, dim / 2), v uint8 (n_pages, kv_heads, page / 32, 4, 16, dim / 16, 4), k_exp
    and v_exp int8 (n_pages, kv_heads, page, 4 or, for more than 128 channels, 8); what they hold: include/tbn.h."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_exp: torch.Tensor, v_exp: torch.Tensor):
        if k.dim() != 4:
            raise ValueError("k must be (n_pages, kv_heads, page, dim / 2)")
        n, h, p, half = k.shape
        d = 2 * half
        if tuple(v.shape) != (n, h, p // 32, 4, 16, d // 16, 4):
            raise ValueError("v must be (n_pages, kv_heads, page / 32, 4, 16, dim / 16, 4)")
        if any(tuple(t.shape) != (n, h, p, 4 if d <= 128 else 8) for t in (k_exp, v_exp)):
            raise ValueError("k_exp and v_exp must be (n_pages, kv_heads, page, 4 or, for more than 128 channels, 8)")
        _same_device(k.device, v, k_exp, v_exp)
        self.k, self.v, self.k_exp, self.v_exp = k, v, k_exp, v_exp
        self.n_pages, self.kv_heads, self.page, self.dim, self.dtype, self.device = n, h, p, d, None, k.device
        self._c = _Pool4(_dev(k, "k", torch.uint8), _dev(v, "v", torch.uint8), _dev(k_exp, "k_exp", torch.int8), _dev(v_exp, "v_exp", torch.int8), n, h, d, p)
        self._at, self._gpu = ctypes.addressof(self._c), k.device.index


class KVIndex:
    """Bookkeeping that the layers of a model share, int32: table (n_seqs, max_pages), lens (n_seqs), refs (n_pages), status (1)."""

    def __init__(self, table: torch.Tensor, lens: torch.Tensor, refs: torch.Tensor, status: torch.Tensor, page: int):
        if table.dim() != 2 or lens.dim() != 1 or lens.numel() != table.shape[0] or refs.dim() != 1 or status.numel() != 1:
            raise ValueError("table must be (n_seqs, max_pages), lens (n_seqs), refs (n_pages), status (1)")
        _same_device(table.device, lens, refs, status)
        self.table, self.lens, self.refs, self.status = table, lens, refs, status
        self.n_seqs, self.max_pages, self.n_pages, self.page, self.device = table.shape[0], table.shape[1], refs.numel(), page, table.device
        self._c = _Index(*(_dev(t, n, torch.int32) for t, n in ((table, "table"), (lens, "lens"), (refs, "refs"), (status, "status"))),
                         self.n_pages, self.n_seqs, self.max_pages, page)
        self._at, self._gpu = ctypes.addressof(self._c), table.device.index
        self._ws = int(lib().tbn_kv_workspace_bytes(self.n_pages, self.n_seqs))


def kv_pool(n_pages: int, kv_heads: int, dim: int, page: int, dtype: torch.dtype, summary: bool = False, device="cuda") -> KVPool:
    """A pool of pages; their contents are undefined until keys are appended."""
    return KVPool(torch.empty(n_pages, kv_heads, page, dim, dtype=dtype, device=device), torch.empty(n_pages, kv_heads, dim, page, dtype=dtype, device=device),
                  torch.empty(n_pages, kv_heads, 2, dim, dtype=torch.int8, device=device) if summary else None,
                  torch.empty(n_pages, kv_heads, dtype=torch.float32, device=device) if summary else None)


def kv4_pool(n_pages: int, kv_heads: int, dim: int, page: int, device="cuda") -> KV4Pool:
    """A pool of pages in 4 bits; their contents are undefined until keys are appended."""
    if dim % 32 or page % 32:
        raise ValueError("dim and page must be multiples of 32")
    new = lambda dtype, *shape: torch.empty(n_pages, kv_heads, *shape, dtype=dtype, device=device)  # noqa: E731
    exps = 4 if dim <= 128 else 8
    return KV4Pool(new(torch.uint8, page, dim // 2), new(torch.uint8, page // 32, 4, 16, dim // 16, 4), new(torch.int8, page, exps), new(torch.int8, page, exps))


def kv_index(n_seqs: int, max_pages: int, n_pages: int, page: int, device="cuda") -> KVIndex:
    """Bookkeeping of empty sequences and free pages."""
    z = lambda *shape: torch.zeros(shape, dtype=torch.int32, device=device)  # noqa: E731
    return KVIndex(z(n_seqs, max_pages) - 1, z(n_seqs), z(n_pages), z(1), page)


def _same_device(device: torch.device, *tensors):
    for t in tensors:
        if t is not None and t.device != device:
            raise ValueError(f"all tensors must live on {device}")


def _ints(t: torch.Tensor, name: str, at_least: int, device: torch.device) -> int:
    if t.numel() < at_least:
        raise ValueError(f"{name} has {t.numel()} entries, {at_least} needed")
    _same_device(device, t)
    return _dev(t, name, torch.int32)


def _rows(t: torch.Tensor, name: str, heads: int, dim: int, like) -> Tuple[int, int]:
    """Address and token stride of (tokens, heads, dim) whose last two axes are dense; of the pool's type, where it has one."""
    if t.dim() != 3 or t.shape[1] != heads or t.shape[2] != dim or t.dtype not in ((like.dtype,) if like.dtype else (torch.float32, torch.bfloat16)):
        raise ValueError(f"{name} must be (tokens, {heads}, {dim}) with dtype {like.dtype or 'float32 or bfloat16'}")
    if not t.is_cuda or t.device != like.device:
        raise ValueError(f"{name} must be a device tensor on {like.device}")
    st = t.stride()
    n = t.shape[0]
    if t.numel() and ((dim > 1 and st[2] != 1) or (heads > 1 and st[1] != dim) or (n > 1 and st[0] < heads * dim)):
        raise ValueError(f"{name}: the heads of a token must be dense and tokens must not overlap (strides {st})")
    return t.data_ptr(), st[0] if n > 1 else heads * dim


def _of(kind: type, x, name: str) -> None:
    """Refuses what is not of the class that a call is for: the structs have one size, and the library would take a byte of one pool for an element of the
    other.  (A call comes here where the type is not the very one.)"""
    if not isinstance(x, kind):
        raise ValueError(f"{name} must be a {kind.__name__}, got {type(x).__name__}")


def _fit(*values: int):
    """Integers as the library's 32 bits hold them, the nearest where they do not: a window beyond them is none, and what has to be at least a number stays it
    (cut to its low bits, it would be another one).  Others are refused there."""
    return tuple(v if -1 << 31 <= v < 1 << 31 else (1 << 31) - 1 if v > 0 else -1 << 31 for v in values)


def _fit64(v: Optional[int]) -> int:
    return 0 if v is None else v if -1 << 63 <= v < 1 << 63 else (1 << 63) - 1 if v > 0 else -1 << 63


def _agree(pool, index: KVIndex):
    if pool.device != index.device:
        raise ValueError(f"pool and index must live on one device, got {pool.device} and {index.device}")


def _workspace(need: int, workspace: Optional[torch.Tensor], device: torch.device, stream):
    if workspace is None:
        if need == 0:
            return None, 0
        workspace = _own(_empty(need, torch.uint8, device, stream, output=False))
    else:
        _same_device(device, workspace)
    return _dev(workspace, "workspace"), workspace.numel() * workspace.element_size()


def _plain(*defaults) -> bool:
    """Whether a call has the plain form that the extension module takes: nothing given that it allocates itself, the current stream."""
    return tbn._host is not None and tbn._recording is None and all(d is None for d in defaults)


def _done(st: int):
    if st != TBN_OK:
        _raise(st)


def tbn_kv_reserve(index: KVIndex, n_new: torch.Tensor, workspace: Optional[torch.Tensor] = None, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Room for n_new[s] more keys of each sequence; returns the pairs of pages (-1: none) for tbn_kv_copy_pages."""
    if type(index) is not KVIndex:
        _of(KVIndex, index, "index")
    if _plain(workspace, stream):
        r = tbn._host.kv_reserve(index._at, index._gpu, n_new)
        if r is not None:
            return r
    pairs = _empty((2, index.n_seqs), torch.int32, index.device, stream)
    ws, size = _workspace(index._ws, workspace, index.device, stream)
    at = pairs.data_ptr()
    _done(_call("tbn_kv_reserve", index._at, _ints(n_new, "n_new", index.n_seqs, index.device), at, at + 4 * index.n_seqs, ws, size, _stream(stream)))
    return pairs[0], pairs[1]


def tbn_kv_fork(index: KVIndex, parents: torch.Tensor, children: torch.Tensor, stream=None) -> None:
    """Sequence children[i], which is empty, shares the pages of parents[i]."""
    if type(index) is not KVIndex:
        _of(KVIndex, index, "index")
    if _plain(stream) and tbn._host.kv_fork(index._at, index._gpu, parents, children):
        return
    n = parents.numel()
    if children.numel() != n:
        raise ValueError("parents and children must have the same length")
    _done(_call("tbn_kv_fork", index._at, _ints(parents, "parents", 0, index.device), _ints(children, "children", 0, index.device), n, _stream(stream)))


def tbn_kv_release(index: KVIndex, keep: torch.Tensor, stream=None) -> None:
    """Sequence s keeps its first keep[s] keys at most and gives back the pages behind them."""
    if type(index) is not KVIndex:
        _of(KVIndex, index, "index")
    if _plain(stream) and tbn._host.kv_release(index._at, index._gpu, keep):
        return
    _done(_call("tbn_kv_release", index._at, _ints(keep, "keep", index.n_seqs, index.device), _stream(stream)))


def tbn_kv_compact(index: KVIndex, workspace: Optional[torch.Tensor] = None, stream=None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """Used pages go to the lowest numbers; returns (src, dst, count) for tbn_kv_copy_pages."""
    if type(index) is not KVIndex:
        _of(KVIndex, index, "index")
    half = max(index.n_pages // 2, 1)
    moves = _empty(2 * half + 1, torch.int32, index.device, stream)
    ws, size = _workspace(index._ws, workspace, index.device, stream)
    at = moves.data_ptr()
    _done(_call("tbn_kv_compact", index._at, at, at + 4 * half, at + 8 * half, ws, size, _stream(stream)))
    return moves[:half], moves[half:2 * half], moves[2 * half:]


def tbn_kv_copy_pages(pool: KVPool, src: torch.Tensor, dst: torch.Tensor, count: Optional[torch.Tensor] = None, stream=None) -> None:
    """Copies page src[i] to page dst[i], of the first count pairs if count is given; pairs with -1 are left out."""
    if type(pool) is not KVPool:
        _of(KVPool, pool, "pool")
    if _plain(stream) and tbn._host.kv_copy_pages(pool._at, pool._gpu, src, dst, count):
        return
    n = src.numel()
    if dst.numel() != n:
        raise ValueError("src and dst must have the same length")
    _done(_call("tbn_kv_copy_pages", pool._at, _ints(src, "src", 0, pool.device), _ints(dst, "dst", 0, pool.device), n,
                None if count is None else _ints(count, "count", 1, pool.device), _stream(stream)))


def tbn_kv_append(pool: KVPool, index: KVIndex, k_new: torch.Tensor, v_new: torch.Tensor, cu_new: torch.Tensor, max_new: int, stream=None) -> None:
    """Keys and values (tokens, kv_heads, dim) become the last cu_new[s + 1] - cu_new[s] <= max_new of each sequence."""
    if type(pool) is not KVPool or type(index) is not KVIndex:
        _of(KVPool, pool, "pool"), _of(KVIndex, index, "index")
    if _plain(stream) and tbn._host.kv_append(pool._at, pool._gpu, index._at, index._gpu, k_new, v_new, cu_new, max_new):
        return
    max_new, = _fit(max_new)
    _agree(pool, index)
    k, ks = _rows(k_new, "k_new", pool.kv_heads, pool.dim, pool)
    v, vs = _rows(v_new, "v_new", pool.kv_heads, pool.dim, pool)
    if k_new.shape[0] != v_new.shape[0]:
        raise ValueError("k_new and v_new must have the same number of tokens")
    _done(_call("tbn_kv_append", pool._at, index._at, k, ks, v, vs, _ints(cu_new, "cu_new", index.n_seqs + 1, index.device), k_new.shape[0], max_new, _stream(stream)))


def tbn_kv_keep(pool: KVPool, index: KVIndex, base: torch.Tensor, picks: torch.Tensor, counts: torch.Tensor, stream=None) -> None:
    """Key base[s] + picks[s, j] moves to base[s] + j for j < counts[s] (picks ascend)."""
    if type(pool) is not KVPool or type(index) is not KVIndex:
        _of(KVPool, pool, "pool"), _of(KVIndex, index, "index")
    if _plain(stream) and tbn._host.kv_keep(pool._at, pool._gpu, index._at, index._gpu, base, picks, counts):
        return
    _agree(pool, index)
    if picks.dim() != 2 or picks.shape[0] != index.n_seqs:
        raise ValueError("picks must be (n_seqs, width)")
    _done(_call("tbn_kv_keep", pool._at, index._at, _ints(base, "base", index.n_seqs, index.device), _ints(picks, "picks", 0, index.device),
                picks.shape[1], _ints(counts, "counts", index.n_seqs, index.device), _stream(stream)))


def _queries(q: torch.Tensor, pool, index: KVIndex, cu_q: torch.Tensor):
    _agree(pool, index)
    if q.dim() != 3 or q.shape[2] != pool.dim:
        raise ValueError(f"q must be (tokens, heads, {pool.dim})")
    at, stride = _rows(q, "q", q.shape[1], pool.dim, pool)
    return at, stride, _ints(cu_q, "cu_q", index.n_seqs + 1, index.device)


def _outputs(q: torch.Tensor, out: Optional[torch.Tensor], lse: Optional[torch.Tensor], stream):
    if out is None:
        out = _empty(q.shape, q.dtype, q.device, stream)
    elif out.shape != q.shape or out.dtype != q.dtype or out.device != q.device:
        raise ValueError("out must have q's shape, dtype and device")
    if lse is None:
        lse = _empty(q.shape[:2], torch.float32, q.device, stream)
    elif lse.shape != q.shape[:2] or lse.device != q.device:
        raise ValueError("lse must be (tokens, heads) on q's device")
    return out, lse


def tbn_tree_attention_workspace_bytes(q: torch.Tensor, pool: KVPool, index: KVIndex, max_q: int, max_len: int = 0) -> int:
    if type(pool) is not KVPool or type(index) is not KVIndex:
        _of(KVPool, pool, "pool"), _of(KVIndex, index, "index")
    max_q, = _fit(max_q)
    return int(lib().tbn_tree_attention_workspace_bytes(pool._at, index._at, q.shape[0], max_q, q.shape[1], _fit64(max_len)))


def tbn_tree_attention(q: torch.Tensor, pool: KVPool, index: KVIndex, cu_q: torch.Tensor, max_q: int, mask: Optional[torch.Tensor] = None,
                       scale: Optional[float] = None, max_len: Optional[int] = None, out: Optional[torch.Tensor] = None,
                       lse: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Queries q (tokens, heads, dim) of each sequence's last keys against its cache; mask int32 (tokens, words): bit j of a row
    is set where the token sees the sequence's j-th query token (None: its own and the earlier ones).  Returns (out, lse)."""
    if type(pool) is not KVPool or type(index) is not KVIndex:
        _of(KVPool, pool, "pool"), _of(KVIndex, index, "index")
    if _plain(out, lse, workspace, stream):
        r = tbn._host.tree_attention(q, pool._at, pool._gpu, index._at, index._gpu, cu_q, max_q, max_len, mask, scale)
        if r is not None:
            return r
    max_q, = _fit(max_q)
    at, stride, cu = _queries(q, pool, index, cu_q)
    out, lse = _outputs(q, out, lse, stream)
    words = 0
    if mask is not None:
        if mask.dim() != 2 or mask.shape[0] != q.shape[0]:
            raise ValueError("mask must be (tokens, words)")
        words = mask.shape[1]
        _same_device(q.device, mask)
    need = int(lib().tbn_tree_attention_workspace_bytes(pool._at, index._at, q.shape[0], max_q, q.shape[1], _fit64(max_len)))
    ws, size = _workspace(need, workspace, q.device, stream)
    _done(_call("tbn_tree_attention", at, stride, _dev(out, "out"), _dev(lse, "lse", torch.float32), pool._at, index._at, cu, q.shape[0], max_q, q.shape[1],
                None if mask is None else _dev(mask, "mask", torch.int32), words, _fit64(max_len), 1.0 / math.sqrt(pool.dim) if scale is None else scale, ws, size,
                _stream(stream)))
    return out, lse


def _mask(mask: Optional[torch.Tensor], q: torch.Tensor):
    """Address and words of a row of a mask, int32 (tokens, words)."""
    if mask is None:
        return None, 0
    if mask.dim() != 2 or mask.shape[0] != q.shape[0]:
        raise ValueError("mask must be (tokens, words)")
    _same_device(q.device, mask)
    return _dev(mask, "mask", torch.int32), mask.shape[1]


def tbn_window_attention_workspace_bytes(q: torch.Tensor, pool: KVPool, index: KVIndex, max_q: int, n_sink: int, window: int, masked: bool = False,
                                         max_len: int = 0) -> int:
    if type(pool) is not KVPool or type(index) is not KVIndex:
        _of(KVPool, pool, "pool"), _of(KVIndex, index, "index")
    max_q, n_sink, window = _fit(max_q, n_sink, window)
    return int(lib().tbn_window_attention_workspace_bytes(pool._at, index._at, q.shape[0], max_q, q.shape[1], n_sink, window, int(masked), _fit64(max_len)))


def tbn_window_attention(q: torch.Tensor, pool: KVPool, index: KVIndex, cu_q: torch.Tensor, max_q: int, n_sink: int, window: int,
                         mask: Optional[torch.Tensor] = None, scale: Optional[float] = None, max_len: Optional[int] = None,
                         out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                         stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """tbn_tree_attention over the sequence's first n_sink keys and the last `window` keys up to the token's own (with a mask: up to its place
    in the tree; then max_q <= window).  Returns (out, lse)."""
    if type(pool) is not KVPool or type(index) is not KVIndex:
        _of(KVPool, pool, "pool"), _of(KVIndex, index, "index")
    if _plain(out, lse, workspace, stream):
        r = tbn._host.window_attention(q, pool._at, pool._gpu, index._at, index._gpu, cu_q, max_q, max_len, mask, scale, n_sink, window)
        if r is not None:
            return r
    max_q, n_sink, window = _fit(max_q, n_sink, window)
    at, stride, cu = _queries(q, pool, index, cu_q)
    out, lse = _outputs(q, out, lse, stream)
    mask_at, words = _mask(mask, q)
    need = int(lib().tbn_window_attention_workspace_bytes(pool._at, index._at, q.shape[0], max_q, q.shape[1], n_sink, window, int(mask is not None), _fit64(max_len)))
    ws, size = _workspace(need, workspace, q.device, stream)
    _done(_call("tbn_window_attention", at, stride, _dev(out, "out"), _dev(lse, "lse", torch.float32), pool._at, index._at, cu, q.shape[0], max_q, q.shape[1],
                n_sink, window, mask_at, words, _fit64(max_len), 1.0 / math.sqrt(pool.dim) if scale is None else scale, ws, size, _stream(stream)))
    return out, lse


def tbn_block_select_workspace_bytes(q: torch.Tensor, pool: KVPool, index: KVIndex, max_q: int, max_len: int = 0) -> int:
    if type(pool) is not KVPool or type(index) is not KVIndex:
        _of(KVPool, pool, "pool"), _of(KVIndex, index, "index")
    max_q, = _fit(max_q)
    return int(lib().tbn_block_select_workspace_bytes(pool._at, index._at, q.shape[0], max_q, q.shape[1], _fit64(max_len)))


def tbn_block_select(q: torch.Tensor, pool: KVPool, index: KVIndex, cu_q: torch.Tensor, max_q: int, n_select: int, n_sink: int = 1, n_recent: int = 1,
                     max_len: Optional[int] = None, picks: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                     stream=None) -> torch.Tensor:
    """Per query and kv head n_select of its sequence's pages: int32 (tokens, kv_heads, n_select), ascending, -1 behind the last."""
    if type(pool) is not KVPool or type(index) is not KVIndex:
        _of(KVPool, pool, "pool"), _of(KVIndex, index, "index")
    if _plain(picks, workspace, stream):
        r = tbn._host.block_select(q, pool._at, pool._gpu, index._at, index._gpu, cu_q, max_q, max_len, n_select, n_sink, n_recent)
        if r is not None:
            return r
    max_q, n_select, n_sink, n_recent = _fit(max_q, n_select, n_sink, n_recent)
    at, stride, cu = _queries(q, pool, index, cu_q)
    shape = (q.shape[0], pool.kv_heads, n_select)
    if picks is None:
        picks = _empty(shape, torch.int32, q.device, stream)
    elif tuple(picks.shape) != shape or picks.device != q.device:
        raise ValueError(f"picks must be {shape} on {q.device}")
    need = int(lib().tbn_block_select_workspace_bytes(pool._at, index._at, q.shape[0], max_q, q.shape[1], _fit64(max_len)))
    ws, size = _workspace(need, workspace, q.device, stream)
    _done(_call("tbn_block_select", at, stride, _dev(picks, "picks", torch.int32), pool._at, index._at, cu, q.shape[0], max_q, q.shape[1], n_select, n_sink,
                n_recent, _fit64(max_len), ws, size, _stream(stream)))
    return picks


def tbn_block_attention_workspace_bytes(q: torch.Tensor, pool: KVPool, index: KVIndex, max_q: int, n_select: int) -> int:
    if type(pool) is not KVPool or type(index) is not KVIndex:
        _of(KVPool, pool, "pool"), _of(KVIndex, index, "index")
    max_q, n_select = _fit(max_q, n_select)
    return int(lib().tbn_block_attention_workspace_bytes(pool._at, index._at, q.shape[0], max_q, q.shape[1], n_select))


def tbn_block_attention(q: torch.Tensor, pool: KVPool, index: KVIndex, cu_q: torch.Tensor, max_q: int, picks: torch.Tensor, scale: Optional[float] = None,
                        out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                        stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """tbn_tree_attention without a mask over the keys of the picked pages only.  Returns (out, lse)."""
    if type(pool) is not KVPool or type(index) is not KVIndex:
        _of(KVPool, pool, "pool"), _of(KVIndex, index, "index")
    if _plain(out, lse, workspace, stream):
        r = tbn._host.block_attention(q, pool._at, pool._gpu, index._at, index._gpu, cu_q, max_q, None, picks, scale)
        if r is not None:
            return r
    max_q, = _fit(max_q)
    at, stride, cu = _queries(q, pool, index, cu_q)
    out, lse = _outputs(q, out, lse, stream)
    if picks.dim() != 3 or tuple(picks.shape[:2]) != (q.shape[0], pool.kv_heads):
        raise ValueError("picks must be (tokens, kv_heads, n_select)")
    _same_device(q.device, picks)
    n = picks.shape[2]
    need = int(lib().tbn_block_attention_workspace_bytes(pool._at, index._at, q.shape[0], max_q, q.shape[1], n))
    ws, size = _workspace(need, workspace, q.device, stream)
    _done(_call("tbn_block_attention", at, stride, _dev(out, "out"), _dev(lse, "lse", torch.float32), pool._at, index._at, cu, q.shape[0], max_q, q.shape[1],
                _dev(picks, "picks", torch.int32), n, 1.0 / math.sqrt(pool.dim) if scale is None else scale, ws, size, _stream(stream)))
    return out, lse


def tbn_kv4_append(pool: KV4Pool, index: KVIndex, k_new: torch.Tensor, v_new: torch.Tensor, cu_new: torch.Tensor, max_new: int, stream=None) -> None:
    """tbn_kv_append into a pool in 4 bits; k_new and v_new float32 or bfloat16."""
    if type(pool) is not KV4Pool or type(index) is not KVIndex:
        _of(KV4Pool, pool, "pool"), _of(KVIndex, index, "index")
    if _plain(stream) and tbn._host.kv4_append(pool._at, pool._gpu, index._at, index._gpu, k_new, v_new, cu_new, max_new):
        return
    max_new, = _fit(max_new)
    _agree(pool, index)
    k, ks = _rows(k_new, "k_new", pool.kv_heads, pool.dim, pool)
    v, vs = _rows(v_new, "v_new", pool.kv_heads, pool.dim, pool)
    if k_new.shape[0] != v_new.shape[0] or k_new.dtype != v_new.dtype:
        raise ValueError("k_new and v_new must have the same number of tokens and dtype")
    _done(_call("tbn_kv4_append", pool._at, index._at, k, ks, v, vs, _dt(k_new), _ints(cu_new, "cu_new", index.n_seqs + 1, index.device), k_new.shape[0], max_new,
                _stream(stream)))


def tbn_kv4_read(pool: KV4Pool, index: KVIndex, cu: torch.Tensor, max_n: int, total: int, dtype: torch.dtype = torch.bfloat16,
                 stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """The last cu[s + 1] - cu[s] <= max_n keys and values of each sequence, (total, kv_heads, dim) each, as the numbers they stand for (rows of
    a sequence that has fewer keys are undefined)."""
    if type(pool) is not KV4Pool or type(index) is not KVIndex:
        _of(KV4Pool, pool, "pool"), _of(KVIndex, index, "index")
    if dtype not in (torch.float32, torch.bfloat16):
        raise ValueError("dtype must be float32 or bfloat16")
    if _plain(stream):
        r = tbn._host.kv4_read(pool._at, pool._gpu, index._at, index._gpu, cu, max_n, total, dtype is torch.float32)
        if r is not None:
            return r
    max_n, = _fit(max_n)
    _agree(pool, index)
    k, v = (_empty((total, pool.kv_heads, pool.dim), dtype, pool.device, stream) for _ in range(2))
    _done(_call("tbn_kv4_read", pool._at, index._at, k.data_ptr(), v.data_ptr(), _dt(k), _ints(cu, "cu", index.n_seqs + 1, index.device), total, max_n, _stream(stream)))
    return k, v


def tbn_kv4_copy_pages(pool: KV4Pool, src: torch.Tensor, dst: torch.Tensor, count: Optional[torch.Tensor] = None, stream=None) -> None:
    """tbn_kv_copy_pages of a pool in 4 bits."""
    if type(pool) is not KV4Pool:
        _of(KV4Pool, pool, "pool")
    if _plain(stream) and tbn._host.kv4_copy_pages(pool._at, pool._gpu, src, dst, count):
        return
    n = src.numel()
    if dst.numel() != n:
        raise ValueError("src and dst must have the same length")
    _done(_call("tbn_kv4_copy_pages", pool._at, _ints(src, "src", 0, pool.device), _ints(dst, "dst", 0, pool.device), n,
                None if count is None else _ints(count, "count", 1, pool.device), _stream(stream)))


def tbn_kv4_keep(pool: KV4Pool, index: KVIndex, base: torch.Tensor, picks: torch.Tensor, counts: torch.Tensor, stream=None) -> None:
    """tbn_kv_keep of a pool in 4 bits."""
    if type(pool) is not KV4Pool or type(index) is not KVIndex:
        _of(KV4Pool, pool, "pool"), _of(KVIndex, index, "index")
    if _plain(stream) and tbn._host.kv4_keep(pool._at, pool._gpu, index._at, index._gpu, base, picks, counts):
        return
    _agree(pool, index)
    if picks.dim() != 2 or picks.shape[0] != index.n_seqs:
        raise ValueError("picks must be (n_seqs, width)")
    _done(_call("tbn_kv4_keep", pool._at, index._at, _ints(base, "base", index.n_seqs, index.device), _ints(picks, "picks", 0, index.device),
                picks.shape[1], _ints(counts, "counts", index.n_seqs, index.device), _stream(stream)))


def tbn_kv4_attention_workspace_bytes(q: torch.Tensor, pool: KV4Pool, index: KVIndex, max_q: int, n_sink: int = 0, window: int = 0, masked: bool = False,
                                      max_len: int = 0) -> int:
    if type(pool) is not KV4Pool or type(index) is not KVIndex:
        _of(KV4Pool, pool, "pool"), _of(KVIndex, index, "index")
    max_q, n_sink, window = _fit(max_q, n_sink, window)
    return int(lib().tbn_kv4_attention_workspace_bytes(pool._at, index._at, _dt(q), q.shape[0], max_q, q.shape[1], n_sink, window, int(masked), _fit64(max_len)))


def tbn_kv4_attention(q: torch.Tensor, pool: KV4Pool, index: KVIndex, cu_q: torch.Tensor, max_q: int, mask: Optional[torch.Tensor] = None,
                      n_sink: int = 0, window: int = 0, scale: Optional[float] = None, max_len: Optional[int] = None,
                      out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                      stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """tbn_tree_attention over a pool in 4 bits, with window > 0 tbn_window_attention; q float32 or bfloat16.  Returns (out, lse)."""
    if type(pool) is not KV4Pool or type(index) is not KVIndex:
        _of(KV4Pool, pool, "pool"), _of(KVIndex, index, "index")
    if _plain(out, lse, workspace, stream):
        r = tbn._host.kv4_attention(q, pool._at, pool._gpu, index._at, index._gpu, cu_q, max_q, max_len, mask, scale, n_sink, window)
        if r is not None:
            return r
    max_q, n_sink, window = _fit(max_q, n_sink, window)
    at, stride, cu = _queries(q, pool, index, cu_q)
    out, lse = _outputs(q, out, lse, stream)
    mask_at, words = _mask(mask, q)
    need = int(lib().tbn_kv4_attention_workspace_bytes(pool._at, index._at, _dt(q), q.shape[0], max_q, q.shape[1], n_sink, window, int(mask is not None), _fit64(max_len)))
    ws, size = _workspace(need, workspace, q.device, stream)
    _done(_call("tbn_kv4_attention", at, stride, _dt(q), _dev(out, "out"), _dev(lse, "lse", torch.float32), pool._at, index._at, cu, q.shape[0], max_q, q.shape[1],
                n_sink, window, mask_at, words, _fit64(max_len), 1.0 / math.sqrt(pool.dim) if scale is None else scale, ws, size, _stream(stream)))
    return out, lse


def _probabilities(t: torch.Tensor, name: str, like: Optional[torch.Tensor] = None) -> Tuple[int, int]:
    """Address and row stride of (tokens, vocab) float32 whose rows are dense."""
    if t.dim() != 2 or t.dtype != torch.float32 or (like is not None and t.shape != like.shape):
        raise ValueError(f"{name} must be float32 (tokens, vocab)")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    n, v = t.shape
    st = t.stride()
    if t.numel() and ((v > 1 and st[1] != 1) or (n > 1 and st[0] < v)):
        raise ValueError(f"{name}: rows must be dense and must not overlap (strides {st})")
    return t.data_ptr(), st[0] if n > 1 else v


def tbn_verify(target: torch.Tensor, tokens: torch.Tensor, u: torch.Tensor, cu_q: torch.Tensor, max_q: int, draft: Optional[torch.Tensor] = None,
               parents: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
               stream=None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """Which drafted tokens stand.  target and draft (tokens, vocab) float32 probabilities, tokens and parents int32, u float32, cu_q int32 (sequences + 1).
    Returns picks (sequences, max_q), counts and next (sequences), int32."""
    if _plain(workspace, stream):
        r = tbn._host.verify(target, tokens, u, cu_q, max_q, draft, parents)
        if r is not None:
            return r
    max_q, = _fit(max_q)
    dev, n_seqs = target.device, cu_q.numel() - 1
    p, ps = _probabilities(target, "target")
    q, qs = (None, 0) if draft is None else _probabilities(draft, "draft", target)
    _same_device(dev, draft, tokens, u, cu_q, parents)
    n, vocab = target.shape
    for t, name in ((tokens, "tokens"), (u, "u"), (parents, "parents")):
        if t is not None and t.numel() < n:
            raise ValueError(f"{name} has {t.numel()} entries, {n} needed")
    if n_seqs < 1 or max_q < 0:
        raise ValueError("cu_q must have an entry more than there are sequences, max_q must be >= 0")
    # sizes that the library refuses get no memory: the call below raises its error
    fine = max_q <= VERIFY_MAX_TOKENS and n_seqs <= MAX_SEQUENCES
    picks, counts, follows = (_empty(shape, torch.int32, dev, stream) for shape in (((n_seqs, max_q), (n_seqs,), (n_seqs,)) if fine else ((0,),) * 3))
    ws, size = _workspace(int(lib().tbn_verify_workspace_bytes(n, max_q, n_seqs, vocab)), workspace, dev, stream)
    _done(_call("tbn_verify", p, ps, q, qs, _dev(tokens, "tokens", torch.int32), None if parents is None else _dev(parents, "parents", torch.int32),
                _dev(u, "u", torch.float32), _dev(cu_q, "cu_q", torch.int32), n, max_q, n_seqs, vocab, picks.data_ptr(), counts.data_ptr(), follows.data_ptr(),
                ws, size, _stream(stream)))
    return picks, counts, follows
