"""Attention over the cache with a sliding window and first keys that stay visible, against the float64 oracle: windows that end inside
pages and steps, begin before the sequence, leave a row nothing; prompts, trees, single tokens; infinities and not-a-numbers outside of
windows; strides, idle places of the index, streams, graphs."""
import math

import numpy as np
import pytest
import torch

from oracle import kv_oracle as orc
from tests.kv_util import compare, make_cache, make_queries, pack_mask, tolerance
from tests.test_kv_attention_gpu import masks

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kv():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2407_12075_amd import kv as binding, tbn
    tbn.lib()
    return binding


def seen_keys(L, T, t, sink, window, row):
    """Which of L keys token t of the last T sees; row: its mask among the T, None for its own and the earlier ones."""
    prefix = L - T
    key = np.arange(L)
    if row is None:
        at = prefix + t
        return (key <= at) & ((key < sink) | (key > at - window))
    at = prefix + int(row.sum()) - 1
    see = (key < sink) | (key > at - window)
    see[prefix:] = row
    return see


def reference(qs, keys, values, counts, sink, window, see, scale):
    H = qs.shape[1]
    out, lse = np.zeros(qs.shape), np.zeros(qs.shape[:2])
    i = 0
    for s, n in enumerate(counts):
        k, v = keys[s], values[s]
        G = H // k.shape[1]
        for t in range(n):
            row = seen_keys(len(k), n, t, sink, window, None if see is None else see[s][t])
            for h in range(H):
                out[i, h], lse[i, h] = orc.attention(qs[i, h], k[:, h // G], v[:, h // G], row, scale)
            i += 1
    return out, lse


def packed(see, counts):
    words = -(-max(counts) // 32)
    return pack_mask(np.concatenate([np.pad(m, ((0, 0), (0, words * 32 - m.shape[1]))) for m in see]), words)


CASES = [
    # heads, kv heads, dim, page, [(keys before, tokens)]
    (4, 1, 64, 32, [(0, 1), (30, 1), (31, 1), (32, 1), (63, 2)]),
    (8, 2, 128, 64, [(62, 1), (64, 1), (65, 1), (700, 3), (0, 5)]),
    (6, 6, 64, 32, [(297, 13), (5, 7), (0, 0), (33, 1)]),
    (5, 1, 128, 128, [(127, 1), (128, 1), (900, 4)]),
    (4, 2, 80, 32, [(350, 9), (100, 2)]),
    (2, 1, 8, 32, [(240, 6), (0, 3)]),
    (2, 1, 256, 64, [(377, 6), (10, 1)]),
    (8, 1, 96, 64, [(450, 70), (0, 40)]),                                   # several tiles of rows
    (4, 1, 128, 32, [(390, 33), (813, 32)]),
]


@pytest.mark.parametrize("sink,window", [(0, 1), (4, 1), (0, 75), (3, 75), (64, 97), (65, 128), (5, 100000), (2000000000, 2), (0, 2147483647)])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("H,KV,D,P,seqs", CASES)
def test_window(kv, H, KV, D, P, seqs, dt, sink, window):
    counts = [n for _, n in seqs]
    pool, index, keys, values = make_cache(kv, dt, KV, D, P, [p + n for p, n in seqs], seed=H * D)
    q, cu, qs = make_queries(dt, counts, H, D)
    scale = 1.0 / math.sqrt(D)
    out, lse = kv.tbn_window_attention(q, pool, index, cu, max(counts), sink, window)
    compare(out, lse, *reference(qs, keys, values, counts, sink, window, None, scale), tolerance(dt, values))
    out2, lse2 = kv.tbn_window_attention(q, pool, index, cu, max(counts), sink, window, scale=scale, max_len=max(p + n for p, n in seqs))
    compare(out2, lse2, out.double().cpu().numpy(), lse.double().cpu().numpy(), tolerance(dt, values))
    if max(counts) > window:
        return
    for kind in ("tree", "any"):   # rows without a bit among the second
        see = masks(kind, counts, 3)
        out, lse = kv.tbn_window_attention(q, pool, index, cu, max(counts), sink, window, mask=packed(see, counts))
        compare(out, lse, *reference(qs, keys, values, counts, sink, window, see, scale), tolerance(dt, values))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("H,KV,D,P,seqs,sink,window", [
    (8, 2, 128, 64, [(5000, 1)], 4, 3000), (4, 1, 64, 32, [(7000, 11), (100, 2), (0, 1)], 70, 4097), (2, 1, 256, 128, [(3000, 3)], 1, 2000),
    (16, 1, 64, 64, [(5500, 20)], 300, 1500), (64, 64, 128, 64, [(2500, 1), (1, 1), (2023, 2), (0, 0), (64, 1), (2, 2), (130, 1), (640, 1)], 4, 1500),
    (4, 2, 64, 64, [(1000, 600)], 4, 130), (4, 2, 128, 128, [(300, 500), (0, 260)], 0, 70)])
def test_long_windows_and_prompts(kv, H, KV, D, P, seqs, sink, window, dt):
    """Keys split over workgroups, many tiles of rows; the same results from run to run."""
    counts = [n for _, n in seqs]
    pool, index, keys, values = make_cache(kv, dt, KV, D, P, [p + n for p, n in seqs], seed=5)
    q, cu, qs = make_queries(dt, counts, H, D)
    out, lse = kv.tbn_window_attention(q, pool, index, cu, max(counts), sink, window)
    compare(out, lse, *reference(qs, keys, values, counts, sink, window, None, 1 / math.sqrt(D)), tolerance(dt, values))
    again, lse2 = kv.tbn_window_attention(q, pool, index, cu, max(counts), sink, window)
    assert torch.equal(out, again) and torch.equal(lse, lse2)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("H,KV,D,P", [(4, 2, 64, 32), (32, 1, 128, 64), (8, 1, 256, 128)])
def test_what_is_outside_of_the_window_has_no_part(kv, H, KV, D, P, dt):
    """Keys and values that are not finite, before the window and behind the last key; one within: as the definition has it."""
    seqs, sink, window = [(400, 3), (259, 1)], 2, 133
    counts = [n for _, n in seqs]
    pool, index, keys, values = make_cache(kv, dt, KV, D, P, [p + n for p, n in seqs], seed=6)
    q, cu, qs = make_queries(dt, counts, H, D)
    for s, (p, n) in enumerate(seqs):
        for at, x in ((sink, math.inf), (sink + 40, math.nan), (p + 1 - window, -math.inf), (p - window, math.nan), (p + n - window - 1, math.nan)):
            page = int(index.table[s, at // P])
            pool.v[page, :, :, at % P] = x
            pool.k[page, :, at % P] = math.nan if at < p - window else pool.k[page, :, at % P]
            values[s][at] = x
            if at < p - window:
                keys[s][at] = math.nan
    out, lse = kv.tbn_window_attention(q, pool, index, cu, max(counts), sink, window)
    ref = reference(qs, keys, values, counts, sink, window, None, 1 / math.sqrt(D))
    assert np.isnan(ref[0]).any() or np.isinf(ref[0]).any()
    assert np.isfinite(ref[0]).any()
    compare(out, lse, *ref, tolerance(dt, values))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_wide_window_is_full_attention(kv, dt):
    """No key is left out: what tbn_tree_attention gives, to the bit where the keys are split alike."""
    counts = [3, 1]
    pool, index, _, values = make_cache(kv, dt, 2, 64, 32, [200, 90], seed=7)
    q, cu, _ = make_queries(dt, counts, 8, 64, stride=8 * 64 + 24)
    a, la = kv.tbn_window_attention(q, pool, index, cu, 3, 0, 1 << 20)
    b, lb = kv.tbn_tree_attention(q, pool, index, cu, 3)
    assert torch.equal(a, b) and torch.equal(la, lb)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_idle_places_streams_and_outputs(kv, dt):
    """An index with more places than the call has sequences; the caller's outputs and workspace, another stream, a negative scale."""
    lens = [0] * 20 + [5000] + [0] * 10 + [40]
    counts = [0] * 20 + [1] + [0] * 10 + [1]
    pool, index, keys, values = make_cache(kv, dt, 2, 128, 64, lens, seed=9)
    q, cu, qs = make_queries(dt, counts, 8, 128)
    ref = reference(qs, keys, values, counts, 4, 2500, None, -0.07)
    out, lse = kv.tbn_window_attention(q, pool, index, cu, 1, 4, 2500, scale=-0.07)
    compare(out, lse, *ref, tolerance(dt, values))
    need = kv.tbn_window_attention_workspace_bytes(q, pool, index, 1, 4, 2500)
    assert need > 0
    mine, mine_lse = torch.full_like(out, 7.0), torch.full_like(lse, 7.0)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    r = kv.tbn_window_attention(q, pool, index, cu, 1, 4, 2500, scale=-0.07, out=mine, lse=mine_lse, workspace=torch.empty(need, dtype=torch.uint8, device="cuda"), stream=side)
    side.synchronize()
    assert r[0] is mine and torch.equal(mine, out) and torch.equal(mine_lse, lse)
    with pytest.raises(RuntimeError):
        kv.tbn_window_attention(q, pool, index, cu, 1, 4, 2500, workspace=torch.empty(need - 16, dtype=torch.uint8, device="cuda"))


def test_graph(kv):
    """Captured and replayed with other keys in the cache and other lengths."""
    pool, index, keys, values = make_cache(kv, "bf16", 2, 128, 64, [3000, 1500], seed=11, n_pages=90, max_pages=60)
    q, cu, qs = make_queries("bf16", [1, 1], 8, 128)
    kv.tbn_window_attention(q, pool, index, cu, 1, 4, 1000)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out, lse = kv.tbn_window_attention(q, pool, index, cu, 1, 4, 1000)
    for lens in ([3000, 1500], [2990, 1], [40, 1300]):
        index.lens.copy_(torch.tensor(lens, dtype=torch.int32))
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        want, want_lse = kv.tbn_window_attention(q, pool, index, cu, 1, 4, 1000)
        assert torch.equal(out, want) and torch.equal(lse, want_lse)
        compare(out, lse, *reference(qs, [k[:n] for k, n in zip(keys, lens)], [v[:n] for v, n in zip(values, lens)], [1, 1], 4, 1000, None, 1 / math.sqrt(128)),
                tolerance("bf16", values))


def test_refusals(kv):
    from paper_2407_12075_amd import tbn
    pool, index, _, _ = make_cache(kv, "bf16", 2, 64, 32, [50, 60])
    q, cu, _ = make_queries("bf16", [3, 2], 4, 64)
    mask = torch.ones(5, 1, dtype=torch.int32, device="cuda")
    for kw in (dict(n_sink=-1, window=5), dict(n_sink=0, window=0), dict(n_sink=0, window=2, mask=mask)):
        with pytest.raises(tbn.TbnError) as e:
            kv.tbn_window_attention(q, pool, index, cu, 3, **kw)
        assert e.value.status == 2
    kv.tbn_window_attention(q, pool, index, cu, 3, 0, 3, mask=mask)
    for bad in (mask.long(), mask[:4], mask.flatten(), mask.cpu()):
        with pytest.raises(ValueError):
            kv.tbn_window_attention(q, pool, index, cu, 3, 0, 3, mask=bad)
    with pytest.raises(ValueError):
        kv.tbn_window_attention(q.float(), pool, index, cu, 3, 0, 3)
