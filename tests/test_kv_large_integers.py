"""Integers beyond 32 (max_len: 64) bits in the cache's calls, on the CPU: a window that is longer than any sequence is no window, and a number that has to be at least another
is; none reaches the library cut to its low bits."""
import ctypes

import pytest
import torch

from tests.test_kv_abi import FAKE, lib  # noqa: F401  (lib is a fixture)
from tests.test_kv_kinds import held
from tests.test_kv_more_abi import pool4

BIG = (1 << 31) - 1


@pytest.fixture()
def objects(lib):  # noqa: F811
    """Long sequences: their keys are split unless a window is short."""
    from paper_2407_12075_amd import kv
    sizes = dict(n_pages=1 << 20, kv_heads=2, dim=64, page=32)
    index = dict(n_pages=1 << 20, n_seqs=3, max_pages=4000, page=32)
    fake = dict(k=FAKE, v=FAKE)
    return (held(kv.KVPool, kv._Pool(**fake, summary=FAKE, step=FAKE, dt=0, **sizes), dtype=torch.float32, **sizes),
            held(kv.KV4Pool, pool4(**sizes), dtype=None, **sizes), held(kv.KVIndex, kv._Index(table=FAKE, lens=FAKE, refs=FAKE, status=FAKE, **index), **index))


def test_workspaces(objects):
    from paper_2407_12075_amd import kv
    pool, four, index = objects
    q = torch.zeros(3, 4, 64)
    for fn, p in ((kv.tbn_window_attention_workspace_bytes, pool), (kv.tbn_kv4_attention_workspace_bytes, four)):
        ask = lambda most, sink, window, *more: fn(q, p, index, most, sink, window, *more)  # noqa: E731
        want = ask(1, 4, BIG)
        assert want > 0 and ask(1, 4, 64) != want
        assert ask(1, 4, 1 << 32 | 64) == ask(1, 4, 1 << 31) == ask(1, 4, 1 << 70) == want
        assert ask(1, 1 << 32 | 4, 64) == ask(1, BIG, 64) == want
        assert ask(1 << 32 | 1, 4, BIG) == ask(3, 4, BIG)
        assert ask(1, -(1 << 32) + 4, BIG) == 0 and ask(1, 4, -(1 << 32) + 64) == 0
        assert ask(1, 4, BIG, False, 1 << 64 | 100) == 0   # beyond what a sequence has room for
    for fn in (kv.tbn_tree_attention_workspace_bytes, kv.tbn_block_select_workspace_bytes):
        assert fn(q, pool, index, 1 << 32 | 1) == fn(q, pool, index, 3) > 0 and fn(q, pool, index, 3, 1 << 64 | 100) == 0
    assert kv.tbn_block_attention_workspace_bytes(q, pool, index, 1 << 32 | 1, 4) == kv.tbn_block_attention_workspace_bytes(q, pool, index, 3, 4)
    assert kv.tbn_block_attention_workspace_bytes(q, pool, index, 3, 1 << 32 | 4) == 0


class Arrived(Exception):
    pass


@pytest.mark.parametrize("host", [False, True])
def test_calls(objects, host, monkeypatch):
    """What arrives at the library, with the tensors' checks left out."""
    from paper_2407_12075_amd import kv, tbn
    pool, four, index = objects
    q, k, i = torch.zeros(3, 4, 64), torch.zeros(3, 2, 64), torch.zeros(9, dtype=torch.int32)

    def arrive(name, *args):
        types = getattr(tbn.lib(), name).argtypes
        bits = {ctypes.c_int32: 31, ctypes.c_int64: 63}
        for a, t in zip(args, types):
            if t in bits:
                assert -1 << bits[t] <= a < 1 << bits[t], (name, a)
        raise Arrived([a for a, t in zip(args, types) if t is ctypes.c_int32])   # a type (float32: 0) among them

    monkeypatch.setattr(kv, "_call", arrive)
    if not host or tbn._host is None:
        monkeypatch.setattr(tbn, "_host", None)
    monkeypatch.setattr(kv, "_queries", lambda *a: (FAKE, 256, FAKE))
    monkeypatch.setattr(kv, "_outputs", lambda *a: (q, q))
    monkeypatch.setattr(kv, "_rows", lambda *a: (FAKE, 128))
    monkeypatch.setattr(kv, "_dev", lambda *a: FAKE)
    monkeypatch.setattr(kv, "_empty", lambda *a, **kw: q)
    monkeypatch.setattr(kv, "_ints", lambda *a: FAKE)
    monkeypatch.setattr(kv, "_workspace", lambda *a: (FAKE, 1 << 60))
    monkeypatch.setattr(kv, "_stream", lambda s: None)
    far, near = 1 << 32 | 5, BIG
    for call, numbers in (
            (lambda x: kv.tbn_kv_append(pool, index, k, k, i, x), [near]), (lambda x: kv.tbn_kv4_append(four, index, k, k, i, x), [0, near]),
            (lambda x: kv.tbn_kv4_read(four, index, i, x, 3), [0, near]), (lambda x: kv.tbn_tree_attention(q, pool, index, i, x, max_len=x << 40), [near, 4, 0]),
            (lambda x: kv.tbn_window_attention(q, pool, index, i, x, x, x, max_len=x << 40), [near, 4, near, near, 0]),
            (lambda x: kv.tbn_kv4_attention(q, four, index, i, x, n_sink=x, window=x, max_len=x << 40), [0, near, 4, near, near, 0]),
            (lambda x: kv.tbn_block_attention(q, pool, index, i, x, torch.zeros(3, 2, 4)), [near, 4, 4]),
            (lambda x: kv.tbn_block_select(q, pool, index, i, x, x, x, x, max_len=x << 40), [near, 4, near, near, near])):
        with pytest.raises(Arrived) as e:
            call(far)
        assert e.value.args[0] == numbers
        with pytest.raises(Arrived):
            call(-far)
