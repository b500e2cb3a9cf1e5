"""The cache's calls through the extension module against the wrappers' own code, the forms that it leaves alone, bound calls, other
streams, a step of bookkeeping in a graph, and scales of any sign."""
import math

import numpy as np
import pytest
import torch

from oracle import kv_oracle as orc
from tests.kv_util import compare, make_cache, make_queries, tolerance

pytestmark = pytest.mark.gpu

H, KV, D, P = 8, 2, 64, 32


@pytest.fixture(scope="module")
def kv():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2407_12075_amd import kv as binding, tbn
    tbn.lib()
    assert tbn._host is not None
    return binding


def ints(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def cache(kv, seed=0, dt="bf16"):
    """Pages that begin as zeros, two sequences with keys, room for two more."""
    pool, index = kv.kv_pool(40, KV, D, P, {"f32": torch.float32, "bf16": torch.bfloat16}[dt], summary=True), kv.kv_index(4, 10, 40, P)
    for t in (pool.k, pool.v, pool.summary, pool.step):
        t.zero_()
    return pool, index


def life(kv, pool, index, stream=None):
    """Every call once or more; what it returned."""
    gen = torch.Generator().manual_seed(2)
    put = lambda *shape: torch.randn(*shape, generator=gen).to(pool.dtype).cuda()  # noqa: E731
    more = {} if stream is None else {"stream": stream}
    got = []

    def add(counts):
        pairs = kv.tbn_kv_reserve(index, ints(*counts), **more)
        kv.tbn_kv_copy_pages(pool, *pairs, **more)
        cu = ints(*np.concatenate([[0], np.cumsum(counts)]).tolist())
        qkv = put(sum(counts), H + 2 * KV, D)
        kv.tbn_kv_append(pool, index, qkv[:, H:H + KV], qkv[:, H + KV:], cu, max(counts), **more)
        got.extend(pairs)
        return qkv[:, :H], cu

    add([150, 70, 0, 0])
    kv.tbn_kv_fork(index, ints(0, 1), ints(2, 3), **more)
    q, cu = add([3, 5, 0, 2])
    mask = ints(1, 3, 5, 1, 3, 7, 9, 17, 1, 3).view(10, 1)
    got.extend(kv.tbn_tree_attention(q, pool, index, cu, 5, mask=mask, **more))
    got.extend(kv.tbn_tree_attention(q, pool, index, cu, 5, scale=0.3, max_len=160, **more))
    picks = kv.tbn_block_select(q, pool, index, cu, 5, 3, n_sink=0, n_recent=2, **more)
    got.extend((picks, *kv.tbn_block_attention(q, pool, index, cu, 5, picks, **more)))
    kv.tbn_kv_keep(pool, index, ints(150, 70, 150, 70), ints(0, 2, 0, 1, 2, 4, 0, 0, 1, 0, 0, 0).view(4, 3), ints(2, 3, 0, 1), **more)
    kv.tbn_kv_release(index, ints(152, 73, 0, 71), **more)
    moves = kv.tbn_kv_compact(index, **more)
    kv.tbn_kv_copy_pages(pool, *moves, **more)
    got.extend(m[:int(moves[2])] if m is not moves[2] else m for m in moves)
    return [t.clone() for t in got] + [index.table.clone(), index.lens.clone(), index.refs.clone(), index.status.clone()] + used(pool, index)


def used(pool, index):
    """What the sequences' pages hold of their keys."""
    out = []
    for s, n in enumerate(index.lens.tolist()):
        for b in range(-(-n // P)):
            p, r = int(index.table[s, b]), min(P, n - b * P)
            out += [pool.k[p, :, :r].clone(), pool.v[p, :, :, :r].clone()]
    return out


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("other", ["wrappers", "stream", "current stream"])
def test_the_same_by_every_way(kv, monkeypatch, dt, other):
    """float32 and bf16 results are the same to the bit: the same kernels in the same order, however they are called."""
    from paper_2407_12075_amd import tbn
    want = life(kv, *cache(kv, dt=dt))
    torch.cuda.synchronize()
    state = cache(kv, dt=dt)
    torch.cuda.synchronize()
    if other == "wrappers":
        monkeypatch.setattr(tbn, "_host", None)
        got = life(kv, *state)
    else:
        side = torch.cuda.Stream()
        if other == "stream":
            # inputs are made on the current stream, so each call's have to be there first
            real = {n: getattr(kv, n) for n in dir(kv) if n.startswith("tbn_kv_") or n in ("tbn_tree_attention", "tbn_block_select", "tbn_block_attention")}

            def waits(fn):
                def call(*args, **kw):
                    torch.cuda.synchronize()
                    r = fn(*args, **kw)
                    torch.cuda.synchronize()
                    return r
                return call
            for n, fn in real.items():
                monkeypatch.setattr(kv, n, waits(fn))
            got = life(kv, *state, stream=side)
        else:
            with torch.cuda.stream(side):
                got = life(kv, *state)
            side.synchronize()
    torch.cuda.synchronize()
    assert int(want[-1].numel()) and len(got) == len(want)
    for i, (a, b) in enumerate(zip(got, want)):
        assert a.shape == b.shape and torch.equal(a, b), i


def test_forms_left_to_the_wrappers(kv):
    """The extension module says None (or False) where a wrapper checks more, and launches nothing."""
    from paper_2407_12075_amd import tbn
    pool, index = cache(kv)
    q, cu, _ = make_queries("bf16", [1, 0, 0, 0], H, D)
    at = (pool._at, pool._gpu, index._at, index._gpu)
    host = tbn._host
    new = q[:, :KV].contiguous()
    base = [q, *at, cu, 1, None, None, None]
    for place, bad in ((0, q.float()), (0, q[:, :3]), (0, q[0]), (0, q.cpu()), (0, q[..., :32]), (0, None), (5, cu[:3]), (5, cu.long()), (5, cu.cpu()), (6, 1.0), (6, -1),
                       (7, "x"), (8, cu[:1]), (8, cu[:1].long().view(1, 1)), (8, torch.zeros(2, 1, dtype=torch.int32, device="cuda")), (9, "x")):
        args = list(base)
        args[place] = bad
        assert host.tree_attention(*args) is None, (place, bad)
    picks = torch.zeros(1, KV, 2, dtype=torch.int32, device="cuda")
    for bad in (picks.long(), picks[0], picks[:, :1], picks[:, :, :0], picks.cpu(), picks.transpose(1, 2)):
        assert host.block_attention(q, *at, cu, 1, None, bad, None) is None
    for bad in ((0, 0, 1), (5000, 1, 1), (2, -1, 1), (2, 1, 0), (2.0, 1, 1)):
        assert host.block_select(q, *at, cu, 1, None, *bad) is None
    assert not host.kv_append(*at, new, new.float(), cu, 1) and not host.kv_append(*at, new, q, cu, 1) and not host.kv_append(*at, new, new, cu[:2], 1)
    assert host.kv_reserve(*at[2:], ints(1, 1, 1)) is None and host.kv_reserve(*at[2:], ints(1, 1, 1, 1).long()) is None
    assert not host.kv_release(*at[2:], ints(1)) and not host.kv_fork(*at[2:], ints(1, 2), ints(3)) and not host.kv_copy_pages(*at[:2], ints(1, 2), ints(3), None)
    assert not host.kv_keep(*at, ints(0, 0, 0, 0), ints(0, 0, 0, 0), ints(0, 0, 0, 0)) and not host.kv_keep(*at, ints(0), ints(0, 0, 0, 0).view(4, 1), ints(0, 0, 0, 0))
    torch.cuda.synchronize()
    assert not index.lens.any() and not index.refs.any()
    # and the wrappers name what is wrong
    with pytest.raises(ValueError, match="q must be"):
        kv.tbn_tree_attention(q.float(), pool, index, cu, 1)
    with pytest.raises(ValueError, match="mask must be"):
        kv.tbn_tree_attention(q, pool, index, cu, 1, mask=cu[:1])
    with pytest.raises(ValueError, match="picks must be"):
        kv.tbn_block_attention(q, pool, index, cu, 1, picks[:, :1])
    with pytest.raises(ValueError, match="the same number"):
        kv.tbn_kv_append(pool, index, new, torch.cat([new, new]), cu, 1)
    with pytest.raises(RuntimeError):
        kv.tbn_block_select(q, pool, index, cu, 1, 0)


def test_bound_calls(kv):
    from paper_2407_12075_amd import tbn
    pool, index, keys, values = make_cache(kv, "bf16", KV, D, P, [100, 40], seed=4)
    q, cu, _ = make_queries("bf16", [1, 1], H, D)
    again = tbn.tbn_bind(kv.tbn_tree_attention, q, pool, index, cu, 1)
    for i in range(3):
        q.copy_(make_queries("bf16", [1, 1], H, D, seed=30 + i)[0])
        out, lse = (t.clone() for t in again())
        want, want_lse = kv.tbn_tree_attention(q, pool, index, cu, 1)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, want_lse)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("scale", [0.0, -0.2, 1.0])
def test_scales(kv, dt, scale):
    counts, lens = [3, 1], [70, 200]
    pool, index, keys, values = make_cache(kv, dt, KV, D, P, lens, seed=6)
    q, cu, qs = make_queries(dt, counts, H, D, scale=0.5)
    out, lse = kv.tbn_tree_attention(q, pool, index, cu, 3, scale=scale)
    want, want_lse, at = np.zeros(qs.shape), np.zeros(qs.shape[:2]), 0
    for s, n in enumerate(counts):
        for t in range(n):
            see = np.arange(lens[s]) <= lens[s] - n + t
            for h in range(H):
                want[at, h], want_lse[at, h] = orc.attention(qs[at, h], keys[s][:, h * KV // H], values[s][:, h * KV // H], see, scale)
            at += 1
    compare(out, lse, want, want_lse, tolerance(dt, values))


def test_a_step_of_bookkeeping_in_a_graph(kv):
    """reserve, copies, append, attention, keep and release captured once and replayed with other tokens; a twin cache runs the same
    calls eagerly between the replays."""
    twins = [cache(kv, dt="f32") for _ in range(2)]
    start = torch.randn(160, 2 * KV, D, generator=torch.Generator().manual_seed(1)).cuda()
    for pool, index in twins:
        kv.tbn_kv_reserve(index, ints(100, 60, 0, 0))
        kv.tbn_kv_append(pool, index, start[:, :KV].contiguous(), start[:, KV:].contiguous(), ints(0, 100, 160, 160, 160), 100)
        kv.tbn_kv_fork(index, ints(0), ints(2))
    new, counts, cu = torch.zeros(12, H + 2 * KV, D, device="cuda"), ints(4, 4, 4, 0), ints(0, 4, 8, 12, 12)
    picks, many = ints(*([0, 2] * 4)).view(4, 2), ints(2, 1, 2, 0)

    def step(pool, index):
        base = index.lens.clone()
        pairs = kv.tbn_kv_reserve(index, counts)
        kv.tbn_kv_copy_pages(pool, *pairs)
        kv.tbn_kv_append(pool, index, new[:, H:H + KV], new[:, H + KV:], cu, 4)
        out = kv.tbn_tree_attention(new[:, :H], pool, index, cu, 4)
        kv.tbn_kv_keep(pool, index, base, picks, many)
        kv.tbn_kv_release(index, base + many)
        return out

    pool, index = twins[0]
    saved = [t.clone() for t in (index.table, index.lens, index.refs, pool.k, pool.v, pool.summary, pool.step)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(pool, index)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    for t, was in zip((index.table, index.lens, index.refs, pool.k, pool.v, pool.summary, pool.step), saved):
        t.copy_(was)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = step(pool, index)
    for i in range(5):
        new.copy_(torch.randn(new.shape, generator=torch.Generator().manual_seed(50 + i)))
        graph.replay()
        torch.cuda.synchronize()
        got = [out.clone(), lse.clone(), index.lens.clone(), index.refs.clone()] + used(pool, index)
        want_out = step(*twins[1])
        torch.cuda.synchronize()
        want = [*want_out, twins[1][1].lens, twins[1][1].refs] + used(*twins[1])
        assert int(index.status) == 0 and all(torch.equal(a, b) for a, b in zip(got, want)), i
    assert index.lens.tolist() == [110, 65, 110, 0]
