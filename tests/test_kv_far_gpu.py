"""Pools, and rows of probabilities, whose offsets pass 32 bits: a window's pages, the cache in 4 bits, the verification."""
import math

import numpy as np
import pytest
import torch

from oracle import kv4_oracle as o4
from oracle.verify_oracle import verify as oracle
from tests.kv_util import compare, make_cache, make_queries, tolerance
from tests.test_kv_window_gpu import reference

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kv():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2407_12075_amd import kv as binding, tbn
    tbn.lib()
    return binding


def ints(*x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("dt,tokens", [("f32", 1), ("bf16", 1), ("bf16", 40)])
def test_window(kv, dt, tokens):
    KV, D, P = 4, 128, 128
    n_pages = (1 << 33) // (KV * D * P * 4) + 60   # 8 GiB of float32 keys, 4 of bfloat16
    pool, index, keys, values = make_cache(kv, dt, KV, D, P, [3000 + tokens], seed=3, n_pages=n_pages, far=True)
    assert pool.k.numel() * pool.k.element_size() > 1 << 32
    q, cu, qs = make_queries(dt, [tokens], 2 * KV, D)
    out, lse = kv.tbn_window_attention(q, pool, index, cu, tokens, 130, 900)
    compare(out, lse, *reference(qs, keys, values, [tokens], 130, 900, None, 1 / math.sqrt(D)), tolerance(dt, values))


def test_cache_in_4_bits(kv):
    KV, D, P, n = 8, 256, 128, 700
    n_pages = (1 << 32) // (KV * P * D // 2) + 300
    pool = kv.kv4_pool(n_pages, KV, D, P)
    assert pool.k.numel() > (1 << 32) + (1 << 24)
    index = kv.kv_index(1, 8, n_pages, P)
    pages = [n_pages - 1 - 3 * i for i in range(7)]
    index.table[0, :7] = ints(*pages)
    index.lens.fill_(n)
    rng = np.random.RandomState(1)
    k, v = (torch.from_numpy(rng.standard_normal((n, KV, D))).to(torch.bfloat16) for _ in range(2))
    kv.tbn_kv4_append(pool, index, k.cuda(), v.cuda(), ints(0, n), n)
    kr, vr = kv.tbn_kv4_read(pool, index, ints(0, n), n, n, torch.float32)
    some = [0, 1, 31, 127, 128, 400, 699]
    for t in some:
        codes = o4.quantize(k[t].double().numpy(), v[t].double().numpy())
        assert np.array_equal(kr[t].double().cpu().numpy(), o4.numbers(codes[0], codes[2]))
        assert np.array_equal(vr[t].double().cpu().numpy(), o4.numbers(codes[1], codes[3]))
    keys, values = [kr.double().cpu().numpy()], [vr.double().cpu().numpy()]
    for dt, H, T, window in (("bf16", 8, 1, 0), ("f32", 16, 3, 200), ("bf16", 32, 20, 0)):
        q, cu, qs = make_queries(dt, [T], H, D)
        out, lse = kv.tbn_kv4_attention(q, pool, index, cu, T, n_sink=2, window=window)
        compare(out, lse, *reference(qs, keys, values, [T], 2, window or 1 << 30, None, 1 / math.sqrt(D)), tolerance(dt, values))
    # to the pool's first pages and back to other last ones
    kv.tbn_kv4_copy_pages(pool, ints(*pages), ints(*range(7)))
    kv.tbn_kv4_copy_pages(pool, ints(*range(7)), ints(*[p - 1 for p in pages]))
    index.table[0, :7] = ints(*[p - 1 for p in pages])
    for t in (pool.k, pool.v, pool.k_exp, pool.v_exp):
        t[pages] = 0
    k2, v2 = kv.tbn_kv4_read(pool, index, ints(0, n), n, n, torch.float32)
    assert torch.equal(k2, kr) and torch.equal(v2, vr)
    picks = list(range(1, 200, 2))
    kv.tbn_kv4_keep(pool, index, ints(500), ints(*picks).view(1, -1), ints(len(picks)))
    k2, v2 = kv.tbn_kv4_read(pool, index, ints(0, n), n, n, torch.float32)
    assert torch.equal(k2[500:600], kr[[500 + p for p in picks]]) and torch.equal(v2[500:600], vr[[500 + p for p in picks]])
    assert torch.equal(k2[:500], kr[:500]) and torch.equal(v2[600:], vr[600:])


@pytest.mark.parametrize("V", [100, 40000])
def test_verification(kv, V):
    stride, T = (1 << 30) + 3, 4
    rng = np.random.RandomState(2)
    p, q = rng.dirichlet(np.ones(V) * 0.1, T).astype(np.float32), rng.dirichlet(np.ones(V) * 0.1, T).astype(np.float32)
    wide = torch.empty((T - 1) * stride + 2 * V, device="cuda")
    target, draft = wide.as_strided((T, V), (stride, 1)), wide.as_strided((T, V), (stride, 1), V)
    target.copy_(torch.from_numpy(p))
    draft.copy_(torch.from_numpy(q))
    tokens, parents = rng.randint(0, V, T).astype(np.int32), np.array([-1, 0, 0, 2], np.int32)
    tokens[2], tokens[3] = int(p[0].argmax()), int(p[2].argmax())
    for seed in range(6):
        u = np.random.RandomState(seed).rand(T).astype(np.float32) * np.array([1, 1, 0.01, 1], np.float32)
        picks, counts, follows = kv.tbn_verify(target, ints(*tokens), torch.from_numpy(u).cuda(), ints(0, T), T, draft=draft, parents=ints(*parents))
        path, token = oracle(p, q, tokens, parents, u)
        assert picks[0, :len(path)].tolist() == path and int(counts[0]) == len(path) and int(follows[0]) == token
