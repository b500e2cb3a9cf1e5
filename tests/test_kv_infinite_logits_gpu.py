"""Logits that are infinite or not a number, in every kernel of the attention over the cache: lse is the logarithm of the sum as it is, infinite where a
logit is, and rows that do not see such a key are as without it."""
import math

import numpy as np
import pytest
import torch

from tests.kv_util import compare, make_cache, make_queries, tolerance
from tests.test_kv_attention_gpu import block_reference, masks, reference

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kv():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2407_12075_amd import kv as binding, tbn
    tbn.lib()
    return binding


def check(got, ref, ref_lse, tol):
    compare(*got, ref, ref_lse, tol)
    lse = got[1].double().cpu().numpy()
    assert np.array_equal(np.isnan(lse), np.isnan(ref_lse)) and np.array_equal(np.isposinf(lse), np.isposinf(ref_lse))


def put(pool, index, keys, values, P, key, d, x, value=False):
    page = int(index.table[0, key // P])
    if value:
        values[0][key, :, d] = x
        pool.v[page, :, d, key % P] = x
    else:
        keys[0][key, :, d] = x
        pool.k[page, :, key % P, d] = x


def positive(q, qs, channels):
    """Queries with the given channels above 0, so that an infinite key there makes an infinite logit of its sign."""
    for d in channels:
        qs[:, :, d] = np.abs(qs[:, :, d]) + 0.25
    qs = torch.from_numpy(qs).to(q.dtype).double().numpy()
    q.copy_(torch.from_numpy(qs))
    return qs


FORMS = [
    # dt, heads, kv heads, dim, page, keys before, tokens: one workgroup; parts; more rows; the staged kernel's 64 and 128 rows
    ("f32", 4, 2, 64, 32, 45, 5), ("bf16", 4, 2, 64, 32, 45, 5), ("f32", 4, 2, 128, 64, 3000, 3), ("bf16", 4, 2, 128, 64, 3000, 3), ("bf16", 2, 1, 64, 64, 7000, 2),
    ("f32", 4, 1, 64, 32, 45, 24), ("f32", 2, 2, 256, 64, 100, 4), ("bf16", 4, 1, 64, 32, 45, 12), ("bf16", 2, 1, 128, 64, 700, 50), ("bf16", 2, 1, 256, 64, 45, 40),
    ("bf16", 4, 1, 96, 32, 45, 12),
]


@pytest.mark.parametrize("dt,H,KV,D,P,prefix,T", FORMS)
def test_logits_of_any_kind(kv, dt, H, KV, D, P, prefix, T):
    """Cached keys are seen by all: first an infinite one among the drafted, then one in the cache, then a not-a-number beside it."""
    pool, index, keys, values = make_cache(kv, dt, KV, D, P, [prefix + T], seed=2)
    q, cu, qs = make_queries(dt, [T], H, D)
    qs = positive(q, qs, (0, 3, 7))
    see = [np.tril(np.ones((T, T), bool))]

    def once():
        ref = reference(qs, keys, values, [T], see, 1 / math.sqrt(D))
        check(kv.tbn_tree_attention(q, pool, index, cu, T), *ref, tolerance(dt, values))
        return ref[1]
    put(pool, index, keys, values, P, prefix + T - 1, 3, math.inf)
    lse = once()
    assert np.isposinf(lse[-1]).all() and np.isfinite(lse[:-1]).all()
    put(pool, index, keys, values, P, prefix // 2, 7, -math.inf)   # a weight of 0
    lse = once()
    assert np.isposinf(lse[-1]).all() and np.isfinite(lse[:-1]).all()
    put(pool, index, keys, values, P, prefix + 1, 0, math.inf)
    lse = once()
    assert np.isposinf(lse[1:]).all() and np.isfinite(lse[0]).all()
    put(pool, index, keys, values, P, prefix // 3, 3, math.inf)
    put(pool, index, keys, values, P, prefix + T - 1, 7, math.nan)
    lse = once()
    assert np.isnan(lse[-1]).all() and np.isposinf(lse[:-1]).all()


@pytest.mark.parametrize("dt,H,KV,D,P,T", [("f32", 4, 2, 64, 32, 3), ("bf16", 4, 2, 64, 32, 3), ("bf16", 4, 1, 128, 64, 20)])
def test_every_logit_minus_infinity(kv, dt, H, KV, D, P, T):
    prefix = 0
    pool, index, keys, values = make_cache(kv, dt, KV, D, P, [prefix + T], seed=2)
    q, cu, qs = make_queries(dt, [T], H, D)
    qs = positive(q, qs, (5,))
    for j in range(T - 1):
        put(pool, index, keys, values, P, j, 5, -math.inf)
    ref = reference(qs, keys, values, [T], [np.tril(np.ones((T, T), bool))], 1 / math.sqrt(D))
    assert np.isneginf(ref[1][:-1]).all() and (ref[0][:-1] == 0).all() and np.isfinite(ref[1][-1]).all()
    check(kv.tbn_tree_attention(q, pool, index, cu, T), *ref, tolerance(dt, values))


@pytest.mark.parametrize("dt,T", [("f32", 5), ("bf16", 5), ("bf16", 90)])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("value", [False, True])
def test_picked_blocks(kv, dt, T, bad, value):
    """The last token's key or value is odd: that token's own query shows it, the others, whose own block it lies in, do not."""
    H, KV, D, P, prefix = 4, 2, 64, 32, 300
    T += -(prefix + T) % P or P   # the last token ends a block
    pool, index, keys, values = make_cache(kv, dt, KV, D, P, [prefix + T], seed=4)
    q, cu, qs = make_queries(dt, [T], H, D)
    qs = positive(q, qs, (3,))
    put(pool, index, keys, values, P, prefix + T - 1, 3, bad, value)
    rng = np.random.RandomState(5)
    picks = np.full((T, KV, 4), -1, np.int32)
    for t in range(T):
        own = (prefix + t) // P
        for h in range(KV):
            picks[t, h] = np.sort(np.concatenate([rng.permutation(own)[:3], [own]]))
    ref = block_reference(qs, keys, values, [T], picks, P, 1 / math.sqrt(D))
    if value:
        assert not np.isfinite(ref[0][-1, :, 3]).any() and np.isfinite(ref[1]).all()
    else:
        assert (np.isneginf(bad) and np.isfinite(ref[1][-1]).all()) or np.array_equal(ref[1][-1], np.full(H, bad), equal_nan=True)
    assert np.isfinite(ref[0][:-1]).all()
    check(kv.tbn_block_attention(q, pool, index, cu, T, torch.from_numpy(picks).cuda()), *ref, tolerance(dt, values))
