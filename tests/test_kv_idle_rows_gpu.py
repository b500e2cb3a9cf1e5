"""Indices with many more places than sequences whose drafts have many rows, so that the kernels for many rows are launched with a row of workgroups per token:
attention with a window and over the cache in 4 bits, 49 to 64 rows of a sequence, more than 64, fewer; trees and chunks, keys split and whole."""
import math

import numpy as np
import pytest
import torch

from tests.kv4_util import make_cache4
from tests.kv_util import compare, make_cache, make_queries, tolerance
from tests.test_kv_attention_gpu import masks
from tests.test_kv_window_gpu import packed, reference

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kv():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2407_12075_amd import kv as binding, tbn
    tbn.lib()
    return binding


CASES = [
    # type, heads, kv heads, dim, page, [(keys before, tokens)], first keys, window
    ("bf16", 8, 1, 64, 32, [(300, 16)], 3, 70),                     # 128 rows
    ("bf16", 8, 1, 128, 64, [(700, 9), (40, 8)], 4, 200),           # 72 and 64
    ("bf16", 16, 2, 128, 64, [(6000, 13)], 4, 3000),                # 104, keys split
    ("bf16", 8, 1, 96, 64, [(5000, 7), (3000, 7)], 70, 2500),       # 56, keys split, channels that fill no tile
    ("bf16", 8, 1, 256, 128, [(900, 10), (0, 7)], 0, 500),
    ("bf16", 7, 1, 64, 64, [(500, 7)], 1, 64),                      # 49
    ("bf16", 24, 1, 128, 64, [(2500, 16)], 4, 1024),                # 384: three tiles
    ("bf16", 8, 1, 160, 32, [(4000, 12)], 5, 2100),
    ("f32", 8, 1, 64, 32, [(3000, 9), (100, 8)], 4, 2000),
    ("f32", 4, 1, 128, 64, [(700, 16)], 4, 300)]


@pytest.mark.parametrize("n_seqs", [300, 8192])
@pytest.mark.parametrize("kind", ["none", "tree"])
@pytest.mark.parametrize("dt,H,KV,D,P,seqs,sink,window", CASES)
def test_idle_places(kv, dt, H, KV, D, P, seqs, sink, window, kind, n_seqs):
    rng = np.random.RandomState(n_seqs + D)
    at = np.sort(rng.permutation(n_seqs)[:len(seqs)])
    lens, counts = np.zeros(n_seqs, int), np.zeros(n_seqs, int)
    for s, (p, n) in zip(at, seqs):
        lens[s], counts[s] = p + n, n
    lens[np.setdiff1d(np.arange(n_seqs), at)[:1]] = 40   # one that has keys and no token
    total, most = int(counts.sum()), int(counts.max())
    assert 16 * total <= n_seqs                          # a row of workgroups for each token
    q, cu, qs = make_queries(dt, counts.tolist(), H, D, stride=H * D + 8)
    few = [n for _, n in seqs]
    see = masks("tree", few, 5) if kind == "tree" else None
    mask = packed(see, few) if see else None
    scale = 1 / math.sqrt(D)
    pool, index, keys, values = make_cache(kv, dt, KV, D, P, lens.tolist(), seed=3)
    mine = lambda x: [x[s] for s in at]  # noqa: E731
    out, lse = kv.tbn_window_attention(q, pool, index, cu, most, sink, window, mask=mask, max_len=int(lens.max()))
    compare(out, lse, *reference(qs, mine(keys), mine(values), few, sink, window, see, scale), tolerance(dt, values))
    again = kv.tbn_window_attention(q, pool, index, cu, most, sink, window, mask=mask, max_len=int(lens.max()))
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])
    if D % 32:
        return
    four, index4, keys, values = make_cache4(kv, KV, D, P, lens.tolist(), seed=4)
    for w in (0, window):
        out, lse = kv.tbn_kv4_attention(q, four, index4, cu, most, mask=mask, n_sink=sink, window=w)
        ref = reference(qs, mine(keys), mine(values), few, sink if w else 0, w or 1 << 30, see, scale)
        compare(out, lse, *ref, tolerance(dt, values))
        again = kv.tbn_kv4_attention(q, four, index4, cu, most, mask=mask, n_sink=sink, window=w)
        assert torch.equal(out, again[0]) and torch.equal(lse, again[1])
