"""Indices with more places than sequences: idle ones in front, between and behind, more of them than the call has tokens and fewer, tokens that
belong to no sequence."""
import math

import numpy as np
import pytest
import torch

from tests.kv_util import compare, make_cache, make_queries, pack_mask, tolerance
from tests.test_kv_attention_gpu import block_reference, masks, reference

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kv():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2407_12075_amd import kv as binding, tbn
    tbn.lib()
    return binding


def spread(live, n_seqs, rng):
    """Places of the live sequences, ascending."""
    return np.sort(rng.permutation(n_seqs)[:live])


@pytest.mark.parametrize("dt,H,KV,D,P,seqs", [
    ("bf16", 8, 2, 128, 64, [(5000, 1)]), ("f32", 8, 2, 64, 32, [(3000, 1), (31, 1)]),                     # single tokens: two launches
    ("bf16", 4, 1, 64, 32, [(50, 3), (700, 1), (0, 7)]), ("f32", 6, 6, 64, 32, [(97, 13), (5, 7)]),
    ("bf16", 4, 1, 128, 64, [(900, 26), (30, 18)]), ("bf16", 8, 1, 256, 64, [(100, 20)])])                 # the staged kernel
@pytest.mark.parametrize("n_seqs", [4, 12, 64, 65, 500, 8192])
def test_idle_places(kv, dt, H, KV, D, P, seqs, n_seqs):
    rng = np.random.RandomState(n_seqs + D)
    at = spread(len(seqs), n_seqs, rng)
    lens, counts = np.zeros(n_seqs, int), np.zeros(n_seqs, int)
    for s, (p, n) in zip(at, seqs):
        lens[s], counts[s] = p + n, n
    full = np.setdiff1d(np.arange(n_seqs), at)[:1]   # one that has keys and no token
    lens[full] = 40
    pool, index, keys, values = make_cache(kv, dt, KV, D, P, lens.tolist(), seed=3)
    q, cu, qs = make_queries(dt, counts.tolist(), H, D)
    n, most = int(counts.sum()), int(counts.max())
    for kind in ("chain", "tree"):
        see = [m for m in masks(kind, [c for _, c in seqs], 5)]
        words = -(-most // 32)
        mask = None if kind == "chain" else pack_mask(np.concatenate([np.pad(m, ((0, 0), (0, words * 32 - m.shape[1]))) for m in see]), words)
        ref = reference(qs, [keys[s] for s in at], [values[s] for s in at], [c for _, c in seqs], see, 1 / math.sqrt(D))
        compare(*kv.tbn_tree_attention(q, pool, index, cu, most, mask=mask, max_len=int(lens.max())), *ref, tolerance(dt, values))
    # picked blocks: the first and the own one
    picks = np.zeros((n, KV, 2), np.int32)
    picks[:, :, 1] = np.concatenate([(p + np.arange(c)) // P for p, c in seqs])[:, None]
    picks[picks[:, :, 1] == 0, 1] = -1
    ref = block_reference(qs, [keys[s] for s in at], [values[s] for s in at], [c for _, c in seqs], picks, P, 1 / math.sqrt(D))
    compare(*kv.tbn_block_attention(q, pool, index, cu, most, torch.from_numpy(picks).cuda()), *ref, tolerance(dt, values))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_the_same_without_idle_places(kv, dt):
    """One token of one sequence among 300 places: the same split, so the same bits, as alone."""
    H, KV, D, P, length = 8, 2, 128, 64, 9000
    lens = [0] * 300
    lens[217] = length
    pool, index, _, _ = make_cache(kv, dt, KV, D, P, lens, seed=3)
    one = kv.KVIndex(index.table[217:218].clone(), index.lens[217:218].clone(), index.refs, index.status, P)
    q, cu, _ = make_queries(dt, [0] * 217 + [1] + [0] * 82, H, D)
    a = kv.tbn_tree_attention(q, pool, index, cu, 1)
    b = kv.tbn_tree_attention(q, pool, one, torch.tensor([0, 1], dtype=torch.int32, device="cuda"), 1)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("n_seqs", [2, 40])
def test_tokens_of_no_sequence_are_left_alone(kv, n_seqs):
    """cu_q ends before the tokens do: outputs of the others stay as they were."""
    H, KV, D, P = 4, 2, 64, 32
    pool, index, keys, values = make_cache(kv, "f32", KV, D, P, [50] + [0] * (n_seqs - 1), seed=3)
    q, _, qs = make_queries("f32", [9], H, D)
    cu = torch.tensor([0] + [3] * n_seqs, dtype=torch.int32, device="cuda")
    out, lse = torch.full_like(q, 7.0), torch.full((9, H), 7.0, device="cuda")
    kv.tbn_tree_attention(q, pool, index, cu, 3, out=out, lse=lse)
    assert bool((out[3:] == 7).all()) and bool((lse[3:] == 7).all())
    ref = reference(qs[:3], keys[:1], values[:1], [3], masks("chain", [3], 0), 1 / math.sqrt(D))
    compare(out[:3], lse[:3], *ref, tolerance("f32", values[:1]))
