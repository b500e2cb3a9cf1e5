"""The staged kernel of many rows (bfloat16) in each of its widths against the float64 oracle: 64 and 128 rows of a workgroup, heads that fill the
width and heads that do not, pages of 32 to 128 keys, lengths that end inside a step, chains, trees and rows that see nothing."""
import math

import numpy as np
import pytest
import torch

from tests.kv_util import compare, make_cache, make_queries, pack_mask, tolerance
from tests.test_kv_attention_gpu import masks, reference

# heads, kv heads, dim, page, [(keys before, tokens)]
CASES = [
    (4, 2, 96, 32, [(131, 9), (0, 5), (64, 1)]),       # 18 rows
    (2, 1, 96, 64, [(77, 35), (200, 3)]),              # 70
    (2, 1, 96, 128, [(100, 65), (0, 1), (0, 0)]),      # 130, two tiles
]


@pytest.fixture(scope="module")
def kv():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2407_12075_amd import kv as binding, tbn
    tbn.lib()
    return binding


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["none", "tree", "any"])
@pytest.mark.parametrize("H,KV,D,P,seqs", CASES)
def test_many_rows(kv, H, KV, D, P, seqs, kind):
    counts = [n for _, n in seqs]
    # no page to spare, the last key in the last row of the last page: nothing lies behind what may be read but the end of the pool
    lens = [p + n for p, n in seqs]
    lens[0] += -lens[0] % P
    pool, index, keys, values = make_cache(kv, "bf16", KV, D, P, lens, seed=H * D, extra_pages=0)
    q, cu, qs = make_queries("bf16", counts, H, D)
    see = masks("chain" if kind == "none" else kind, counts, 3)
    words = -(-max(counts) // 32)
    mask = None if kind == "none" else pack_mask(np.concatenate([np.pad(m, ((0, 0), (0, words * 32 - m.shape[1]))) for m in see]), words)
    out, lse = kv.tbn_tree_attention(q, pool, index, cu, max(counts), mask=mask)
    compare(out, lse, *reference(qs, keys, values, counts, see, 1 / math.sqrt(D)), tolerance("bf16", values))
