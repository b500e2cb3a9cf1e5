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
    (4, 2, 40, 32, [(95, 9), (0, 3)]), (2, 1, 40, 64, [(63, 70), (5, 2)]), (3, 1, 64, 128, [(130, 7), (1, 6)]), (2, 1, 64, 32, [(33, 40)]),
    (2, 1, 80, 64, [(100, 12), (300, 1)]), (4, 4, 80, 32, [(31, 90), (0, 65)]),
    (2, 1, 104, 64, [(10, 20), (129, 2)]), (2, 1, 104, 128, [(128, 36), (1, 33)]), (4, 1, 128, 32, [(97, 8)]), (2, 1, 128, 64, [(0, 80), (66, 64)]),
    (2, 1, 136, 32, [(75, 13), (0, 2)]), (2, 1, 136, 64, [(40, 37), (31, 1)]), (4, 1, 256, 64, [(191, 6), (0, 1)]),
    (2, 1, 256, 32, [(45, 36), (100, 2)]), (2, 2, 256, 128, [(130, 66)]), (2, 1, 200, 128, [(64, 70), (0, 34)]),
]


def test_every_instance_has_a_case():
    """Widths of 64, 96, 128 and 256 channels, 64 or 128 rows, heads that fill the width or do not: as launch_kv_rows takes them."""
    widths = (64, 96, 128, 256)
    seen = set()
    for H, KV, D, _, seqs in CASES:
        rows = max(n for _, n in seqs) * H // KV
        assert rows > 16
        width = next(w for w in widths if D <= w)
        seen.add((width, 64 if rows <= 64 else 128, D == width))
    assert seen == {(w, r, even) for w in widths for r in (64, 128) for even in (True, False)}


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


@pytest.mark.gpu
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("D,P,H,KV,T", [(96, 64, 2, 1, 20), (96, 32, 2, 1, 40), (128, 64, 4, 2, 40), (136, 64, 2, 1, 12), (256, 32, 2, 1, 20), (256, 64, 2, 1, 40),
                                        (80, 128, 2, 1, 40)])
def test_values_that_are_not_finite(kv, D, P, H, KV, T, bad):
    """Drafted tokens' values hold `bad` in some channels: queries that see them show it there, the others are as without it."""
    prefix = 45
    pool, index, keys, values = make_cache(kv, "bf16", KV, D, P, [prefix + T], seed=2)
    table = index.table.cpu().numpy()[0]
    for j, d in ((3, 5), (10, 0), (T - 1, D - 1), (7, D // 2)):
        at = prefix + j
        values[0][at, :, d] = bad
        pool.v[int(table[at // P]), :, d, at % P] = bad
    q, cu, qs = make_queries("bf16", [T], H, D)
    for kind in ("tree", "any", "chain"):
        see = masks(kind, [T], 4)
        mask = None if kind == "chain" else pack_mask(np.pad(see[0], ((0, 0), (0, 64 - T))), 2)
        ref, ref_lse = reference(qs, keys, values, [T], see, 1 / math.sqrt(D))
        assert not np.isfinite(ref).all() and np.isfinite(ref).any()
        compare(*kv.tbn_tree_attention(q, pool, index, cu, T, mask=mask), ref, ref_lse, tolerance("bf16", values))
