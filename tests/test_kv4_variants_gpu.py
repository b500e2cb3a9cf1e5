"""Every width of the kernels over the cache in 4 bits, in the forms that the number of rows chooses, and prompts with a window in the tiles that the
number of workgroups chooses, against the float64 oracle."""
import math

import numpy as np
import pytest
import torch

from tests.kv4_util import make_cache4
from tests.kv_util import compare, make_cache, make_queries, tolerance
from tests.test_kv_attention_gpu import masks
from tests.test_kv_window_gpu import packed, reference

pytestmark = pytest.mark.gpu
WIDTHS = [32, 64, 96, 128, 160, 192, 224, 256]


@pytest.fixture(scope="module")
def kv():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2407_12075_amd import kv as binding, tbn
    tbn.lib()
    return binding


def check(kv, dt, H, KV, D, P, seqs, sink, window, kind, seed=3, no_number=0.0):
    counts = [n for _, n in seqs]
    pool, index, keys, values = make_cache4(kv, KV, D, P, [p + n for p, n in seqs], seed=D + seed, no_number=no_number)
    q, cu, qs = make_queries(dt, counts, H, D, seed=seed)
    see = None if kind == "none" else masks(kind, counts, seed)
    mask = None if see is None else packed(see, counts)
    out, lse = kv.tbn_kv4_attention(q, pool, index, cu, max(counts), mask=mask, n_sink=sink, window=window)
    compare(out, lse, *reference(qs, keys, values, counts, sink, window or 1 << 30, see, 1 / math.sqrt(D)), tolerance(dt, values))


@pytest.mark.parametrize("window", [0, 90])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("D", WIDTHS)
def test_one_or_two_rows(kv, D, dt, window):
    """So few that the groups of channels share the columns of a product."""
    check(kv, dt, 2, 1, D, 32, [(0, 1), (31, 1), (200, 1), (333, 1)], 3, window, "none")
    check(kv, dt, 3, 3, D, 64, [(70, 2), (500, 1), (0, 0), (64, 2)], 3, window, "any")


@pytest.mark.parametrize("window", [0, 90])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("D", WIDTHS)
def test_up_to_48_rows(kv, D, dt, window):
    check(kv, dt, 6, 2, D, 64, [(70, 3), (300, 16), (0, 1)], 5, window, "tree")
    check(kv, dt, 20, 1, D, 128, [(150, 1), (127, 2)], 5, window, "none")


@pytest.mark.parametrize("window", [0, 170])
@pytest.mark.parametrize("T", [14, 40])
@pytest.mark.parametrize("D", WIDTHS)
def test_staged(kv, D, T, window):
    """56 rows in tiles of 64, 160 in tiles of 128; pages of half a step, ends inside of one."""
    check(kv, "bf16", 8, 2, D, 32, [(301, T), (0, T - 3), (63, 1), (0, 0)], 40, window, "any")
    check(kv, "bf16", 4, 1, D, 128, [(450, T), (64 - T, T)], 1, window, "none")


@pytest.mark.parametrize("D,T", [(64, 14), (128, 40), (160, 40), (256, 14)])
def test_staged_keys_that_are_no_numbers(kv, D, T):
    check(kv, "bf16", 8, 2, D, 64, [(5, T), (0, T - 3)], 0, 0, "any", no_number=0.03)


@pytest.mark.parametrize("window,sink", [(130, 4), (40, 70)])
@pytest.mark.parametrize("seqs", [[(300, 600)], [(0, 290), (500, 300)], [(90, 1250)]])
def test_prompts_with_a_window(kv, seqs, window, sink):
    """8 kv heads: tiles of 128 rows would leave half of the GPU without one (600 and 2 x 300 tokens), or not (1250)."""
    counts = [n for _, n in seqs]
    H, KV, D, P = 16, 8, 64, 64
    scale = 1 / math.sqrt(D)
    pool, index, keys, values = make_cache(kv, "bf16", KV, D, P, [p + n for p, n in seqs], seed=2)
    q, cu, qs = make_queries("bf16", counts, H, D)
    take = np.random.RandomState(0).permutation(sum(counts))[:120]   # some of the tokens
    out, lse = kv.tbn_window_attention(q, pool, index, cu, max(counts), sink, window)
    compare(out[take], lse[take], *some(qs, keys, values, counts, sink, window, scale, take), tolerance("bf16", values))
    pool, index, keys, values = make_cache4(kv, KV, D, P, [p + n for p, n in seqs], seed=2)
    out, lse = kv.tbn_kv4_attention(q, pool, index, cu, max(counts), n_sink=sink, window=window)
    compare(out[take], lse[take], *some(qs, keys, values, counts, sink, window, scale, take), tolerance("bf16", values))


def some(qs, keys, values, counts, sink, window, scale, take):
    """The oracle's rows of some tokens: each as the last one of a sequence that ends with it."""
    first = np.concatenate([[0], np.cumsum(counts)])
    out, lse = np.zeros((len(take),) + qs.shape[1:]), np.zeros((len(take), qs.shape[1]))
    for i, t in enumerate(take):
        s = int(np.searchsorted(first, t, side="right")) - 1
        n = len(keys[s]) - counts[s] + (t - first[s]) + 1
        o, l = reference(qs[t:t + 1], [keys[s][:n]], [values[s][:n]], [1], sink, window, None, scale)
        out[i], lse[i] = o[0], l[0]
    return out, lse


@pytest.mark.parametrize("rows", [1, 12])
def test_largest_float32_queries(kv, rows):
    """Queries whose nearest bfloat16 number is infinite, on keys so small that the logits are of ordinary size."""
    H, KV, D, lens = 2, 1, 128, [200, 65]
    pool, index, keys, values = make_cache4(kv, KV, D, 32, lens, seed=4)
    pool.k_exp -= 98
    keys = [k * 2.0 ** -98 for k in keys]
    rng = np.random.RandomState(5)
    q = torch.from_numpy((rng.uniform(3.3962e38, 3.4028e38, (2 * rows, H, D)) * rng.choice([-1, 1], (2 * rows, H, D))).astype(np.float32))
    q[0] = torch.finfo(torch.float32).max
    assert q.isfinite().all() and q.to(torch.bfloat16).isinf().all()
    cu = torch.tensor([0, rows, 2 * rows], dtype=torch.int32, device="cuda")
    scale = 2.0 ** -30 / math.sqrt(D)
    out, lse = kv.tbn_kv4_attention(q.cuda(), pool, index, cu, rows, scale=scale)
    compare(out, lse, *reference(q.double().numpy(), keys, values, [rows] * 2, 0, 1 << 30, None, scale), tolerance("f32", values))
