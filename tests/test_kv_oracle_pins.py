"""Pins of the cache's oracle on the CPU: hand-worked bookkeeping, attention against torch's softmax, summaries and picks by hand."""
import math

import numpy as np
import torch

from oracle import kv_oracle as orc


def test_reserve_by_hand():
    c = orc.Cache(3, 4, 6, 32)
    assert c.reserve([33, 0, 1]) == [(-1, -1)] * 3
    assert c.rows == [[0, 1], [], [2]] and c.refs == [1, 1, 1, 0, 0, 0]
    c.fork([0], [1])
    assert c.refs == [2, 2, 1, 0, 0, 0]
    assert c.reserve([1, 1, 0]) == [(1, 3), (-1, -1), (-1, -1)]      # the first owner moves out, the second one keeps the page
    assert c.rows == [[0, 3], [0, 1], [2]] and c.refs == [2, 1, 1, 1, 0, 0]
    c.release([0, 40, 0])
    assert c.refs == [1, 1, 0, 0, 0, 0]
    assert c.reserve([0, 0, 200]) == [(-1, -1)] * 3 and c.status == 2
    c.status = 0
    assert c.reserve([128, 60, 0]) == [(-1, -1)] * 3 and c.status == 1 and c.lens == [0, 34, 0]


def test_compact_by_hand():
    c = orc.Cache(2, 4, 8, 32)
    c.rows, c.lens, c.refs = [[6, 1], [7, 1]], [64, 50], [0, 2, 0, 0, 0, 0, 1, 1]
    assert c.compact() == ([6, 7], [0, 2])
    assert c.rows == [[0, 1], [2, 1]] and c.refs == [1, 2, 1, 0, 0, 0, 0, 0]


def test_attention_against_torch():
    rng = np.random.RandomState(0)
    q, k, v = rng.standard_normal(16), rng.standard_normal((40, 16)), rng.standard_normal((40, 16))
    see = rng.rand(40) < 0.5
    out, lse = orc.attention(q, k, v, see, 0.25)
    a = torch.from_numpy(k @ q * 0.25).masked_fill(torch.from_numpy(~see), -math.inf)
    assert np.allclose(out, (torch.softmax(a, 0) @ torch.from_numpy(v)).numpy(), atol=1e-14) and abs(lse - float(torch.logsumexp(a, 0))) < 1e-13
    out, lse = orc.attention(q, k, v, np.zeros(40, bool), 0.25)
    assert (out == 0).all() and lse == -math.inf


def test_summary_bounds_the_keys():
    rng = np.random.RandomState(1)
    for scale in (1e-30, 1.0, 3e4):
        k = rng.standard_normal((32, 8)) * scale
        codes, step = orc.summary(k)
        assert np.abs(codes).max() <= 64 and (codes[0] * step >= k.max(0)).all() and (codes[1] * step <= k.min(0)).all()
        assert ((codes[0] - 1) * step < k.max(0)).all() and math.log2(step) == round(math.log2(step))
    assert orc.summary(np.array([[1.0, 2.0]]))[0].tolist() == [[16, 32], [16, 32]]     # 2 = 0.5 * 2^2: step 1/16
    assert orc.summary(np.zeros((3, 2)))[1] == 2.0 ** -106
    assert orc.summary(np.array([[math.inf, 1.0]]))[1] == math.inf


def test_scores_bound_the_summed_logits():
    """Up to the rounding of q (half a unit per channel) the score of a block is at least the group's summed logits of any of its keys."""
    rng = np.random.RandomState(2)
    for _ in range(20):
        q, k = rng.standard_normal((4, 16)), rng.standard_normal((32, 16))
        codes, step = orc.summary(k)
        x = 2.0 ** (6 - orc.exponent(np.abs(q).max()))
        c = np.rint(q * x)
        score = np.maximum(c * codes[0], c * codes[1]).sum() * step / x
        assert score >= max((k @ q.T).sum(1)) - 0.5 * 4 * 16 * np.abs(k).max() / x


def test_picks_by_hand():
    codes = np.zeros((6, 2, 2), np.int64)
    codes[:, 0], codes[:, 1] = [[9, 9], [1, 0], [5, 0], [5, 0], [7, 0], [0, 0]], 0
    q = np.array([[1.0, 0.0]])
    assert orc.picks(q, codes, [1.0] * 6, 5, 4, 1, 1) == [0, 2, 4, 5]
    assert orc.picks(q, codes, [1.0] * 6, 5, 3, 1, 2) == [0, 4, 5]
    assert orc.picks(q, codes, [1.0] * 6, 3, 4, 1, 1) == [0, 1, 2, 3]
    assert orc.picks(q, codes, [1.0, 10.0, 1.0, 1.0, 1.0, 1.0], 5, 3, 1, 1) == [0, 1, 5]
