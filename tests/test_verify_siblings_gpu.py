"""Trees of which many tokens hang on one, with the draft's probabilities, against the oracle: as many refusals as are kept, one less and more, several times as
many; accepted behind them; two such tokens on one path and several sequences; rows of one workgroup, of several runs, of slices.  Each refusal costs one pass over the row."""
import numpy as np
import pytest
import torch

from tests.test_verify_gpu import check, dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kv():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2407_12075_amd import kv as binding, tbn
    tbn.lib()
    return binding


def rows(rng, n, V, near=0.5):
    a = rng.standard_normal((n, V)) * 2
    soft = lambda x: (np.exp(x - x.max(1, keepdims=True)) / np.exp(x - x.max(1, keepdims=True)).sum(1, keepdims=True)).astype(np.float32)  # noqa: E731
    return soft(a), soft(a + near * rng.standard_normal((n, V)))


def least(p, q, k):
    """The k tokens that the target gives least beside the draft, and the one that it gives most."""
    ratio = p.astype(np.float64) / q
    order = np.argsort(ratio)
    return order[:k], order[-1]


@pytest.mark.parametrize("V", [40, 4096, 4097, 9001, 16385, 40000])
@pytest.mark.parametrize("n", [33, 63, 64, 65, 66, 67, 127, 128, 130, 200])
def test_refused_siblings(kv, V, n):
    """n of them, then the token that the target favours: refused or accepted; a sequence in front, one behind, one with as many siblings in between."""
    rng, refused = np.random.RandomState(n), set()
    sizes = [3, n + 2, 0, n + 1, 1]
    N = sum(sizes)
    p, q = rows(rng, 1, V)
    p, q = np.repeat(p, N, 0), np.repeat(q, N, 0)
    low, high = least(p[0], q[0], max(V // 4, 1))
    tokens = np.zeros(N, np.int32)
    parents = np.concatenate([[-1, 0, 1], [-1] + [0] * (n + 1), [-1] + [0] * n, [-1]]).astype(np.int32)
    for seed, last in ((0, 0.0), (1, 0.7), (2, 1e30)):
        u = np.random.RandomState(seed).rand(N).astype(np.float32)
        first, second = 3, 3 + n + 2
        for t0, k in ((first, n), (second, n)):
            tokens[t0 + 1:t0 + 1 + k] = rng.choice(low, k)
            u[t0 + 1:t0 + 1 + k] = 1.0
        tokens[first + n + 1], u[first + n + 1] = high, last
        got = check(kv, p, q, tokens, parents, u, sizes)
        if (p[0][low] < q[0][low]).all():   # all n are refused, so that the cases are those that they are meant to be
            assert got[1].tolist()[3] == 1 and got[1].tolist()[1] == (1 if last > 1 else 2)
            refused.add(last)
    assert len(refused) == 3 or V == 40   # few elements: the least are not always below the draft's


@pytest.mark.parametrize("V", [500, 6000, 20000])
def test_two_of_them_on_one_path(kv, V):
    """What the first left is not taken for what the second leaves; tokens out of the vocabulary among the siblings."""
    rng = np.random.RandomState(V)
    n = 70
    p, q = rows(rng, 2, V)
    size = 1 + (n + 1) + n
    at = np.zeros(size, int)
    at[n + 1] = 1   # the accepted one has rows of its own
    p, q = p[at], q[at]
    tokens, u = np.zeros(size, np.int32), rng.rand(size).astype(np.float32)
    low, high = least(p[0], q[0], V // 4)
    tokens[1:n + 1], u[1:n + 1] = rng.choice(low, n), 1.0
    tokens[[5, 40, 66]] = [-1, V, 2 ** 31 - 1]
    tokens[n + 1], u[n + 1] = high, 0.0
    low, _ = least(p[n + 1], q[n + 1], V // 4)
    tokens[n + 2:], u[n + 2:] = rng.choice(low, n), 1.0
    parents = np.array([-1] + [0] * (n + 1) + [n + 1] * n, np.int32)
    got = check(kv, p, q, tokens, parents, u, [size])
    assert got[1].tolist() == [2]


@pytest.mark.parametrize("V", [3000, 17000])
def test_2047_siblings(kv, V):
    """All refused, and what is left after them drawn from; also where nothing is left, and with rows that are no probabilities."""
    rng = np.random.RandomState(1)
    n = 2048
    p, q = rows(rng, 1, V)
    low, _ = least(p[0], q[0], V // 4)
    tokens = np.concatenate([[0], rng.choice(low, n - 1)]).astype(np.int32)
    parents = np.zeros(n, np.int32)
    u = np.full(n, 1.0, np.float32)
    u[0] = 0.37
    check(kv, np.repeat(p, n, 0), np.repeat(q, n, 0), tokens, parents, u, [n])
    check(kv, np.repeat(p, n, 0), np.repeat(p, n, 0), tokens, parents, u, [n])
    odd, strange = p.copy(), q.copy()
    odd[0, ::7], strange[0, ::5], strange[0, 3] = np.nan, -1.0, np.inf
    check(kv, np.repeat(odd, n, 0), np.repeat(strange, n, 0), tokens, parents, u, [n])


def test_a_refusal_costs_one_pass(kv):
    """2047 siblings on 131072 elements, 2.7e8 of them with at most 64 refusals to take off each: 0.23 s.  With all earlier ones taken off in every pass, 1024
    in the mean, it would be some 30 times as long."""
    n, V = 2048, 131072
    p = torch.rand(1, V, device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    q = torch.rand(1, V, device="cuda", generator=torch.Generator("cuda").manual_seed(2)) * 2 / V
    p = p / p.sum()
    token = int((p / q).argmin())
    p, q = p.repeat(n, 1), q.repeat(n, 1)
    tokens = torch.full((n,), token, dtype=torch.int32, device="cuda")
    u = torch.ones(n, device="cuda")
    cu, parents = dev(np.array([0, n], np.int32)), torch.zeros(n, dtype=torch.int32, device="cuda")
    kv.tbn_verify(p[:40], tokens[:40], u[:40], dev(np.array([0, 40], np.int32)), 40, draft=q[:40], parents=parents[:40])
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    start.record()
    picks, counts, follows = kv.tbn_verify(p, tokens, u, cu, n, draft=q, parents=parents)
    end.record()
    end.synchronize()
    ms = start.elapsed_time(end)
    print(f"2047 refusals on 131072 elements: {ms:.1f} ms")
    assert counts.tolist() == [1] and 0 <= int(follows) < V
    assert ms < 2000


@pytest.mark.parametrize("V", [16385, 40000])
@pytest.mark.parametrize("n", [64, 65, 66, 130])
def test_among_many_sequences(kv, V, n):
    """A sequence of n refused siblings among 260 others: a workgroup draws from what they left in runs of the row."""
    rng = np.random.RandomState(n)
    sizes = [1] * 120 + [n + 1] + [1] * 100 + [n + 1] + [1] * 40
    N = sum(sizes)
    p, q = rows(rng, 1, V)
    low, _ = least(p[0], q[0], V // 4)
    p, q = np.repeat(p, N, 0), np.repeat(q, N, 0)
    tokens, parents, u = np.zeros(N, np.int32), np.full(N, -1, np.int32), rng.rand(N).astype(np.float32)
    for first in (120, 120 + n + 1 + 100):
        tokens[first + 1:first + n + 1], parents[first + 1:first + n + 1], u[first + 1:first + n + 1] = rng.choice(low, n), 0, 1.0
    assert kv.lib().tbn_verify_workspace_bytes(N, n + 1, len(sizes), V) == (8 * V * (N // 66) if n >= 65 else 0)
    got = check(kv, p, q, tokens, parents, u, sizes)
    assert max(got[1].tolist()) == 1
