"""Verification of drafted tokens against the oracle: chains and trees, with the draft's probabilities and for picked tokens, vocabularies that
one workgroup sums and that many do, borders, rows that are no probabilities, idle sequences, the distribution of what is emitted."""
import math

import numpy as np
import pytest
import torch

from oracle.verify_oracle import verify as oracle

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kv():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2407_12075_amd import kv as binding, tbn
    tbn.lib()
    return binding


def tree(rng, n, kids):
    return [-1] + [int(rng.randint(max(0, i - 4), i)) if kids > 1 else i - 1 for i in range(1, n)]


def case(counts, V, kids, seed, near=0.5):
    """Probabilities, tokens drawn from the draft (some from anywhere), parents, uniform numbers."""
    rng = np.random.RandomState(seed)
    N = sum(counts)
    a = rng.standard_normal((N, V)) * 2
    soft = lambda x: (np.exp(x - x.max(1, keepdims=True)) / np.exp(x - x.max(1, keepdims=True)).sum(1, keepdims=True)).astype(np.float32)  # noqa: E731
    p, q = soft(a), soft(a + near * rng.standard_normal((N, V)))
    parents, tokens, at = [], np.zeros(N, np.int32), 0
    for n in counts:
        up = tree(rng, n, kids) if n else []
        parents += up
        for i in range(1, n):
            w = q[at + up[i]].astype(np.float64)
            tokens[at + i] = rng.choice(V, p=w / w.sum()) if rng.rand() < 0.9 else rng.randint(V)
        at += n
    return p, q, tokens, np.array(parents, np.int32), rng.rand(N).astype(np.float32)


def expected(p, q, tokens, parents, u, counts, width):
    picks, many, follows = np.full((len(counts), width), -1), [], []
    at = 0
    for s, n in enumerate(counts):
        if n == 0:
            many.append(0)
            follows.append(-1)
            continue
        here = slice(at, at + n)
        path, token = oracle(p[here], None if q is None else q[here], tokens[here], None if parents is None else parents[here], u[here])
        picks[s, :len(path)] = path
        many.append(len(path))
        follows.append(token)
        at += n
    return picks, many, follows


def dev(x):
    return None if x is None else torch.from_numpy(np.ascontiguousarray(x)).cuda()


def check(kv, p, q, tokens, parents, u, counts, width=None, **kw):
    width = max(counts) if width is None else width
    cu = dev(np.concatenate([[0], np.cumsum(counts)]).astype(np.int32))
    got = kv.tbn_verify(p if torch.is_tensor(p) else dev(p), dev(tokens), dev(u), cu, width, draft=q if torch.is_tensor(q) else dev(q), parents=dev(parents), **kw)
    host = lambda t: t.cpu().numpy() if torch.is_tensor(t) else t  # noqa: E731
    picks, many, follows = expected(host(p), host(q), tokens, parents, u, counts, width)
    assert got[1].tolist() == many
    assert got[2].tolist() == follows
    assert np.array_equal(got[0].cpu().numpy(), picks)
    return got


@pytest.mark.parametrize("draft", [True, False])
@pytest.mark.parametrize("kids", [1, 3])
@pytest.mark.parametrize("V", [1, 2, 7, 64, 513, 1021, 5000, 16384, 16385, 33333])
def test_random(kv, V, kids, draft):
    counts = [6, 1, 0, 17, 2, 70, 3, 0, 9]
    p, q, tokens, parents, u = case(counts, V, kids, V)
    check(kv, p, q if draft else None, tokens, parents, u, counts)
    if kids == 1:
        check(kv, p, q if draft else None, tokens, None, u, counts, width=80)


@pytest.mark.parametrize("draft", [True, False])
def test_rows_apart(kv, draft):
    """Rows of a wider tensor at odd addresses."""
    counts, V = [5, 9, 1], 17001
    p, q, tokens, parents, u = case(counts, V, 3, 5)
    wide = torch.full((sum(counts), 2 * V + 5), -3.0, device="cuda")
    wide[:, 1:1 + V], wide[:, V + 3:2 * V + 3] = dev(p), dev(q)
    check(kv, wide[:, 1:1 + V], wide[:, V + 3:2 * V + 3] if draft else None, tokens, parents, u, counts)


@pytest.mark.parametrize("V", [8, 40000])
def test_borders(kv, V):
    """Numbers that lie on a border exactly: a draft is accepted below it, a draw goes behind it."""
    p, q = np.zeros((3, V), np.float32), np.zeros((3, V), np.float32)
    p[:, [1, V // 2, V - 1]] = [0.25, 0.5, 0.25]
    q[:, [1, V // 2]] = [0.5, 0.5]
    tokens = np.array([0, 1, 1], np.int32)
    for uc in (0.0, np.nextafter(np.float32(0.5), np.float32(0)), 0.5, 0.75):
        for ur in (0.0, 0.25, np.nextafter(np.float32(0.25), np.float32(0)), 0.75, 1 - 2.0 ** -24, 1.0, -0.5):
            check(kv, p, q, tokens, None, np.array([ur, uc, uc], np.float32), [3])
            check(kv, p, None, tokens, np.array([-1, 0, 0], np.int32), np.array([ur, uc, uc], np.float32), [3])
    # a number that is none: nothing is accepted, the last token that has a share
    got = kv.tbn_verify(dev(p), dev(tokens), dev(np.full(3, np.nan, np.float32)), dev(np.array([0, 3], np.int32)), 3)
    assert got[0].tolist() == [[0, -1, -1]] and got[2].tolist() == [V - 1]


@pytest.mark.parametrize("V", [9, 30000])
@pytest.mark.parametrize("draft", [True, False])
def test_rows_that_are_no_probabilities(kv, V, draft):
    counts = [4, 3, 3, 2, 2]
    p, q, tokens, parents, u = case(counts, V, 3, 3)
    p[0, 1:] = 0
    p[0, 0] = 1
    p[4] = 0                      # nothing to draw
    p[7, ::2], p[7, 3] = -1, np.nan
    q[7, ::3] = np.nan
    p[10] *= 1e-38                # sums far from one
    p[12, V - 1] = np.inf         # no finite sum
    tokens[1], tokens[5], tokens[8] = -1, V, 2 ** 31 - 1
    check(kv, p, q if draft else None, tokens, parents, u, counts)
    # target and draft alike, refused all the same: drawn from the target
    p, _, tokens, parents, u = case([3], V, 3, 4)
    u[1:] = 2.0
    check(kv, p, p if draft else None, tokens, np.array([-1, 0, 0], np.int32), u, [3])


def test_parents_that_are_none(kv):
    counts = [7]
    p, q, tokens, _, u = case(counts, 50, 3, 8)
    u[1:] = 0
    for parents in ([-1, -1, -1, -1, -1, -1, -1], [-1, 0, 5, 2, 3, 1, 6], [0, 0, 1, 1, 2, 2, 3], [3, 2 ** 31 - 1, -2 ** 31, 0, 3, 3, 5]):
        check(kv, p, q, tokens, np.array(parents, np.int32), u, counts)
        check(kv, p, None, tokens, np.array(parents, np.int32), u, counts)


@pytest.mark.parametrize("draft", [True, False])
def test_long_chains_and_many_siblings(kv, draft):
    n, V = 2048, 40
    p, q, tokens, _, u = case([n], V, 1, 9, near=0.05)
    check(kv, p, q if draft else None, tokens, None, u * 0.3, [n])
    parents = np.zeros(n, np.int32)
    check(kv, p, q if draft else None, tokens, parents, np.full(n, 0.9999, np.float32), [n])


def test_a_vocabulary_in_slices_for_one_sequence_and_for_many(kv):
    V = 131072
    p, q, tokens, parents, u = case([3, 2], V, 3, 10)
    need = kv.lib().tbn_verify_workspace_bytes(5, 3, 2, V)
    assert need > 0 and kv.lib().tbn_verify_workspace_bytes(5, 3, 2, 1024) == 0
    a = check(kv, p, q, tokens, parents, u, [3, 2])
    for seed in range(20):
        u = np.random.RandomState(seed).rand(5).astype(np.float32)
        check(kv, p, q, tokens, parents, u, [3, 2])
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    b = check(kv, p, q, tokens, parents, u, [3, 2], workspace=ws, stream=side)
    with pytest.raises(RuntimeError):
        check(kv, p, q, tokens, parents, u, [3, 2], workspace=ws[:need - 8])
    assert a is not b


@pytest.mark.parametrize("kids,draft", [(1, True), (2, True), (2, False)])
def test_what_is_emitted_has_the_targets_distribution(kv, kids, draft):
    """8192 sequences: the token behind the first one, be it an accepted draft or the one that follows, against the target's row."""
    rng = np.random.RandomState(0)
    B, V, T = 8192, 12, 1 + kids
    p = rng.dirichlet(np.ones(V)).astype(np.float32)
    q = rng.dirichlet(np.ones(V)).astype(np.float32)
    tokens = np.zeros((B, T), np.int32)
    if draft:
        tokens[:, 1:] = rng.choice(V, (B, kids), p=q.astype(np.float64) / q.astype(np.float64).sum())
    else:
        tokens[:, 1:] = np.argsort(-q)[:kids]
    parents = np.tile(np.array([-1] + [0] * kids, np.int32), B)
    u = torch.rand(B * T, generator=torch.Generator().manual_seed(1))
    picks, counts, follows = kv.tbn_verify(dev(np.tile(p, (B * T, 1))), dev(tokens.reshape(-1)), u.cuda(), dev(np.arange(0, B * T + 1, T).astype(np.int32)), T,
                                           draft=dev(np.tile(q, (B * T, 1))) if draft else None, parents=dev(parents))
    first = np.where(counts.cpu().numpy() > 1, np.take_along_axis(tokens, np.maximum(picks.cpu().numpy()[:, 1:2], 0), 1)[:, 0], follows.cpu().numpy())
    seen = np.bincount(first, minlength=V) / B
    assert np.all(np.abs(seen - p) <= 5 * np.sqrt(p * (1 - p) / B))   # five standard deviations: one in 10^6 for each of a dozen


@pytest.mark.parametrize("V", [500, 50000])
def test_graph(kv, V):
    counts = [4, 6]
    p, q, tokens, parents, u = (dev(x) for x in case(counts, V, 3, 12))
    cu = dev(np.array([0, 4, 10], np.int32))
    kv.tbn_verify(p, tokens, u, cu, 6, draft=q, parents=parents)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = kv.tbn_verify(p, tokens, u, cu, 6, draft=q, parents=parents)
    for seed in range(4):
        u.copy_(torch.rand(10, generator=torch.Generator().manual_seed(seed)))
        g.replay()
        torch.cuda.synchronize()
        want = kv.tbn_verify(p, tokens, u, cu, 6, draft=q, parents=parents)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        picks, many, follows = expected(*(x.cpu().numpy() for x in (p, q, tokens, parents, u)), counts, 6)
        assert got[1].tolist() == many and got[2].tolist() == follows and np.array_equal(got[0].cpu().numpy(), picks)


def test_refusals(kv):
    from paper_2407_12075_amd import tbn
    p, q, tokens, parents, u = (dev(x) for x in case([4], 30, 1, 1))
    cu = dev(np.array([0, 4], np.int32))
    for kw in (dict(draft=q[:3]), dict(draft=q.double()), dict(parents=parents[:2]), dict(parents=parents.long())):
        with pytest.raises(ValueError):
            kv.tbn_verify(p, tokens, u, cu, 4, **kw)
    for args in ((p.bfloat16(), tokens, u), (p.t().contiguous().t(), tokens, u), (p, tokens.long(), u), (p, tokens, u[:3]), (p, tokens, u.cpu()), (p[:, ::2], tokens, u)):
        with pytest.raises(ValueError):
            kv.tbn_verify(*args, cu, 4)
    with pytest.raises(tbn.TbnError) as e:
        kv.tbn_verify(p, tokens, u, cu, 2049)
    assert e.value.status == 3
    # fewer places than tokens: those behind are not there
    got = kv.tbn_verify(p, tokens, torch.zeros_like(u), cu, 2)
    assert got[1].tolist() == [2]
