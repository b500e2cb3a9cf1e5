"""Verification of batches that give every CU a sequence (256 and more) with rows beyond what a workgroup's registers hold: a workgroup per sequence sums its row in runs, narrows
them down, once or more often, and scans the last; against the oracle.  And calls on another stream than the current one."""
import numpy as np
import pytest
import torch

from oracle.verify_oracle import verify as oracle
from tests.test_verify_gpu import case, dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kv():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2407_12075_amd import kv as binding, tbn
    tbn.lib()
    return binding


def base_rows(rng, V):
    """Targets and drafts: ordinary ones, alike (nothing is left), all in the last elements, sums far from one, nothing but one element, nothing at all."""
    a = rng.standard_normal((6, V)) * 2
    soft = lambda x: (np.exp(x - x.max(1, keepdims=True)) / np.exp(x - x.max(1, keepdims=True)).sum(1, keepdims=True)).astype(np.float32)  # noqa: E731
    p, q = soft(a), soft(a + 0.5 * rng.standard_normal((6, V)))
    q[1] = p[1]
    p[2, :-7] = 0
    p[3] *= 1e-30
    p[4] = 0
    p[4, V // 2 + 1] = 0.25
    p[5] = 0
    return p, q


def patterns(rng, V, p, q, chain):
    """Sequences that the batch repeats: rows, tokens, parents, numbers."""
    found = [([], [], [], [])]
    edge = [0.0, 1 - 2.0 ** -24, 2.0 ** -24, 0.5, 1.0]
    for n, x in ((1, 0), (1, 2), (1, 3), (1, 4), (1, 5)):
        found += [([x], [0], [-1], [u]) for u in edge[:3 if x else 5]]
    for i in range(10):
        n = 2 + i % 3
        parents = [-1] + [j - 1 if chain else 0 if j < 3 else 1 for j in range(1, n)]
        rows = [int(rng.choice([0, 0, 1, 2, 3])) for _ in range(n)]
        tokens = [0] + [int(rng.choice(V, p=q[rows[parents[j]]].astype(np.float64) / q[rows[parents[j]]].astype(np.float64).sum())) for j in range(1, n)]
        found.append((rows, tokens, parents, [float(rng.rand())] + [float(rng.rand()) if i % 2 else 2.0 for _ in range(1, n)]))   # every other one: all refused
    return found


@pytest.mark.parametrize("draft", [True, False])
@pytest.mark.parametrize("V,n_seqs", [(16385, 256), (33333, 300), (300001, 257)])
@pytest.mark.parametrize("chain", [False, True])
def test_rows_in_runs(kv, V, n_seqs, draft, chain):
    rng = np.random.RandomState(V % 1000)
    p, q = base_rows(rng, V)
    kinds = patterns(rng, V, p, q, chain)
    results = []
    for rows, tokens, parents, u in kinds:
        u32 = np.array(u, np.float32)
        results.append(oracle(p[rows], q[rows] if draft else None, tokens, parents, u32) if rows else ([], -1))
    order = list(range(len(kinds))) + list(rng.randint(0, len(kinds), n_seqs - len(kinds)))
    idle = sum(1 for k in order if not kinds[k][0])
    order += [5] * idle                             # tokens enough for every sequence of the index to have one
    rows, tokens, parents, u = (np.concatenate([np.asarray(kinds[k][f], t) for k in order]) for f, t in enumerate((np.int64, np.int32, np.int32, np.float32)))
    cu = np.concatenate([[0], np.cumsum([len(kinds[k][0]) for k in order])]).astype(np.int32)
    need = kv.lib().tbn_verify_workspace_bytes(len(rows), 4, len(order), V)
    assert need == 0, "the rows go in slices"
    at = dev(rows)
    got = kv.tbn_verify(dev(p)[at], dev(tokens), dev(u), dev(cu), 4, draft=dev(q)[at] if draft else None, parents=None if chain else dev(parents))
    picks, counts, follows = (t.cpu().numpy() for t in got)
    for s, k in enumerate(order):
        path, token = results[k]
        assert counts[s] == len(path) and follows[s] == token, (s, k, counts[s], follows[s], results[k])
        assert picks[s].tolist() == path + [-1] * (4 - len(path))


@pytest.mark.parametrize("V", [1000, 40000, 131072])
def test_on_another_stream(kv, V):
    """The same inputs on the current stream and on another one, with a workspace of the caller's and without: the same results, once the other stream is done."""
    p, q, tokens, parents, u = (dev(x) for x in case([3, 2], V, 3, 10))
    cu = dev(np.array([0, 3, 5], np.int32))
    here = kv.tbn_verify(p, tokens, u, cu, 3, draft=q, parents=parents)
    need = kv.lib().tbn_verify_workspace_bytes(5, 3, 2, V)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    there = kv.tbn_verify(p, tokens, u, cu, 3, draft=q, parents=parents, stream=side)
    with torch.cuda.stream(side):
        current = kv.tbn_verify(p, tokens, u, cu, 3, draft=q, parents=parents)
    ws = torch.full((max(need, 16),), 255, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    mine = kv.tbn_verify(p, tokens, u, cu, 3, draft=q, parents=parents, workspace=ws, stream=side)
    side.synchronize()
    for other in (there, current, mine):
        for a, b in zip(here, other):
            assert torch.equal(a, b)
