"""Pages of the key/value cache against the oracle's lists: reserve with copy on write, fork, release, compact, copy, append, keep,
summaries; failures that change nothing; long random lives."""
import math

import numpy as np
import pytest
import torch

from oracle import kv_oracle as orc
from tests.kv_util import DT

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kv():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2407_12075_amd import kv as binding, tbn
    tbn.lib()
    return binding


def ints(x):
    return torch.tensor(list(x), dtype=torch.int32, device="cuda")


class Both:
    """The library's cache and the oracle's, side by side."""

    def __init__(self, kv, dt, n_seqs, max_pages, n_pages, page, kv_heads=2, dim=16, summary=True):
        self.kv, self.dt = kv, dt
        self.pool = kv.kv_pool(n_pages, kv_heads, dim, page, DT[dt], summary)
        self.pool.k.zero_()
        self.pool.v.zero_()
        self.index = kv.kv_index(n_seqs, max_pages, n_pages, page)
        self.o = orc.Cache(n_seqs, max_pages, n_pages, page, kv_heads, dim)

    def draw(self, rng, n):
        x = torch.from_numpy(rng.standard_normal((n, self.pool.kv_heads, self.pool.dim)) * 2.0 ** rng.randint(-8, 9)).to(DT[self.dt])
        return x.cuda(), x.double().numpy()

    def reserve(self, n_new):
        src, dst = self.kv.tbn_kv_reserve(self.index, ints(n_new))
        pairs = self.o.reserve(list(n_new))
        assert list(zip(src.tolist(), dst.tolist())) == pairs
        self.kv.tbn_kv_copy_pages(self.pool, src, dst)
        self.o.copy(pairs)
        self.check()

    def append(self, rng, n_new):
        k, kd = self.draw(rng, sum(n_new))
        v, vd = self.draw(rng, sum(n_new))
        cu = np.concatenate([[0], np.cumsum(n_new)])
        self.kv.tbn_kv_append(self.pool, self.index, k, v, ints(cu), max(n_new))
        if not self.o.status:
            for s in range(len(n_new)):
                self.o.append(s, kd[cu[s]:cu[s + 1]], vd[cu[s]:cu[s + 1]])
                self.summaries(s, self.o.lens[s] - n_new[s], self.o.lens[s])

    def summaries(self, s, begin, end):
        """Those of the pages that hold keys begin .. end - 1 are over all their keys before `end`."""
        if self.pool.summary is None or begin >= end:
            return
        P = self.pool.page
        for b in range(begin // P, -(-end // P)):
            p = self.o.rows[s][b]
            for h in range(self.pool.kv_heads):
                codes, step = orc.summary(self.o.k[p, h, :min(P, end - b * P)])
                assert np.array_equal(self.pool.summary[p, h].cpu().numpy(), codes) and float(self.pool.step[p, h]) == step

    def check(self):
        o = self.o
        assert self.index.lens.tolist() == o.lens and self.index.refs.tolist() == o.refs and int(self.index.status) == o.status
        table = self.index.table.cpu().numpy()
        for s, row in enumerate(o.rows):
            assert table[s, :len(row)].tolist() == row

    def check_data(self):
        k, v, table = self.pool.k.double().cpu().numpy(), self.pool.v.double().cpu().numpy(), self.index.table.cpu().numpy()
        P = self.pool.page
        for s, n in enumerate(self.o.lens):
            want = self.o.keys(s)
            for i in range(n):
                p = table[s, i // P]
                assert np.array_equal(k[p, :, i % P], want[0][i]) and np.array_equal(v[p, :, :, i % P], want[1][i])


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("page,heads,dim", [(32, 2, 16), (64, 1, 8), (128, 3, 80), (32, 1, 256), (64, 2, 128)])
def test_append_of_all_lengths(kv, dt, page, heads, dim):
    rng = np.random.RandomState(page + dim)
    b = Both(kv, dt, 7, 6, 60, page, heads, dim)
    for n_new in ([1, 0, page, page + 1, 2 * page - 1, 3, 0], [1, 5, 1, page - 1, 9, 0, 0], [2 * page, page, 7, 1, 0, 1, 8], [1, 1, 1, 1, 1, 1, 1]):
        b.reserve(n_new)
        b.append(rng, n_new)
        b.check()
    b.check_data()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_strided_and_unaligned_tokens(kv, dt):
    rng = np.random.RandomState(3)
    for off, stride in ((0, 2 * 16 * 2 + 8), (1, 2 * 16 * 2 + 3), (3, 2 * 16 * 2 + 16)):
        b = Both(kv, dt, 2, 4, 10, 32)
        n_new = [40, 33]
        b.reserve(n_new)
        x = torch.from_numpy(rng.standard_normal((73, stride + off))).to(DT[dt])
        dev = x.cuda()
        k, v = dev[:, off:off + 32].unflatten(1, (2, 16)), dev[:, off + 32:off + 64].unflatten(1, (2, 16))
        kv.tbn_kv_append(b.pool, b.index, k, v, ints([0, 40, 73]), 40)
        for s, (i, j) in enumerate(((0, 40), (40, 73))):
            b.o.append(s, x[i:j, off:off + 32].double().numpy().reshape(-1, 2, 16), x[i:j, off + 32:off + 64].double().numpy().reshape(-1, 2, 16))
        b.check_data()


def test_fork_copies_on_write(kv):
    rng = np.random.RandomState(0)
    b = Both(kv, "f32", 6, 4, 24, 32)
    b.reserve([40, 0, 64, 0, 0, 0])
    b.append(rng, [40, 0, 64, 0, 0, 0])
    kv.tbn_kv_fork(b.index, ints([0, 0, 2, 0]), ints([1, 3, 4, 5]))
    b.o.fork([0, 0, 2, 0], [1, 3, 4, 5])
    b.check()
    b.reserve([0, 1, 1, 2, 1, 0])        # two of four owners of a last page write: both copy; a full last page is not copied
    b.append(rng, [0, 1, 1, 2, 1, 0])
    b.reserve([1, 0, 0, 0, 0, 1])        # the other two: the first copies, the last one keeps the page
    b.append(rng, [1, 0, 0, 0, 0, 1])
    b.check_data()
    kv.tbn_kv_release(b.index, ints([33, 0, 64, 1000, -5, 32]))
    b.o.release([33, 0, 64, 1000, -5, 32])
    b.check()
    b.check_data()


def test_a_sequence_cut_back_into_a_shared_page_copies_it(kv):
    rng = np.random.RandomState(1)
    b = Both(kv, "f32", 2, 4, 12, 32)
    b.reserve([64, 0])
    b.append(rng, [64, 0])
    kv.tbn_kv_fork(b.index, ints([0]), ints([1]))
    b.o.fork([0], [1])
    kv.tbn_kv_release(b.index, ints([40, 64]))
    b.o.release([40, 64])
    b.reserve([3, 0])
    b.append(rng, [3, 0])
    b.check()
    b.check_data()


def test_pairs_that_cannot_be_forked(kv):
    b = Both(kv, "f32", 6, 4, 12, 32)
    b.reserve([10, 0, 5, 0, 0, 0])
    b.append(np.random.RandomState(0), [10, 0, 5, 0, 0, 0])
    parents, children = [0, 0, 1, 2, 0, 9, 0], [1, 1, 3, 0, -1, 4, 5]   # named twice, a child as parent, not empty, outside
    kv.tbn_kv_fork(b.index, ints(parents[:6]), ints(children[:6]))
    b.o.fork(parents[:6], children[:6])
    b.check()
    assert b.o.status == 2 and b.o.lens == [10, 0, 5, 0, 0, 0]
    b.index.status.zero_()
    b.o.status = 0
    kv.tbn_kv_fork(b.index, ints([0, 0, 2]), ints([4, 2, 5]))              # only the pair in the middle is left out
    b.o.fork([0, 0, 2], [4, 2, 5])
    b.check()
    assert b.o.status == 2 and b.o.lens == [10, 0, 5, 0, 10, 5]


def test_failures_change_nothing(kv):
    rng = np.random.RandomState(0)
    b = Both(kv, "f32", 3, 4, 5, 32)
    b.reserve([33, 10, 0])
    b.append(rng, [33, 10, 0])
    before = [t.clone() for t in (b.pool.k, b.pool.v, b.index.table, b.index.lens, b.index.refs)]
    b.reserve([32, 0, 64])               # three pages wanted, two free
    assert b.o.status == 1
    b.append(rng, [32, 0, 64])           # does nothing
    b.reserve([1, 0, 0])                 # neither
    kv.tbn_kv_keep(b.pool, b.index, ints([0, 0, 0]), ints([3, 3, 3]).view(3, 1), ints([1, 1, 1]))
    assert all(torch.equal(x, y) for x, y in zip(before, (b.pool.k, b.pool.v, b.index.table, b.index.lens, b.index.refs)))
    b.index.status.zero_()
    b.o.status = 0
    b.reserve([-1, 0, 0])
    assert b.o.status == 2
    b.index.status.zero_()
    b.o.status = 0
    b.reserve([0, 0, 2 ** 31 - 1])       # a row too short
    assert b.o.status == 2
    b.index.status.zero_()
    b.o.status = 0
    b.reserve([31, 1, 32])
    b.append(rng, [31, 1, 32])
    b.check_data()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("base,n", [(0, 20), (30, 40), (31, 3), (64, 70)])
def test_keep(kv, dt, base, n):
    rng = np.random.RandomState(base + n)
    b = Both(kv, dt, 4, 6, 40, 32, 2, 24)
    first = [base, base + 1, 5, 0]
    b.reserve(first)
    b.append(rng, first)
    new = [n, 2, 1, 0]
    b.reserve(new)
    b.append(rng, new)
    picks = np.full((4, n), 1 << 20, np.int32)
    counts = [rng.randint(1, n + 1), 1, 1, 0]
    for s in range(3):
        picks[s, :counts[s]] = np.sort(rng.permutation(new[s])[:counts[s]])
    kv.tbn_kv_keep(b.pool, b.index, ints(first), torch.from_numpy(picks).cuda(), ints(counts))
    for s in range(4):
        b.o.keep(s, first[s], picks[s, :counts[s]].tolist())
        b.summaries(s, first[s], first[s] + counts[s])
    kv.tbn_kv_release(b.index, ints(a + c for a, c in zip(first, counts)))
    b.o.release([a + c for a, c in zip(first, counts)])
    b.check()
    b.check_data()


def test_keep_leaves_out_what_is_not_there(kv):
    rng = np.random.RandomState(5)
    b = Both(kv, "f32", 2, 2, 6, 32, summary=False)
    b.reserve([20, 20])
    b.append(rng, [20, 20])
    # a pick below its place, one behind the last key, one far outside; a base outside the sequence
    kv.tbn_kv_keep(b.pool, b.index, ints([10, 30]), ints([2, 0, 10, 1 << 30, 0, 1, 2, 3]).view(2, 4), ints([4, 4]))
    b.o.keep(0, 10, [2])
    b.check_data()


@pytest.mark.parametrize("n_pages", [1, 7, 1000, 40000])
def test_compact(kv, n_pages):
    rng = np.random.RandomState(n_pages)
    n = min(n_pages, 200)
    width = max(n_pages // n, 1)
    b = Both(kv, "f32", n, width, n_pages, 32, 1, 8, summary=False)
    held = rng.permutation(n_pages)[:max(n_pages // 3, 1)]
    for i, p in enumerate(held):
        s = i % n
        if len(b.o.rows[s]) < width:
            b.o.rows[s].append(int(p))
            b.o.refs[int(p)] = 1
            b.o.lens[s] += 32
    if n > 1 and n_pages > 1:   # a shared page
        b.o.rows[n - 1], b.o.lens[n - 1] = list(b.o.rows[0]), b.o.lens[0]
        b.o.refs = [sum(p in r for r in b.o.rows) if n_pages <= 1000 else v for p, v in enumerate(b.o.refs)]
        if n_pages > 1000:
            counts = np.bincount([p for r in b.o.rows for p in r], minlength=n_pages)
            b.o.refs = counts.tolist()
    table = np.full((n, width), -1, np.int32)
    for s, r in enumerate(b.o.rows):
        table[s, :len(r)] = r
    b.index.table.copy_(torch.from_numpy(table))
    b.index.lens.copy_(ints(b.o.lens))
    b.index.refs.copy_(ints(b.o.refs))
    mark = torch.arange(n_pages, device="cuda", dtype=torch.float32)
    b.pool.k.copy_(mark.view(-1, 1, 1, 1).expand_as(b.pool.k))
    b.pool.v.copy_(-mark.view(-1, 1, 1, 1).expand_as(b.pool.v))
    old = [list(r) for r in b.o.rows]
    src, dst, count = kv.tbn_kv_compact(b.index)
    want = b.o.compact()
    c = int(count)
    assert (src[:c].tolist(), dst[:c].tolist()) == want
    kv.tbn_kv_copy_pages(b.pool, src, dst, count)
    b.check()
    for r, o in zip(b.o.rows, old):
        for p, q in zip(r, o):
            assert float(b.pool.k[p, 0, 31, 7]) == q if len(old) < 20 else True
    at = torch.tensor([p for r in b.o.rows for p in r], device="cuda")
    was = torch.tensor([float(p) for r in old for p in r], device="cuda")
    assert bool((b.pool.k[at].flatten(1) == was[:, None]).all()) and bool((b.pool.v[at].flatten(1) == -was[:, None]).all())


def test_copy_pages_with_summary_and_odd_pairs(kv):
    for dt, heads, dim, page in (("bf16", 3, 40, 32), ("f32", 8, 256, 128), ("bf16", 1, 8, 32)):
        pool = kv.kv_pool(9, heads, dim, page, DT[dt], summary=True)
        g = torch.Generator(device="cuda").manual_seed(1)
        pool.k.copy_(torch.randn(pool.k.shape, generator=g, device="cuda"))
        pool.v.copy_(torch.randn(pool.v.shape, generator=g, device="cuda"))
        pool.summary.copy_(torch.randint(-64, 65, pool.summary.shape, generator=g, device="cuda"))
        pool.step.copy_(torch.rand(pool.step.shape, generator=g, device="cuda"))
        old = [t.clone() for t in (pool.k, pool.v, pool.summary, pool.step)]
        kv.tbn_kv_copy_pages(pool, ints([3, -1, 8, 5, 9, 2, 0]), ints([1, 4, 7, -1, 4, 9, 6]))
        kv.tbn_kv_copy_pages(pool, ints([8, 3]), ints([4, 5]), ints([1]))
        for t, o in zip((pool.k, pool.v, pool.summary, pool.step), old):
            for a, p in ((3, 1), (8, 7), (0, 6), (8, 4)):
                o[p] = o[a]
            assert torch.equal(t, o)


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf, 0.0, 1e-42, 3e38, 2.0, 127.99])
def test_summaries_of_odd_keys(kv, bad):
    b = Both(kv, "f32", 1, 2, 4, 32, 1, 16)
    b.reserve([5])
    k = torch.full((5, 1, 16), 0.0 if bad in (0.0, 1e-42) else 0.3)
    k[3, 0, 2] = bad
    kv.tbn_kv_append(b.pool, b.index, k.cuda(), k.cuda(), ints([0, 5]), 5)
    b.o.append(0, k.double().numpy(), k.double().numpy())
    b.summaries(0, 0, 5)


@pytest.mark.parametrize("seed", range(6))
def test_random_lives(kv, seed):
    """Many sequences grow, fork, are cut, end and are compacted; bookkeeping equals the oracle's at every step, data at the end."""
    rng = np.random.RandomState(seed)
    n, P = int(rng.choice([3, 17, 40])), int(rng.choice([32, 64]))
    b = Both(kv, "bf16" if seed % 2 else "f32", n, 8, int(n * rng.choice([3, 6])), P, 1, 8)
    for _ in range(25):
        kind = rng.choice(["grow", "grow", "fork", "cut", "end", "compact"])
        if kind == "grow":
            new = [int(rng.choice([0, 1, 2, P - 1, P + 3])) if rng.rand() < 0.6 else 0 for _ in range(n)]
            b.reserve(new)
            if b.o.status == 0 and sum(new):
                b.append(rng, new)
            elif b.o.status:
                b.index.status.zero_()
                b.o.status = 0
        elif kind == "fork":
            m = int(rng.randint(0, n + 1))
            parents, children = rng.randint(0, n, m).tolist(), rng.permutation(n)[:m].tolist()
            kv.tbn_kv_fork(b.index, ints(parents), ints(children))
            b.o.fork(parents, children)
            b.check()
            b.index.status.zero_()
            b.o.status = 0
        elif kind in ("cut", "end"):
            keep = [(0 if kind == "end" else int(rng.randint(0, l + 2))) if rng.rand() < 0.3 else 1 << 30 for l in b.o.lens]
            kv.tbn_kv_release(b.index, ints(keep))
            b.o.release(keep)
        else:
            src, dst, count = kv.tbn_kv_compact(b.index)
            pairs = b.o.compact()
            assert (src[:int(count)].tolist(), dst[:int(count)].tolist()) == pairs
            kv.tbn_kv_copy_pages(b.pool, src, dst, count)
            b.o.copy(list(zip(*pairs)))
        b.check()
    b.check_data()


def test_many_sequences(kv):
    """Lists of thousands of sequences, pages beyond one round of the ranking."""
    n, P = 5000, 32
    rng = np.random.RandomState(9)
    b = Both(kv, "f32", n, 9, 30000, P, 1, 8, summary=False)
    new = rng.randint(0, 2 * P, n).tolist()
    b.reserve(new)
    b.reserve([int(x) for x in rng.randint(0, 70, n)])
    b.check()
