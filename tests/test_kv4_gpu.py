"""The cache held in 4 bits: what new keys become, what is read back, copies, kept keys, and attention over it, against the float64 oracle."""
import math

import numpy as np
import pytest
import torch

from oracle import kv4_oracle as o4
from oracle import kv_oracle as orc
from tests.kv4_util import host_of, make_cache4
from tests.kv_util import DT, compare, make_queries, tolerance
from tests.test_kv_attention_gpu import masks
from tests.test_kv_window_gpu import packed, reference as window_reference

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kv():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2407_12075_amd import kv as binding, tbn
    tbn.lib()
    return binding


def state(pool):
    return [t.clone() for t in (pool.k, pool.v, pool.k_exp, pool.v_exp)]


def numbers_to_store(rng, n, kv_heads, dim, dt):
    """Sizes of all kinds: ordinary ones, groups of zeros, tiny and huge ones, numbers on the borders between codes, infinities and not-a-numbers."""
    x = rng.standard_normal((n, kv_heads, dim))
    g = x.reshape(n, kv_heads, dim // 32, 32)
    g *= 2.0 ** rng.randint(-6, 6, g.shape[:3] + (1,))
    kind = rng.rand(*g.shape[:3])
    border = rng.choice([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 0.0, -0.25, -1.75, -3.5, -5.0], g.shape) * 2.0 ** rng.randint(-3, 4, g.shape[:3] + (1,))
    g[kind < 0.3] = border[kind < 0.3]
    g[kind < 0.08] = 0.0
    g[(kind > 0.96)] *= 2.0 ** -110
    g[(kind > 0.93) & (kind < 0.95)] *= 2.0 ** 119
    t = torch.from_numpy(x).float().to(DT[dt])
    bad = torch.from_numpy(rng.rand(n, kv_heads) < 0.04)
    t[bad, 7 % dim] = math.inf
    t[torch.from_numpy(rng.rand(n, kv_heads) < 0.03), 31] = math.nan
    t[0, 0, :32] = 3.3e38
    return t


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("KV,D,P,seqs", [
    (1, 32, 32, [(0, 1), (31, 1), (32, 1), (7, 2), (8, 0)]), (2, 64, 64, [(0, 70), (63, 3), (5, 1), (30, 4)]), (3, 96, 32, [(1, 40), (90, 9)]),
    (2, 128, 64, [(60, 10), (0, 64), (127, 1), (0, 0), (3, 130)]), (1, 160, 128, [(100, 60), (7, 1)]), (1, 192, 64, [(17, 20)]), (2, 224, 32, [(33, 7)]),
    (1, 256, 128, [(250, 9), (0, 33)])])
def test_append_and_read(kv, KV, D, P, seqs, dt):
    counts = [n for _, n in seqs]
    pool, index, keys, values = make_cache4(kv, KV, D, P, [p + n for p, n in seqs], seed=D)
    rng = np.random.RandomState(D + P)
    N = sum(counts)
    fused = torch.full((N, 2 * KV * D + 3), 9.0, dtype=DT[dt])      # odd stride: no alignment but the element's
    kn, vn = numbers_to_store(rng, N, KV, D, dt), numbers_to_store(rng, N, KV, D, dt)
    fused[:, 1:1 + KV * D], fused[:, 2 + KV * D:2 + 2 * KV * D] = kn.reshape(N, -1), vn.reshape(N, -1)
    fused = fused.cuda()
    k_new, v_new = fused[:, 1:1 + KV * D].unflatten(1, (KV, D)), fused[:, 2 + KV * D:2 + 2 * KV * D].unflatten(1, (KV, D))
    cu = torch.tensor([0] + list(np.cumsum(counts)), dtype=torch.int32, device="cuda")
    want, table = host_of(pool), index.table.cpu().numpy()
    i = 0
    for s, (p, n) in enumerate(seqs):
        for t in range(n):
            want.write(table[s, (p + t) // P], (p + t) % P, o4.quantize(kn[i].double().numpy(), vn[i].double().numpy()))
            i += 1
    kv.tbn_kv4_append(pool, index, k_new, v_new, cu, max(counts))
    got = host_of(pool)
    no_number = want.k_exp[..., :D // 32] == -128
    for name in ("k_exp", "v_exp"):
        assert np.array_equal(getattr(got, name)[..., :D // 32], getattr(want, name)[..., :D // 32]), name
    # codes of keys that are no numbers are free
    free = no_number[..., 0]
    assert np.array_equal(got.k[~free], want.k[~free])
    for s, (p, n) in enumerate(seqs):
        for t in range(p + n):
            page, row = table[s, t // P], t % P
            a, b = got.read(page, row), want.read(page, row)
            for h in range(KV):
                if not free[page, h, row]:
                    assert np.array_equal(a[1][h], b[1][h]), (s, t, h)
    # pages that no sequence holds, and rows behind the last key, are as they were
    used = {int(table[s, j]) for s, (p, n) in enumerate(seqs) for j in range(-(-(p + n) // P))}
    before = make_cache4(kv, KV, D, P, [p + n for p, n in seqs], seed=D)[0]
    for page in set(range(index.n_pages)) - used:
        assert torch.equal(pool.v[page], before.v[page]) and torch.equal(pool.k[page], before.k[page])
    # read back: all keys of every sequence, and the last of some
    lens = [p + n for p, n in seqs]
    for ask in (lens, [min(l, 3 + s) for s, l in enumerate(lens)], counts):
        cu_r = torch.tensor([0] + list(np.cumsum(ask)), dtype=torch.int32, device="cuda")
        if not sum(ask):
            continue
        for dtype in (torch.float32, torch.bfloat16):
            kr, vr = kv.tbn_kv4_read(pool, index, cu_r, max(ask), sum(ask), dtype)
            i = 0
            for s, l in enumerate(lens):
                for t in range(l - ask[s], l):
                    kc, vc, ke, ve = want.read(table[s, t // P], t % P)
                    assert np.array_equal(kr[i].double().cpu().numpy(), o4.numbers(kc, ke), equal_nan=True)
                    assert np.array_equal(vr[i].double().cpu().numpy(), o4.numbers(vc, ve), equal_nan=True)
                    i += 1


def test_appending_token_by_token_is_appending_at_once(kv):
    D, P, n = 64, 32, 45
    rng = np.random.RandomState(3)
    kn, vn = (torch.from_numpy(rng.standard_normal((n, 2, D))).to(torch.bfloat16).cuda() for _ in range(2))
    a, b = kv.kv4_pool(4, 2, D, P), kv.kv4_pool(4, 2, D, P)
    for pool in (a, b):
        for t in (pool.k, pool.v, pool.k_exp, pool.v_exp):
            t.zero_()
    ia, ib = kv.kv_index(1, 3, 4, P), kv.kv_index(1, 3, 4, P)
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    kv.tbn_kv_reserve(ia, ints(n))
    kv.tbn_kv4_append(a, ia, kn, vn, ints(0, n), n)
    for i in range(n):
        kv.tbn_kv_reserve(ib, ints(1))
        kv.tbn_kv4_append(b, ib, kn[i:i + 1], vn[i:i + 1], ints(0, 1), 1)
    assert torch.equal(ia.table, ib.table)
    assert all(torch.equal(x, y) for x, y in zip(state(a), state(b)))
    # a failed step appends nothing
    before = state(a)
    kv.tbn_kv_reserve(ia, ints(1000))
    assert int(ia.status) == 2
    kv.tbn_kv4_append(a, ia, -kn, -vn, ints(0, n), n)
    assert all(torch.equal(x, y) for x, y in zip(state(a), before))


@pytest.mark.parametrize("KV,D,P", [(2, 64, 32), (3, 96, 64), (1, 256, 128), (9, 128, 128)])
def test_copy_pages(kv, KV, D, P):
    pool, _, _, _ = make_cache4(kv, KV, D, P, [3 * P], seed=4, n_pages=9)
    want = [t.clone() for t in state(pool)]
    src, dst = [0, -1, 7, 3, 9], [5, 2, -1, 1, 4]
    for t in want:
        t[5], t[1] = t[0], t[3]
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    kv.tbn_kv4_copy_pages(pool, ints(src), ints(dst))
    assert all(torch.equal(x, y) for x, y in zip(state(pool), want))
    kv.tbn_kv4_copy_pages(pool, ints([8, 1]), ints([6, 2]), count=ints([1]))
    for t in want:
        t[6] = t[8]
    assert all(torch.equal(x, y) for x, y in zip(state(pool), want))


@pytest.mark.parametrize("KV,D,P", [(2, 64, 32), (1, 160, 64), (2, 128, 128)])
def test_keep(kv, KV, D, P):
    lens, base = [100, 40, 7, 300, 20], [60, 33, 7, 3, -4]
    picks = [[0, 2, 3, 9, 38, 1000], [1, 1, 6, 6, 0, 0], [0, 1, 2, 3, 4, 5], list(range(0, 280, 2)), [1, 2, 3, 4, 5, 6]]
    counts = [5, 3, 4, 140, 2]
    pool, index, _, _ = make_cache4(kv, KV, D, P, lens, seed=11)
    want, table = host_of(pool), index.table.cpu().numpy()
    for s in range(5):
        if base[s] < 0:
            continue
        got = []
        for j in range(min(counts[s], lens[s] - base[s])):
            f = picks[s][j]
            got.append(want.read(table[s, (base[s] + f) // P], (base[s] + f) % P) if j < f < lens[s] - base[s] else None)
        for j, c in enumerate(got):
            if c is not None:
                want.write(table[s, (base[s] + j) // P], (base[s] + j) % P, c)
    width = max(map(len, picks))
    rows = torch.tensor([p + [0] * (width - len(p)) for p in picks], dtype=torch.int32, device="cuda")
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    kv.tbn_kv4_keep(pool, index, ints(base), rows, ints(counts))
    got = host_of(pool)
    assert np.array_equal(got.k, want.k) and np.array_equal(got.v, want.v)
    assert np.array_equal(got.k_exp[..., :D // 32], want.k_exp[..., :D // 32]) and np.array_equal(got.v_exp[..., :D // 32], want.v_exp[..., :D // 32])


def everything(qs, keys, values, counts, see, scale):
    return window_reference(qs, keys, values, counts, 0, 1 << 30, see, scale)


CASES = [
    # heads, kv heads, dim, page, [(keys before, tokens)]
    (4, 1, 64, 32, [(0, 1), (30, 1), (31, 1), (32, 1), (63, 2)]),
    (8, 2, 128, 64, [(62, 1), (63, 1), (64, 1), (65, 1), (200, 3), (0, 5)]),
    (6, 6, 64, 32, [(97, 13), (5, 7), (0, 0), (33, 1)]),
    (5, 1, 128, 128, [(127, 1), (128, 1), (300, 4)]),
    (20, 1, 64, 64, [(70, 3), (1, 1)]),
    (2, 1, 32, 32, [(40, 6), (0, 3)]),
    (4, 4, 96, 64, [(129, 2)]),
    (2, 1, 160, 64, [(100, 5)]),
    (4, 2, 192, 32, [(90, 5), (3, 1)]),
    (2, 2, 224, 128, [(200, 3)]),
    (8, 2, 256, 64, [(77, 6), (10, 1)]),
    (8, 1, 64, 64, [(150, 70), (0, 40)]),
    (4, 1, 128, 64, [(90, 33), (513, 32)]),
]


@pytest.mark.parametrize("kind", ["none", "tree", "any"])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("H,KV,D,P,seqs", CASES)
def test_attention(kv, H, KV, D, P, seqs, dt, kind):
    counts = [n for _, n in seqs]
    pool, index, keys, values = make_cache4(kv, KV, D, P, [p + n for p, n in seqs], seed=H * D)
    q, cu, qs = make_queries(dt, counts, H, D, stride=H * D + 5)
    see = masks("chain" if kind == "none" else kind, counts, 3)
    mask = None if kind == "none" else packed(see, counts)
    scale = 1.0 / math.sqrt(D)
    out, lse = kv.tbn_kv4_attention(q, pool, index, cu, max(counts), mask=mask)
    compare(out, lse, *everything(qs, keys, values, counts, see if mask is not None else None, scale), tolerance(dt, values))
    out2, lse2 = kv.tbn_kv4_attention(q, pool, index, cu, max(counts), mask=mask, scale=-scale, max_len=max(p + n for p, n in seqs))
    compare(out2, lse2, *everything(qs, keys, values, counts, see if mask is not None else None, -scale), tolerance(dt, values))


@pytest.mark.parametrize("sink,window", [(0, 1), (4, 1), (3, 75), (64, 97), (5, 100000)])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("H,KV,D,P,seqs", [
    (4, 1, 64, 32, [(0, 1), (30, 1), (31, 1), (63, 2)]), (8, 2, 128, 64, [(62, 1), (64, 1), (700, 3), (0, 5)]), (5, 1, 128, 128, [(127, 1), (900, 4)]),
    (2, 1, 256, 64, [(377, 6), (10, 1)]), (8, 1, 96, 64, [(450, 70), (0, 40)]), (4, 1, 128, 32, [(390, 33), (813, 32)])])
def test_window(kv, H, KV, D, P, seqs, dt, sink, window):
    counts = [n for _, n in seqs]
    pool, index, keys, values = make_cache4(kv, KV, D, P, [p + n for p, n in seqs], seed=H * D)
    q, cu, qs = make_queries(dt, counts, H, D)
    scale = 1.0 / math.sqrt(D)
    out, lse = kv.tbn_kv4_attention(q, pool, index, cu, max(counts), n_sink=sink, window=window)
    compare(out, lse, *window_reference(qs, keys, values, counts, sink, window, None, scale), tolerance(dt, values))
    if max(counts) <= window:
        see = masks("any", counts, 3)
        out, lse = kv.tbn_kv4_attention(q, pool, index, cu, max(counts), mask=packed(see, counts), n_sink=sink, window=window)
        compare(out, lse, *window_reference(qs, keys, values, counts, sink, window, see, scale), tolerance(dt, values))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("H,KV,D,P,seqs", [
    (8, 2, 128, 64, [(5000, 1)]), (4, 1, 64, 32, [(7000, 11), (100, 2), (0, 1)]), (2, 1, 256, 128, [(3000, 3)]), (8, 8, 64, 64, [(2048, 1), (2049, 1), (255, 1)]),
    (16, 1, 64, 64, [(1500, 20)]), (4, 2, 128, 64, [(1000, 300), (0, 200)])])
def test_many_keys_and_rows(kv, H, KV, D, P, seqs, dt):
    counts = [n for _, n in seqs]
    pool, index, keys, values = make_cache4(kv, KV, D, P, [p + n for p, n in seqs], seed=5)
    q, cu, qs = make_queries(dt, counts, H, D)
    for kind in ("none", "tree") if max(counts) < 64 else ("none",):
        see = masks(kind, counts, 9) if kind != "none" else None
        mask = packed(see, counts) if see else None
        out, lse = kv.tbn_kv4_attention(q, pool, index, cu, max(counts), mask=mask)
        compare(out, lse, *everything(qs, keys, values, counts, see, 1 / math.sqrt(D)), tolerance(dt, values))
        again, lse2 = kv.tbn_kv4_attention(q, pool, index, cu, max(counts), mask=mask)
        assert torch.equal(out, again) and torch.equal(lse, lse2)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("H,KV,D,P", [(4, 2, 64, 32), (32, 1, 128, 64), (8, 1, 256, 128), (8, 8, 96, 64)])
def test_keys_that_are_no_numbers(kv, H, KV, D, P, dt):
    """Rows that see one are not-a-number all over, the others do not notice; also rows without a visible key."""
    counts = [9, 2, 40]
    pool, index, keys, values = make_cache4(kv, KV, D, P, [80, 12, 41], seed=13, no_number=0.15)
    for s in range(3):   # most rows see only numbers among the keys before
        n = len(keys[s]) - counts[s]
        keep = np.isnan(keys[s][:n]).any((1, 2))
        for t in np.nonzero(keep)[0]:
            page, row = int(index.table[s, t // P]), t % P
            pool.k_exp[page, :, row] = 0
            pool.v_exp[page, :, row] = 0
            host = host_of(pool).read(page, row)
            keys[s][t], values[s][t] = o4.numbers(host[0], host[2]), o4.numbers(host[1], host[3])
    q, cu, qs = make_queries(dt, counts, H, D)
    see = masks("any", counts, 5)
    for t in range(0, 40, 7):
        see[2][t] = False
    mask = packed(see, counts)
    ref = everything(qs, keys, values, counts, see, 0.11)
    out, lse = kv.tbn_kv4_attention(q, pool, index, cu, max(counts), mask=mask, scale=0.11)
    assert np.isnan(ref[0]).any() and np.isfinite(ref[0]).any()
    compare(out, lse, *ref, tolerance(dt, values))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_infinite_logits_and_queries(kv, dt):
    """A logit of +infinity: lse is +infinity and out no number; all of -infinity: as if no key were seen; a query that is no number: that all over."""
    pool, index, keys, values = make_cache4(kv, 1, 64, 32, [70], seed=14)
    pool.k[:], pool.k_exp[:] = 0x22, 100     # every key is 2^100 in all channels
    q = torch.zeros(3, 2, 64, dtype=DT[dt], device="cuda")
    q[0] = 1e30
    q[1] = -1e30
    q[2, 0, 5] = math.nan
    q[2, 1, 5] = 1.0
    cu = torch.tensor([0, 3], dtype=torch.int32, device="cuda")
    out, lse = kv.tbn_kv4_attention(q, pool, index, cu, 3, scale=1.0)
    assert torch.isnan(out[0]).all() and (lse[0] == math.inf).all()
    assert (out[1] == 0).all() and (lse[1] == -math.inf).all()
    assert torch.isnan(out[2, 0]).all() and torch.isnan(lse[2, 0])
    assert torch.isfinite(out[2, 1].float()).all()


def test_float32_is_not_lost(kv):
    """Small differences of large logits, long sums: float32 queries are not rounded to bfloat16."""
    pool, index, keys, values = make_cache4(kv, 2, 128, 64, [3000, 1], seed=15)
    q, cu, qs = make_queries("f32", [1, 1], 4, 128, scale=6.0)
    out, lse = kv.tbn_kv4_attention(q, pool, index, cu, 1, scale=0.3)
    ref, ref_lse = everything(qs, keys, values, [1, 1], None, float(np.float32(0.3)))
    # logits of up to about 100 from 128 products: 128 * 2^-24 * 100 / 4 of error at most, relative to the weights
    assert np.abs(out.double().cpu().numpy() - ref).max() <= 2e-4 * max(np.abs(v).max() for v in values)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_idle_places_streams_and_outputs(kv, dt):
    lens = [0] * 20 + [5000] + [0] * 10 + [40]
    counts = [0] * 20 + [1] + [0] * 10 + [1]
    pool, index, keys, values = make_cache4(kv, 2, 128, 64, lens, seed=9)
    q, cu, qs = make_queries(dt, counts, 8, 128)
    out, lse = kv.tbn_kv4_attention(q, pool, index, cu, 1)
    compare(out, lse, *everything(qs, keys, values, counts, None, 1 / math.sqrt(128)), tolerance(dt, values))
    need = kv.tbn_kv4_attention_workspace_bytes(q, pool, index, 1)
    assert need > 0
    mine, mine_lse = torch.full_like(out, 7.0), torch.full_like(lse, 7.0)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    r = kv.tbn_kv4_attention(q, pool, index, cu, 1, out=mine, lse=mine_lse, workspace=torch.empty(need, dtype=torch.uint8, device="cuda"), stream=side)
    k2, _ = kv.tbn_kv4_read(pool, index, torch.tensor([0] * 21 + [3] * 11 + [5], dtype=torch.int32, device="cuda"), 3, 5, stream=side)
    side.synchronize()
    assert r[0] is mine and torch.equal(mine, out) and torch.equal(mine_lse, lse)
    assert np.array_equal(k2.double().cpu().numpy(), np.concatenate([keys[20][-3:], keys[31][-2:]]))


def test_graph(kv):
    """A step of bookkeeping, append and attention, captured and replayed."""
    KV, D, P = 2, 64, 32
    pool, index, _, _ = make_cache4(kv, KV, D, P, [100, 31], seed=17, n_pages=20, max_pages=8)
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    one, cu = ints(1, 1), ints(0, 1, 2)
    x = torch.zeros(2, 3 * KV, D, dtype=torch.bfloat16, device="cuda")

    def step(pool, index):
        src, dst = kv.tbn_kv_reserve(index, one)
        kv.tbn_kv4_copy_pages(pool, src, dst)
        kv.tbn_kv4_append(pool, index, x[:, KV:2 * KV], x[:, 2 * KV:], cu, 1)
        return kv.tbn_kv4_attention(x[:, :KV], pool, index, cu, 1, n_sink=2, window=40)

    def copy():
        i2 = kv.KVIndex(index.table.clone(), index.lens.clone(), index.refs.clone(), index.status.clone(), P)
        return kv.KV4Pool(*state(pool)), i2

    step(*copy())
    torch.cuda.synchronize()
    other, oi = copy()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out, lse = step(pool, index)
    for i in range(4):
        x.copy_(torch.randn(2, 3 * KV, D, generator=torch.Generator().manual_seed(i)))
        g.replay()
        torch.cuda.synchronize()
        want, want_lse = step(other, oi)
        assert torch.equal(out, want) and torch.equal(lse, want_lse)
    assert int(index.status) == 0 and index.lens.tolist() == [104, 35]
    assert all(torch.equal(a, b) for a, b in zip(state(pool), state(other)))


def test_refusals(kv):
    from paper_2407_12075_amd import tbn
    pool, index, _, _ = make_cache4(kv, 2, 64, 32, [50, 60])
    q, cu, _ = make_queries("bf16", [3, 2], 4, 64)
    mask = torch.ones(5, 1, dtype=torch.int32, device="cuda")
    for kw in (dict(n_sink=-1, window=5), dict(window=-1), dict(window=2, mask=mask)):
        with pytest.raises(tbn.TbnError) as e:
            kv.tbn_kv4_attention(q, pool, index, cu, 3, **kw)
        assert e.value.status == 2
    for bad in (q.half(), q[:, :, :32], q.cpu(), q.transpose(0, 1)):
        with pytest.raises(ValueError):
            kv.tbn_kv4_attention(bad, pool, index, cu, 3)
    k = torch.zeros(5, 2, 64, device="cuda")
    with pytest.raises(ValueError):
        kv.tbn_kv4_append(pool, index, k, k.bfloat16(), cu, 3)
    with pytest.raises(ValueError):
        kv.tbn_kv4_append(pool, index, k, k[:4], cu, 3)
    with pytest.raises(ValueError):
        kv.tbn_kv4_read(pool, index, cu, 3, 5, torch.float16)
    with pytest.raises(ValueError):
        kv.KV4Pool(pool.k, pool.v.view(torch.int8), pool.k_exp, pool.v_exp)
    with pytest.raises(ValueError):
        kv.KV4Pool(pool.k, pool.v, pool.k_exp[..., :2].contiguous(), pool.v_exp)
    with pytest.raises(ValueError):
        kv.kv4_pool(4, 2, 80, 32)
