"""Attention over the paged cache against the float64 oracle: trees of drafted tokens, chains, single tokens, empty rows, pages that
end inside a step, garbage behind the last key, infinities and not-a-numbers in masked places, strides, far pages, picked blocks."""
import math

import numpy as np
import pytest
import torch

from oracle import kv_oracle as orc
from tests.kv_util import compare, make_cache, make_queries, pack_mask, tolerance

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kv():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2407_12075_amd import kv as binding, tbn
    tbn.lib()
    return binding


def tree_rows(rng, n):
    """Ancestors of each of n drafted tokens, itself included."""
    see = np.zeros((n, n), bool)
    for i in range(n):
        parent = rng.randint(-1, i) if i else -1
        if parent >= 0:
            see[i] = see[parent]
        see[i, i] = True
    return see


def masks(kind, counts, seed):
    rng = np.random.RandomState(seed)
    rows = []
    for n in counts:
        if kind == "chain":
            rows.append(np.tril(np.ones((n, n), bool)))
        elif kind == "tree":
            rows.append(tree_rows(rng, n))
        else:   # anything, rows without a bit among them
            see = rng.rand(n, n) < 0.4
            see[rng.rand(n) < 0.3] = False
            rows.append(see)
    return rows


def reference(qs, keys, values, counts, see, scale):
    """see: per sequence (T, T) for its last T keys."""
    H, D = qs.shape[1:]
    out, lse = np.zeros(qs.shape), np.zeros(qs.shape[:2])
    at = 0
    for s, n in enumerate(counts):
        k, v = keys[s], values[s]
        G, prefix = H // k.shape[1], len(k) - n
        for t in range(n):
            row = np.concatenate([np.ones(prefix, bool), see[s][t]])
            for h in range(H):
                out[at, h], lse[at, h] = orc.attention(qs[at, h], k[:, h // G], v[:, h // G], row, scale)
            at += 1
    return out, lse


CASES = [
    # heads, kv heads, dim, page, [(keys before, tokens)]
    (4, 1, 64, 32, [(0, 1), (30, 1), (31, 1), (32, 1), (63, 2)]),
    (8, 2, 128, 64, [(62, 1), (63, 1), (64, 1), (65, 1), (200, 3), (0, 5)]),
    (6, 6, 64, 32, [(97, 13), (5, 7), (0, 0), (33, 1)]),                    # one head per kv head, a sequence without tokens
    (5, 1, 128, 128, [(127, 1), (128, 1), (300, 4)]),                       # five heads share one
    (20, 1, 64, 64, [(70, 3), (1, 1)]),                                     # more heads of a group than a tile has rows
    (4, 2, 80, 32, [(50, 9), (100, 2)]),                                    # channels that end inside an operand
    (2, 1, 8, 32, [(40, 6), (0, 3)]),
    (4, 4, 96, 64, [(129, 2)]),
    (2, 1, 136, 64, [(100, 5)]),
    (8, 2, 256, 64, [(77, 6), (10, 1)]),
    (8, 1, 64, 64, [(150, 70), (0, 40)]),                                   # masks of several words, several tiles of rows
    (4, 1, 128, 64, [(90, 33), (513, 32)]),
]


@pytest.mark.parametrize("kind", ["none", "tree", "any"])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("H,KV,D,P,seqs", CASES)
def test_tree_attention(kv, H, KV, D, P, seqs, dt, kind):
    counts = [n for _, n in seqs]
    pool, index, keys, values = make_cache(kv, dt, KV, D, P, [p + n for p, n in seqs], seed=H * D)
    q, cu, qs = make_queries(dt, counts, H, D)
    see = masks("chain" if kind == "none" else kind, counts, 3)
    words = -(-max(counts) // 32) + 1   # one more than needed
    mask = None if kind == "none" else pack_mask(np.concatenate([np.pad(m, ((0, 0), (0, words * 32 - m.shape[1]))) for m in see]), words)
    scale = 1.0 / math.sqrt(D)
    out, lse = kv.tbn_tree_attention(q, pool, index, cu, max(counts), mask=mask)
    compare(out, lse, *reference(qs, keys, values, counts, see, scale), tolerance(dt, values))
    # a bound on the lengths changes nothing that can be seen but the split of the keys
    out2, lse2 = kv.tbn_tree_attention(q, pool, index, cu, max(counts), mask=mask, scale=scale, max_len=max(p + n for p, n in seqs))
    compare(out2, lse2, out.double().cpu().numpy(), lse.double().cpu().numpy(), tolerance(dt, values))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("H,KV,D,P,seqs", [
    (8, 2, 128, 64, [(5000, 1)]), (4, 1, 64, 32, [(7000, 11), (100, 2), (0, 1)]), (2, 1, 256, 128, [(3000, 3)]), (8, 8, 64, 64, [(2048, 1), (2049, 1), (255, 1)]),
    (16, 1, 64, 64, [(1500, 20)])])
def test_keys_split_over_workgroups(kv, H, KV, D, P, seqs, dt):
    counts = [n for _, n in seqs]
    pool, index, keys, values = make_cache(kv, dt, KV, D, P, [p + n for p, n in seqs], seed=5)
    q, cu, qs = make_queries(dt, counts, H, D)
    assert kv.tbn_tree_attention_workspace_bytes(q, pool, index, max(counts)) > 0
    for kind in ("chain", "tree"):
        see = masks(kind, counts, 9)
        mask = None
        if kind == "tree":
            mask = pack_mask(np.concatenate([np.pad(m, ((0, 0), (0, 32 - m.shape[1]))) for m in see]), 1)
        out, lse = kv.tbn_tree_attention(q, pool, index, cu, max(counts), mask=mask)
        compare(out, lse, *reference(qs, keys, values, counts, see, 1 / math.sqrt(D)), tolerance(dt, values))
        again, lse2 = kv.tbn_tree_attention(q, pool, index, cu, max(counts), mask=mask)
        assert torch.equal(out, again) and torch.equal(lse, lse2)


@pytest.mark.parametrize("H,KV,D,P,seqs", [
    (4, 4, 128, 64, [(33000, 1), (0, 1), (700, 1)]),                        # one row, stretches that most sequences do not reach
    (8, 8, 104, 128, [(17100, 2)]),                                         # channels that end inside an operand
    (10, 2, 128, 32, [(9001, 3)] * 8),                                      # 15 rows, pages of half a step
    (64, 64, 128, 64, [(1500, 1), (1, 1), (1023, 2), (0, 0), (64, 1), (2, 2), (130, 1), (640, 1)])])   # a stretch is a sequence
def test_few_rows_on_many_keys(kv, H, KV, D, P, seqs):
    """bfloat16, few rows, enough keys for every CU: the kernel that stages keys in LDS."""
    counts = [n for _, n in seqs]
    pool, index, keys, values = make_cache(kv, "bf16", KV, D, P, [p + n for p, n in seqs], seed=8)
    q, cu, qs = make_queries("bf16", counts, H, D)
    see = masks("any", counts, 4)
    mask = pack_mask(np.concatenate([np.pad(m, ((0, 0), (0, 32 - m.shape[1]))) for m in see]), 1)
    ref = reference(qs, keys, values, counts, see, 1 / math.sqrt(D))
    out, lse = kv.tbn_tree_attention(q, pool, index, cu, max(counts), mask=mask)
    compare(out, lse, *ref, tolerance("bf16", values))
    again, lse2 = kv.tbn_tree_attention(q, pool, index, cu, max(counts), mask=mask)
    assert torch.equal(out, again) and torch.equal(lse, lse2)


@pytest.mark.parametrize("H,KV,D", [(4, 2, 256), (2, 1, 128), (6, 6, 64)])
def test_float32_is_not_lost_in_long_sums(kv, H, KV, D):
    """A logit of magnitude up to 8 is summed in chains of at most 64 products: about sqrt(64) roundings of 2^-24 of it, 8 * 8 * 2^-24 / 2 = 2e-6 at worst
    and a fifth of that in the mean, since the partial sums are mostly smaller; it is what a weight is off by."""
    pool, index, keys, values = make_cache(kv, "f32", KV, D, 64, [1814, 700], seed=3)
    q, cu, qs = make_queries("f32", [1, 1], H, D)
    out, _ = kv.tbn_tree_attention(q, pool, index, cu, 1)
    ref, _ = reference(qs, keys, values, [1, 1], masks("chain", [1, 1], 0), 1 / math.sqrt(D))
    err = np.linalg.norm(out.double().cpu().numpy() - ref) / np.linalg.norm(ref)
    assert err <= 1e-6, f"{err:.2e}"


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_what_a_query_does_not_see_has_no_part(kv, dt, bad):
    """Drafted keys and values that hold `bad`: rows that see them show it, the others are as without it."""
    H, KV, D, P, prefix, n = 4, 2, 64, 32, 45, 24
    for where in ("key", "value"):
        pool, index, keys, values = make_cache(kv, dt, KV, D, P, [prefix + n], seed=2)
        table = index.table.cpu().numpy()[0]
        for j, d in ((3, 5), (10, 0), (17, 63), (23, 33)):
            at = prefix + j
            if where == "key":
                keys[0][at, :, d] = bad
                pool.k[int(table[at // P]), :, at % P, d] = bad
            else:
                values[0][at, :, d] = bad
                pool.v[int(table[at // P]), :, d, at % P] = bad
        q, cu, qs = make_queries(dt, [n], H, D)
        if where == "key":
            # infinite logits: keep those of them that are +infinity away from the reference's inf - inf by a common sign
            sign = np.sign(bad) if math.isinf(bad) else 1.0
            for _, d in ((3, 5), (10, 0), (17, 63), (23, 33)):
                qs[:, :, d] = -sign * np.abs(qs[:, :, d]) - sign * 0.01
            qs = torch.from_numpy(qs).to(q.dtype).double().numpy()
            q.copy_(torch.from_numpy(qs))
        for kind in ("tree", "any", "chain"):
            see = masks(kind, [n], 4)
            mask = None if kind == "chain" else pack_mask(see[0], 1)
            out, lse = kv.tbn_tree_attention(q, pool, index, cu, n, mask=mask)
            ref, ref_lse = reference(qs, keys, values, [n], see, 1 / math.sqrt(D))
            compare(out, lse, ref, ref_lse, tolerance(dt, values))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_both_infinities_of_values_cancel_to_nan(kv, dt):
    pool, index, keys, values = make_cache(kv, dt, 1, 64, 32, [40], seed=2)
    p = int(index.table[0, 1])
    for j, x in ((0, math.inf), (1, -math.inf), (2, math.inf)):
        pool.v[p, 0, j // 2, j] = x   # channel 0: both, channel 1: +infinity
        values[0][32 + j, 0, j // 2] = x
    q, cu, qs = make_queries(dt, [8], 2, 64)
    ref, ref_lse = reference(qs, keys, values, [8], [np.tril(np.ones((8, 8), bool))], 0.125)
    assert np.isnan(ref[7, 0, 0]) and ref[7, 0, 1] == math.inf and ref[0, 0, 0] == math.inf
    compare(*kv.tbn_tree_attention(q, pool, index, cu, 8), ref, ref_lse, tolerance(dt, values))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_empty_sequences_and_rows(kv, dt):
    pool, index, _, _ = make_cache(kv, dt, 2, 64, 32, [0, 5, 0], seed=1)
    q, cu, _ = make_queries(dt, [2, 5, 0], 4, 64)
    out = torch.full_like(q, 7.0)
    lse = torch.zeros(7, 4, device="cuda")
    mask = torch.zeros(7, 1, dtype=torch.int32, device="cuda")   # nobody sees anything; the first sequence has fewer keys than tokens
    kv.tbn_tree_attention(q, pool, index, cu, 5, mask=mask, out=out, lse=lse)
    assert bool((out == 0).all()) and bool(torch.isneginf(lse).all())
    o, l = kv.tbn_tree_attention(q[:0], pool, index, torch.zeros(4, dtype=torch.int32, device="cuda"), 0)
    assert o.shape == (0, 4, 64) and l.shape == (0, 4)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("pad", [0, 8, 3])
def test_strided_queries(kv, dt, pad):
    counts = [3, 1, 6]
    pool, index, keys, values = make_cache(kv, dt, 2, 64, 64, [70, 33, 129], seed=8)
    q, cu, qs = make_queries(dt, counts, 4, 64, stride=4 * 64 + 256 + pad)
    q2, _, _ = make_queries(dt, counts, 4, 64)
    a = kv.tbn_tree_attention(q, pool, index, cu, 6)
    b = kv.tbn_tree_attention(q2, pool, index, cu, 6)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_peaked_and_large_logits(kv, dt):
    """Logits of hundreds: the running maximum is what keeps the weights finite."""
    pool, index, keys, values = make_cache(kv, dt, 1, 64, 32, [300], seed=3)
    q, cu, qs = make_queries(dt, [4], 2, 64, scale=40.0)
    ref, ref_lse = reference(qs, keys, values, [4], [np.tril(np.ones((4, 4), bool))], 1.0)
    out, lse = kv.tbn_tree_attention(q, pool, index, cu, 4, scale=1.0)
    # logits of up to some 2000, off by 2^-23 of that: weights off by 1e-3 where two compete
    err = np.abs(out.double().cpu().numpy() - ref).max()
    assert err <= tolerance(dt, values) + 2e-3 * np.abs(values[0]).max()
    np.testing.assert_allclose(lse.double().cpu().numpy(), ref_lse, rtol=2e-6, atol=1e-3)


def test_pages_beyond_32_bit_offsets(kv):
    """Pages behind the first 2^32 bytes and 2^31 elements of k and v."""
    pool, index, keys, values = make_cache(kv, "bf16", 8, 128, 128, [200, 129, 1], seed=6, n_pages=17000, far=True)
    assert pool.k.numel() > 2 ** 31 and int(index.table[0, 0]) * pool.k[0].numel() > 2 ** 31
    q, cu, qs = make_queries("bf16", [2, 1, 1], 8, 128)
    ref = reference(qs, keys, values, [2, 1, 1], [np.tril(np.ones((n, n), bool)) for n in (2, 1, 1)], 1 / math.sqrt(128))
    compare(*kv.tbn_tree_attention(q, pool, index, cu, 2), *ref, tolerance("bf16", values))
    picks = torch.zeros(4, 8, 3, dtype=torch.int32, device="cuda")
    picks[:, :, 1], picks[:, :, 2] = 1, -1
    compare(*kv.tbn_block_attention(q, pool, index, cu, 2, picks), *ref, tolerance("bf16", values))
    # and the copy of such a page
    kv.tbn_kv_copy_pages(pool, index.table[0, :1].contiguous(), torch.zeros(1, dtype=torch.int32, device="cuda"))
    assert torch.equal(pool.k[0], pool.k[int(index.table[0, 0])]) and torch.equal(pool.v[0], pool.v[int(index.table[0, 0])])


def block_reference(qs, keys, values, counts, picks, P, scale):
    H = qs.shape[1]
    out, lse, at = np.zeros(qs.shape), np.zeros(qs.shape[:2]), 0
    for s, n in enumerate(counts):
        k, v = keys[s], values[s]
        G = H // k.shape[1]
        for t in range(n):
            own = len(k) - n + t
            for h in range(H):
                see = np.isin(np.arange(len(k)) // P, [b for b in picks[at][h // G] if b >= 0]) & (np.arange(len(k)) <= own)
                out[at, h], lse[at, h] = orc.attention(qs[at, h], k[:, h // G], v[:, h // G], see, scale)
            at += 1
    return out, lse


def oracle_picks(qs, keys, counts, P, n, sink, recent):
    H, D = qs.shape[1:]
    rows, at = [], 0
    for s, c in enumerate(counts):
        k = keys[s]
        KV = k.shape[1]
        G = H // KV
        sums = [[orc.summary(k[b:b + P, h]) for b in range(0, len(k), P)] for h in range(KV)]
        for t in range(c):
            own = (len(k) - c + t) // P
            rows.append([])
            for h in range(KV):
                codes = np.array([x[0] for x in sums[h]])
                got = orc.picks(qs[at, h * G:(h + 1) * G], codes, [x[1] for x in sums[h]], own, n, sink, recent)
                rows[-1].append(got + [-1] * (n - len(got)))
            at += 1
    return np.array(rows)


def set_summary(pool, index, keys, P):
    for s, k in enumerate(keys):
        for b in range(0, len(k), P):
            for h in range(k.shape[1]):
                codes, step = orc.summary(k[b:b + P, h])
                p = int(index.table[s, b // P])
                pool.summary[p, h] = torch.from_numpy(codes.astype(np.int8)).cuda()
                pool.step[p, h] = step


BLOCKS = [
    # heads, kv heads, dim, page, [(keys before, tokens)], n_select, n_sink, n_recent
    (4, 1, 64, 32, [(400, 1), (31, 1), (0, 1), (96, 3)], 5, 1, 1),
    (8, 2, 128, 64, [(1000, 2), (640, 5)], 6, 1, 2),
    (6, 6, 64, 32, [(700, 4), (0, 0), (255, 1)], 7, 0, 1),
    (5, 1, 80, 64, [(900, 3)], 4, 2, 2),         # nothing left to choose
    (20, 1, 64, 32, [(500, 2)], 9, 0, 3),        # more heads than rows of a tile
    (2, 1, 8, 32, [(300, 30)], 3, 1, 1),
    (4, 2, 256, 128, [(1500, 2)], 5, 1, 1),
    (4, 1, 64, 32, [(640, 1)], 40, 1, 1),        # more picks than blocks
    (1, 1, 64, 32, [(100, 1)], 1, 0, 1),
]


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("H,KV,D,P,seqs,n,sink,recent", BLOCKS)
def test_picked_blocks(kv, H, KV, D, P, seqs, n, sink, recent, dt):
    counts = [c for _, c in seqs]
    pool, index, keys, values = make_cache(kv, dt, KV, D, P, [p + c for p, c in seqs], seed=D + n, summary=True)
    set_summary(pool, index, keys, P)
    q, cu, qs = make_queries(dt, counts, H, D, stride=H * D + 40)
    picks = kv.tbn_block_select(q, pool, index, cu, max(counts), n, n_sink=sink, n_recent=recent)
    want = oracle_picks(qs, keys, counts, P, n, sink, recent)
    assert np.array_equal(picks.cpu().numpy(), want)
    out, lse = kv.tbn_block_attention(q, pool, index, cu, max(counts), picks)
    compare(out, lse, *block_reference(qs, keys, values, counts, want, P, 1 / math.sqrt(D)), tolerance(dt, values))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_picks_are_passed_over(kv, dt):
    """-1 in front, blocks behind the query's own, numbers far outside, no picks at all."""
    pool, index, keys, values = make_cache(kv, dt, 1, 64, 32, [200], seed=4)
    q, cu, qs = make_queries(dt, [3], 2, 64)
    picks = torch.tensor([[[-1, 2, 5, 6, 100000]], [[-1, -1, -1, -1, -5]], [[6, 0, -1, 7, 3]]], dtype=torch.int32, device="cuda")
    ref = block_reference(qs, keys, values, [3], picks.cpu().numpy().tolist(), 32, 0.125)
    assert np.isneginf(ref[1][1]).all()
    compare(*kv.tbn_block_attention(q, pool, index, cu, 3, picks), *ref, tolerance(dt, values))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_later_keys_of_the_own_block_have_no_part(kv, dt, bad):
    """A prompt's later tokens lie in the query's own block: whatever they hold, it is not seen."""
    pool, index, keys, values = make_cache(kv, dt, 1, 64, 32, [60], seed=4)
    p = int(index.table[0, 1])
    pool.k[p, 0, 27, 3], pool.v[p, 0, 9, 27] = bad, bad   # the last token's
    keys[0][59, 0, 3], values[0][59, 0, 9] = bad, bad
    q, cu, qs = make_queries(dt, [5], 2, 64)
    picks = torch.tensor([0, 1], dtype=torch.int32, device="cuda").expand(5, 1, 2).contiguous()
    out, lse = kv.tbn_block_attention(q, pool, index, cu, 5, picks)
    ref, ref_lse = block_reference(qs[:4], [keys[0][:59]], [values[0][:59]], [4], picks[:4].cpu().numpy().tolist(), 32, 0.125)
    compare(out[:4], lse[:4], ref, ref_lse, tolerance(dt, [values[0][:59]]))
    assert bool(torch.isnan(out[4, :, 9]).all()) or math.isinf(bad)


def test_select_ties_infinite_steps_and_odd_queries(kv):
    KV, D, P, blocks = 1, 64, 32, 40
    pool, index, keys, _ = make_cache(kv, "f32", KV, D, P, [blocks * P], seed=4, summary=True)
    q, cu, qs = make_queries("f32", [1], 2, D)
    table = index.table[0].long()

    def got(n, sink=1, recent=1):
        return kv.tbn_block_select(q, pool, index, cu, 1, n, n_sink=sink, n_recent=recent)[0, 0].tolist()

    pool.summary.fill_(3)
    pool.step.fill_(1.0)
    assert got(6) == [0, 1, 2, 3, 4, 39]                       # all equal: the lowest
    pool.step[table[20]] = math.inf
    pool.step[table[30]] = math.inf
    pool.summary[table[20]] = 0
    assert got(6) == [0, 1, 2, 20, 30, 39]
    assert got(3) == [0, 20, 39]
    q[0, 0, 5] = math.nan                                      # counts as 0
    q[0, 1, 7] = -math.inf
    assert got(6) == [0, 1, 2, 20, 30, 39]
    q.zero_()
    assert got(7, 2, 3) == [0, 1, 20, 30, 37, 38, 39]
    pool.step.fill_(1.0)
    assert got(7, 2, 3) == [0, 1, 2, 3, 37, 38, 39]


@pytest.mark.parametrize("blocks,P", [(600, 32), (1700, 64), (17000, 32)])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_select_of_many_blocks(kv, blocks, P, dt):
    """Scores made by many workgroups, in LDS and beyond it; summaries drawn as they are (their keys do not matter here)."""
    KV, D, G = 2, 8, 3
    rng = np.random.RandomState(blocks)
    L = blocks * P - 5
    pool = kv.kv_pool(blocks, KV, D, P, torch.float32 if dt == "f32" else torch.bfloat16, summary=True)
    index = kv.kv_index(1, blocks, blocks, P)
    order = rng.permutation(blocks)
    index.table.copy_(torch.from_numpy(order.astype(np.int32)[None]))
    index.lens.fill_(L)
    hi = rng.randint(-40, 65, (blocks, KV, D))
    codes = np.stack([hi, np.maximum(hi - rng.randint(0, 60, hi.shape), -64)], 2)
    steps = 2.0 ** rng.randint(-6, -3, (blocks, KV))
    pool.summary.copy_(torch.from_numpy(codes.astype(np.int8)))
    pool.step.copy_(torch.from_numpy(steps.astype(np.float32)))
    q, cu, qs = make_queries(dt, [2], KV * G, D)
    for n, sink, recent in ((20, 1, 2), (500, 0, 1), (3, 1, 1)):
        got = kv.tbn_block_select(q, pool, index, cu, 2, n, n_sink=sink, n_recent=recent).cpu().numpy()
        for t in range(2):
            for h in range(KV):
                own = (L - 2 + t) // P
                want = orc.picks(qs[t, h * G:(h + 1) * G], codes[order, h], steps[order, h], own, n, sink, recent)
                assert got[t, h].tolist() == want + [-1] * (n - len(want))


@pytest.mark.parametrize("blocks,P,D,G", [(300, 32, 8, 3), (600, 32, 64, 1), (1500, 64, 128, 4), (3000, 32, 16, 8), (5000, 32, 8, 2), (17000, 32, 8, 3), (400, 128, 256, 12)])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("tokens", [1, 11])
def test_select_by_one_and_by_several(kv, blocks, P, D, G, dt, tokens):
    """One token of each of many blocks, and neighbouring ones that share the records; scores of every sign, ties among them."""
    KV = 2
    rng = np.random.RandomState(blocks + D)
    L = blocks * P - 5
    pool = kv.kv_pool(blocks, KV, D, P, torch.float32 if dt == "f32" else torch.bfloat16, summary=True)
    index = kv.kv_index(1, blocks, blocks, P)
    order = rng.permutation(blocks)
    index.table.copy_(torch.from_numpy(order.astype(np.int32)[None]))
    index.lens.fill_(L)
    hi = rng.randint(-64, 65, (blocks, KV, D))
    codes = np.stack([hi, np.maximum(hi - rng.randint(0, 60, hi.shape), -64)], 2)
    codes[rng.randint(0, blocks, blocks // 8)] = codes[0]
    steps = 2.0 ** rng.randint(-3, 2, (blocks, KV))
    steps[rng.randint(0, blocks, 3)] = math.inf
    pool.summary.copy_(torch.from_numpy(codes.astype(np.int8)))
    pool.step.copy_(torch.from_numpy(steps.astype(np.float32)))
    q, cu, qs = make_queries(dt, [tokens], KV * G, D, stride=KV * G * D + 8)
    for n, sink, recent in ((20, 1, 2), (min(250, blocks - 30), 0, 1), (3, 1, 1), (4, 0, 1)):
        got = kv.tbn_block_select(q, pool, index, cu, tokens, n, n_sink=sink, n_recent=recent).cpu().numpy()
        for t in range(tokens):
            for h in range(KV):
                own = (L - tokens + t) // P
                want = orc.picks(qs[t, h * G:(h + 1) * G], codes[order, h], steps[order, h], own, n, sink, recent)
                assert got[t, h].tolist() == want + [-1] * (n - len(want))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_many_queries_of_a_prompt(kv, dt):
    """More queries than the rule for shared scoring takes, each with blocks of its own."""
    H, KV, D, P = 4, 2, 64, 32
    pool, index, keys, values = make_cache(kv, dt, KV, D, P, [500, 260], seed=11, summary=True)
    set_summary(pool, index, keys, P)
    q, cu, qs = make_queries(dt, [100, 37], H, D)
    picks = kv.tbn_block_select(q, pool, index, cu, 100, 6, n_sink=1, n_recent=2)
    want = oracle_picks(qs, keys, [100, 37], P, 6, 1, 2)
    assert np.array_equal(picks.cpu().numpy(), want)
    out, lse = kv.tbn_block_attention(q, pool, index, cu, 100, picks)
    compare(out, lse, *block_reference(qs, keys, values, [100, 37], want, P, 0.125), tolerance(dt, values))


@pytest.mark.parametrize("H,KV,D,P,seqs,n", [
    (32, 8, 128, 64, [(900, 40), (64, 3), (0, 70), (1, 0)], 5), (8, 8, 64, 128, [(1500, 33), (127, 130)], 4), (20, 4, 80, 64, [(700, 100), (63, 2)], 6),
    (6, 3, 96, 64, [(640, 130)], 3), (64, 4, 128, 64, [(500, 40)], 4), (8, 2, 256, 64, [(800, 300)], 5), (4, 1, 128, 128, [(5000, 300)], 120),
    (32, 8, 128, 32, [(450, 40), (32, 3), (0, 70), (1, 0)], 5), (8, 8, 64, 32, [(370, 33), (31, 130)], 7), (20, 4, 80, 32, [(350, 100), (31, 2)], 6),
    (6, 3, 96, 32, [(320, 130)], 3), (4, 2, 256, 32, [(1000, 200)], 21), (8, 2, 136, 32, [(90, 140)], 4)])
def test_queries_that_share_a_workgroup(kv, H, KV, D, P, seqs, n):
    """Neighbouring queries go through the union of their picks: any picks, some of them outside, none at all."""
    rng = np.random.RandomState(n + D)
    counts = [c for _, c in seqs]
    pool, index, keys, values = make_cache(kv, "bf16", KV, D, P, [p + c for p, c in seqs], seed=D, extra_pages=4)
    q, cu, qs = make_queries("bf16", counts, H, D, stride=H * D + 8)
    picks = np.full((sum(counts), KV, n), -1, np.int32)
    at = 0
    for p, c in seqs:
        for t in range(c):
            blocks = (p + t) // P + 1
            for h in range(KV):
                m = rng.randint(0, min(n, blocks + 2) + 1)
                picks[at, h, :m] = np.sort(rng.permutation(blocks + 2)[:m])   # the last two lie behind the query's own
                if rng.rand() < 0.8 and m:
                    picks[at, h, m - 1] = blocks - 1 if blocks - 1 not in picks[at, h, :m] else picks[at, h, m - 1]
            at += 1
    out, lse = kv.tbn_block_attention(q, pool, index, cu, max(counts), torch.from_numpy(picks).cuda())
    ref = block_reference(qs, keys, values, counts, picks, P, 1 / math.sqrt(D))
    compare(out, lse, *ref, tolerance("bf16", values))


@pytest.mark.parametrize("P", [64, 32])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_queries_that_share_a_workgroup_keep_odd_values_apart(kv, bad, P):
    """A page with such values is seen by the queries that picked it and by no other of the same workgroup."""
    H, KV, D, prefix, n = 32, 8, 128, 400, 70
    pool, index, keys, values = make_cache(kv, "bf16", KV, D, P, [prefix + n], seed=2)
    table = index.table.cpu().numpy()[0]
    for key, d in ((70, 3), (200, 127), (prefix + 20, 64), (prefix + 69, 0)):
        values[0][key, :, d] = bad
        pool.v[int(table[key // P]), :, d, key % P] = bad
    for key, d in ((140, 9),):   # a key of a page that few pick
        keys[0][key, :, d] = bad
        pool.k[int(table[key // P]), :, key % P, d] = bad
    q, cu, qs = make_queries("bf16", [n], H, D)
    if math.isinf(bad):
        qs[:, :, 9] = -np.sign(bad) * (np.abs(qs[:, :, 9]) + 0.01)   # -infinity: a weight of 0
        qs = torch.from_numpy(qs).to(q.dtype).double().numpy()
        q.copy_(torch.from_numpy(qs))
    rng = np.random.RandomState(4)
    picks = np.full((n, KV, 4), -1, np.int32)
    for t in range(n):
        for h in range(KV):
            m = rng.randint(1, 5)
            picks[t, h, :m] = np.sort(rng.permutation((prefix + t) // P + 1)[:m])
    ref = block_reference(qs, keys, values, [n], picks, P, 1 / math.sqrt(D))
    assert not np.isfinite(ref[0]).all() and np.isfinite(ref[0]).any()
    compare(*kv.tbn_block_attention(q, pool, index, cu, n, torch.from_numpy(picks).cuda()), *ref, tolerance("bf16", values))


def test_streams_workspaces_and_graphs(kv):
    """The caller's stream, the caller's workspace, the calls of a step in a graph that is replayed with other queries."""
    H, KV, D, P = 8, 2, 64, 32
    pool, index, keys, values = make_cache(kv, "bf16", KV, D, P, [3000, 900], seed=12, summary=True)
    set_summary(pool, index, keys, P)
    q, cu, _ = make_queries("bf16", [1, 1], H, D)
    out, lse, picks = torch.empty_like(q), torch.empty(2, H, device="cuda"), torch.empty(2, KV, 8, dtype=torch.int32, device="cuda")
    need = max(kv.tbn_tree_attention_workspace_bytes(q, pool, index, 1), kv.tbn_block_select_workspace_bytes(q, pool, index, 1),
               kv.tbn_block_attention_workspace_bytes(q, pool, index, 1, 8))
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    out2, lse2 = torch.empty_like(q), torch.empty_like(lse)

    def step():
        kv.tbn_tree_attention(q, pool, index, cu, 1, out=out, lse=lse, workspace=ws)
        kv.tbn_block_select(q, pool, index, cu, 1, 8, picks=picks, workspace=ws)
        kv.tbn_block_attention(q, pool, index, cu, 1, picks, out=out2, lse=lse2, workspace=ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        q.copy_(make_queries("bf16", [1, 1], H, D, seed=20 + i)[0])
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (out, lse, picks, out2, lse2)]
        want = kv.tbn_tree_attention(q, pool, index, cu, 1) + (kv.tbn_block_select(q, pool, index, cu, 1, 8),)
        want += kv.tbn_block_attention(q, pool, index, cu, 1, want[2])
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
