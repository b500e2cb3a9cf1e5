"""Performance cases of the paged key/value cache and of the attention that reads it.

A case is a dict of plain values; its "op" names the path:

* ``tree``   -- ``tbn_tree_attention``: the drafted tokens of each sequence attend to its cached keys and, by a bit mask,
  to each other; one token per sequence is ordinary decoding;
* ``sparse`` -- ``tbn_block_select`` and ``tbn_block_attention``: each query picks cache pages by their scores, then
  attends to those;
* ``fork``   -- sequences are forked, every one grows by a token: ``tbn_kv_fork``, ``tbn_kv_reserve``,
  ``tbn_kv_copy_pages`` (the shared last pages), ``tbn_kv_append``;
* ``prompt`` -- prompts enter the cache: ``tbn_kv_reserve``, ``tbn_kv_append``;
* ``accept`` -- drafted tokens enter the cache and the accepted path of each tree stays: ``tbn_kv_reserve``,
  ``tbn_kv_append``, ``tbn_kv_keep``, ``tbn_kv_release``;
* ``compact`` -- some sequences end and the pages that are left move to the lowest places: ``tbn_kv_release``,
  ``tbn_kv_compact``, ``tbn_kv_copy_pages``.

Head layouts are 4096 = 32 x 128 with 8 key heads (the transformer layers of the benchmark) and 384 = 6 x 64 (the small
vision transformer), others are drawn.  Keys have a direction per channel and one per page, as trained ones do, and
queries are a little larger than one, so that the weights of a row are neither flat nor all on one key.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

_DT = {"f32": torch.float32, "bf16": torch.bfloat16}
_ESZ = {"f32": 4, "bf16": 2}


def listed():
    return [
        # one user, one token, a short history: latency and launches
        dict(name="tree_one_token", op="tree", dt="bf16", B=1, T=1, ctx=513, H=32, KV=8, D=128, P=64, tree=False, rag=1),
        # a full decode batch over long, ragged histories
        dict(name="tree_decode_batch", op="tree", dt="bf16", B=64, T=1, ctx=16384, H=32, KV=8, D=128, P=64, tree=False, rag=2),
        # speculative decoding: trees of up to 26 drafted tokens
        dict(name="tree_drafts", op="tree", dt="bf16", B=16, T=26, ctx=4100, H=32, KV=8, D=128, P=64, tree=True, rag=3),
        # one long document and the largest tree
        dict(name="tree_long_document", op="tree", dt="bf16", B=1, T=64, ctx=131000, H=32, KV=8, D=128, P=128, tree=True, rag=4),
        # float32, a key head for each query head, an odd number of everything
        dict(name="tree_drafts_f32", op="tree", dt="f32", B=7, T=13, ctx=1009, H=6, KV=6, D=64, P=32, tree=True, rag=5),
        # one token over a long document, 64 of about 2048 pages
        dict(name="sparse_one_token", op="sparse", dt="bf16", B=1, T=1, ctx=131000, H=32, KV=8, D=128, P=64, n=64, sink=1, recent=2, rag=6),
        # a decode batch, float32
        dict(name="sparse_batch_f32", op="sparse", dt="f32", B=24, T=1, ctx=9000, H=12, KV=6, D=64, P=32, n=24, sink=1, recent=1, rag=7),
        # a chunk of a prompt: 512 queries that each pick 24 pages
        dict(name="sparse_prompt_chunk", op="sparse", dt="bf16", B=1, T=512, ctx=16000, H=32, KV=8, D=128, P=64, n=24, sink=1, recent=2, rag=8),
        # parallel sampling: four prompts forked eight times each, every branch writes its first token
        dict(name="pages_fork", op="fork", dt="bf16", B=4, kids=8, ctx=1000, KV=8, D=128, P=64, summary=True, rag=9),
        # eight prompts enter the cache
        dict(name="pages_prompt", op="prompt", dt="bf16", B=8, T=4096, ctx=700, KV=8, D=128, P=64, summary=True, rag=10),
        # the accepted path of each drafted tree stays, the rest is freed
        dict(name="pages_accept", op="accept", dt="f32", B=48, T=26, ctx=900, KV=6, D=64, P=32, summary=True, rag=11),
        # about a third of the sequences end, the others' pages move down
        dict(name="pages_compact", op="compact", dt="bf16", B=96, ctx=3000, KV=8, D=128, P=64, summary=True, rag=12),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _heads(rng):
    KV = rng.choice([1, 2, 4, 6, 8])
    G = rng.choice([1, 2, 4, 4, 5, 8])
    return dict(H=KV * G, KV=KV, D=rng.choice([64, 64, 80, 128, 128, 128, 256]), P=rng.choice([32, 64, 64, 128]))


def draw(rng):
    while True:
        op = rng.choice(["tree", "tree", "tree", "sparse", "sparse", "fork", "prompt", "accept", "compact"])
        dt = rng.choice(["bf16", "bf16", "f32"])
        c = dict(op=op, dt=dt, rag=rng.randrange(1 << 30), **_heads(rng))
        if op == "tree":
            T = rng.choice([1, 1, _log_int(rng, 2, 64)])
            c.update(B=_log_int(rng, 1, 64), T=T, ctx=_log_int(rng, 1, 131000), tree=T > 1 and rng.random() < 0.75)
        elif op == "sparse":
            sink, recent = rng.choice([0, 1, 2]), rng.choice([1, 1, 2, 4])
            T = rng.choice([1, 1, _log_int(rng, 2, 512)])
            c.update(B=_log_int(rng, 1, 32), T=T, ctx=_log_int(rng, 64, 131000), n=sink + recent + _log_int(rng, 1, 64), sink=sink, recent=recent)
        else:
            del c["H"]
            c.update(B=_log_int(rng, 1, 96), ctx=_log_int(rng, 1, 4000), summary=rng.random() < 0.7)
            if op == "fork":
                c.update(kids=rng.randrange(1, 9))
            elif op == "prompt":
                c.update(T=_log_int(rng, 1, 4096))
            elif op == "accept":
                c.update(T=_log_int(rng, 2, 64))
        if _fits(c):
            return c


def _fits(c):
    """No more than the largest listed cases, in bytes, operations and in what the plain form keeps."""
    esz, keys, w = _ESZ[c["dt"]], c["B"] * (c["ctx"] + c.get("T", 1)), work(c)
    if w["bytes"] > 1.3e9 or w["flops"] > 2.5e11 or 2 * keys * c["KV"] * c["D"] * esz > 3.5e9:
        return False
    if c["op"] == "tree":
        return keys * c["H"] * c["T"] <= 3e8
    if c["op"] == "sparse":   # gathered pages, and scores of all blocks
        return c["B"] * c["T"] * c["KV"] * (c["n"] * c["P"] * c["D"] + c["ctx"] / c["P"] * 8) <= 9e8
    return 2 * keys * c["KV"] * c["D"] * esz <= 1.2e9


# ---- sizes of a case's sequences (from the case alone) -------------------------------------------------------------


def _ragged(case, most, salt):
    """Lengths between a quarter of `most` and `most` (the first one has it)."""
    rng = np.random.RandomState((case["rag"] * 7 + salt) % (1 << 31))
    n = case["B"]
    v = rng.randint((most + 3) // 4, most + 1, n)
    v[0] = most
    return v.astype(np.int64)


def _sizes(case):
    """Cached keys before the call and tokens of the call, for each sequence."""
    before = _ragged(case, case["ctx"], 1)
    t = case.get("T", 1)
    new = _ragged(case, t, 2) if t > 1 else np.ones(case["B"], np.int64)
    return before, new


def _pages(keys, P):
    return -(-np.asarray(keys) // P)


def work(case):
    esz, KV, D, P = _ESZ[case["dt"]], case["KV"], case["D"], case["P"]
    before, new = _sizes(case)
    row = 2 * KV * D * esz   # one key and its value, all heads
    if case["op"] == "tree":
        H = case["H"]
        return {"bytes": float((before + new).sum() * row + new.sum() * H * (2 * D * esz + 4)),
                "flops": float(4 * H * D * (new * (before + (new + 1) / 2)).sum())}
    if case["op"] == "sparse":
        H, n = case["H"], case["n"]
        total = before + new
        picked = np.minimum(n, _pages(total, P))
        pages = np.minimum(picked * new, _pages(total, P))   # every page at most once
        b = (pages * P * row + _pages(total, P) * KV * (2 * D + 4)).sum() + new.sum() * (H * (2 * D * esz + 4) + KV * n * 4)
        return {"bytes": float(b), "flops": float((4 * H * D * new * np.minimum(picked * P, total) + 4 * KV * D * new * _pages(total, P)).sum())}
    if case["op"] == "fork":
        kids = case["B"] * case["kids"]
        partial = (before % P != 0).sum() * case["kids"]
        return {"bytes": float(2 * partial * P * row + 2 * (kids + case["B"]) * row + 8 * kids * _pages(before, P).mean()), "flops": float(kids)}
    if case["op"] == "prompt":
        return {"bytes": float(2 * new.sum() * row), "flops": float(new.sum())}
    if case["op"] == "accept":
        return {"bytes": float(4 * new.sum() * row), "flops": float(new.sum())}
    table, lens, refs, _, ends = _tables(case)
    live = np.zeros(len(refs), bool)
    for s in range(case["B"]):
        if not ends[s]:
            live[table[s, :_pages(lens[s], P)]] = True
    moved = int(live[live.sum():].sum())
    return {"bytes": float(2 * moved * P * row + 8 * len(refs) + 4 * table.size), "flops": float(len(refs))}


# ---- inputs ----------------------------------------------------------------------------------------------------------


def _tables(case):
    """Page tables as a server has them: every sequence's pages anywhere in the pool, an eighth of it free."""
    B, P, op = case["B"], case["P"], case["op"]
    before, new = _sizes(case)
    lens = before + new if op in ("tree", "sparse") else before.copy()
    if op == "prompt" and B > 1:
        lens[B // 2] = 0   # one sequence has no history
    rows = B * (1 + case.get("kids", 0))
    most = before + (0 if op == "compact" else new)
    need = _pages(lens, P)
    spare = rows + int(_pages(new, P).sum()) + B   # what reserve takes
    n_pages = int(need.sum() + spare + need.sum() // 8)
    width = int(_pages(most, P).max()) + 1
    rng = np.random.RandomState((case["rag"] * 13 + 5) % (1 << 31))
    order = rng.permutation(n_pages)
    table = np.full((rows, width), -1, np.int32)
    refs = np.zeros(n_pages, np.int32)
    at = 0
    for s in range(B):
        table[s, :need[s]] = order[at:at + need[s]]
        at += need[s]
    refs[order[:at]] = 1
    full = np.zeros(rows, np.int64)
    full[:B] = lens
    ends = rng.rand(B) < 0.36
    ends[0] = False
    return table, full, refs, new, ends


def _values(case, seed, n_pages):
    """Pool tensors: keys with a direction per channel and per page, values N(0, 1)."""
    dt, KV, D, P = _DT[case["dt"]], case["KV"], case["D"], case["P"]
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    k = torch.randn(n_pages, KV, P, D, generator=g, device="cuda", dtype=dt)
    k += torch.randn(KV, 1, D, generator=g, device="cuda", dtype=dt)
    k += torch.randn(n_pages, KV, 1, D, generator=g, device="cuda", dtype=dt) * 0.5
    v = torch.randn(n_pages, KV, D, P, generator=g, device="cuda", dtype=dt)
    return k, v, g


def _pow2(e):
    """2 to the power of whole numbers -126 .. 127, exactly."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _codes_of(lo, hi):
    """Summary of pages from the least and the largest key per channel: codes (.., 2, D) and the step (..)."""
    a = torch.maximum(hi.abs(), lo.abs()).amax(-1)
    bad = ~torch.isfinite(a)
    x = torch.frexp(torch.where(bad, torch.zeros_like(a), a)).exponent.clamp(min=-100)
    x = torch.where(a == 0, torch.full_like(x, -100), x)
    up = _pow2(6 - x).unsqueeze(-1)
    codes = torch.stack([torch.ceil(hi * up), torch.floor(lo * up)], -2)
    codes = torch.where(bad[..., None, None], torch.zeros_like(codes), codes).to(torch.int8)
    step = torch.where(bad, torch.full_like(a, math.inf), _pow2(x - 6))
    return codes, step


def prepare(case, seed):
    dt, KV, D, P, B, op = _DT[case["dt"]], case["KV"], case["D"], case["P"], case["B"], case["op"]
    table, lens, refs, new, ends = _tables(case)
    k, v, g = _values(case, seed, len(refs))
    # one buffer for all bookkeeping, so that a pass can put it back with one copy
    meta0 = torch.from_numpy(np.concatenate([table.ravel(), lens.astype(np.int32), refs, np.zeros(1, np.int32)])).cuda()
    meta = meta0.clone()
    a, b, c = table.size, table.size + len(lens), table.size + len(lens) + len(refs)
    s = dict(case, k=k, v=v, meta=meta, meta0=meta0, table=meta[:a].view(table.shape), lens=meta[a:b], refs=meta[b:c], status=meta[c:])
    s["summary"] = s["step"] = None
    if op == "sparse" or case.get("summary"):
        s["summary"], s["step"] = torch.empty(len(refs), KV, 2, D, dtype=torch.int8, device="cuda"), torch.empty(len(refs), KV, device="cuda")
        for i in range(0, len(refs), 4096):
            f = k[i:i + 4096].float()
            s["summary"][i:i + 4096], s["step"][i:i + 4096] = _codes_of(f.amin(2), f.amax(2))
            del f
    ints = lambda x: torch.from_numpy(np.ascontiguousarray(x, np.int32)).cuda()  # noqa: E731
    if op == "fork":
        s["parents"] = ints(np.repeat(np.arange(B), case["kids"]))
        s["children"] = ints(np.arange(B, B * (1 + case["kids"])))
        new = np.ones(len(lens), np.int64)
    s["max_len"], s["max_new"], s["total"] = int(lens.max()), int(new.max()), int(new.sum())
    s["cu"] = ints(np.concatenate([[0], np.cumsum(new)]))
    s["new"] = ints(new)
    N = s["total"]
    if op in ("tree", "sparse"):
        # the query part of a fused projection's output: rows are further apart than H * D
        H = case["H"]
        s["qkv"] = torch.randn(N, (H + 2 * KV) * D, generator=g, device="cuda", dtype=dt) * 1.5
        s["q"] = s["qkv"][:, :H * D].unflatten(1, (H, D))
        s["scale"] = 1.0 / math.sqrt(D)
    elif op != "compact":
        s["kvnew"] = torch.randn(N, 2 * KV * D, generator=g, device="cuda", dtype=dt)
        s["k_new"], s["v_new"] = s["kvnew"][:, :KV * D].unflatten(1, (KV, D)), s["kvnew"][:, KV * D:].unflatten(1, (KV, D))
    if op == "tree":
        s["mask"] = None
        if case["tree"]:   # each drafted token hangs on an earlier one or on the last cached one
            T = s["max_new"]
            words = -(-T // 32)
            rng = np.random.RandomState(seed % (1 << 31))
            see = np.zeros((B, T, words * 32), np.uint8)
            for i in range(T):
                parent = rng.randint(-1, i, B) if i else np.full(B, -1)
                see[:, i] = np.where(parent[:, None] >= 0, see[np.arange(B), np.maximum(parent, 0)], 0)
                see[:, i, i] = 1
            rows = np.concatenate([see[b, :new[b]] for b in range(B)])
            s["mask"] = torch.from_numpy(np.packbits(rows, axis=1, bitorder="little").view(np.int32).copy()).cuda()
    if op == "accept":   # the accepted path of each tree: some of the drafted tokens, in order
        rng = np.random.RandomState(seed % (1 << 31))
        counts = np.array([rng.randint(1, n + 1) for n in new])
        picks = np.zeros((B, s["max_new"]), np.int32)
        for b in range(B):
            picks[b, :counts[b]] = np.sort(rng.permutation(int(new[b]))[:counts[b]])
        s["base"], s["picks"], s["counts"], s["left"] = ints(lens), ints(picks), ints(counts), ints(lens + counts)
    if op == "compact":
        s["left"] = ints(np.where(ends, 0, lens))
    if op in ("tree", "sparse"):
        del s["meta"], s["meta0"]
    return s


def run(s):
    if own:
        return _run_own(s)
    return {"tree": _plain_tree, "sparse": _plain_sparse, "fork": _plain_fork, "prompt": _plain_prompt, "accept": _plain_accept,
            "compact": _plain_compact}[s["op"]](s)


def _run_own(s):
    from paper_2407_12075_amd import kv
    op = s["op"]
    if "pool" not in s:   # the handles that a program keeps with its cache
        s["pool"], s["index"] = kv.KVPool(s["k"], s["v"], s["summary"], s["step"]), kv.KVIndex(s["table"], s["lens"], s["refs"], s["status"], s["P"])
    pool, index = s["pool"], s["index"]
    if op == "tree":
        return kv.tbn_tree_attention(s["q"], pool, index, s["cu"], s["max_new"], mask=s["mask"], scale=s["scale"], max_len=s["max_len"])
    if op == "sparse":
        picks = kv.tbn_block_select(s["q"], pool, index, s["cu"], s["max_new"], s["n"], n_sink=s["sink"], n_recent=s["recent"], max_len=s["max_len"])
        out, lse = kv.tbn_block_attention(s["q"], pool, index, s["cu"], s["max_new"], picks, scale=s["scale"])
        return picks, out, lse
    s["meta"].copy_(s["meta0"])   # the bookkeeping of the pass's start, so that every pass does the same
    if op == "compact":
        kv.tbn_kv_release(index, s["left"])
        src, dst, count = kv.tbn_kv_compact(index)
        kv.tbn_kv_copy_pages(pool, src, dst, count)
        return _cache(s)
    if op == "fork":
        kv.tbn_kv_fork(index, s["parents"], s["children"])
    src, dst = kv.tbn_kv_reserve(index, s["new"])
    if op == "fork":
        kv.tbn_kv_copy_pages(pool, src, dst)
    kv.tbn_kv_append(pool, index, s["k_new"], s["v_new"], s["cu"], s["max_new"])
    if op == "accept":
        kv.tbn_kv_keep(pool, index, s["base"], s["picks"], s["counts"])
        kv.tbn_kv_release(index, s["left"])
    return _cache(s)


def _cache(s):
    return [t for t in (s["table"], s["lens"], s["refs"], s["status"], s["k"], s["v"], s["summary"], s["step"]) if t is not None]


# ---- the plain forms -------------------------------------------------------------------------------------------------


def _rows(s):
    """For the call's tokens: sequence, place within its tokens; and the padded (B, T) indices of the tokens."""
    cu, dev = s["cu"].long(), s["cu"].device
    i = torch.arange(s["total"], device=dev)
    seq = (i[:, None] >= cu[None, 1:]).sum(1)
    padded = (cu[:-1, None] + torch.arange(s["max_new"], device=dev)).clamp(max=s["total"] - 1)
    return seq, i - cu[seq], padded


def _plain_tree(s):
    KV, D, P, H, T = s["KV"], s["D"], s["P"], s["H"], s["max_new"]
    G, B, np_ = H // KV, s["B"], -(-s["max_len"] // P)
    seq, place, padded = _rows(s)
    pages = s["table"][:, :np_].long().clamp(min=0)
    k = s["k"][pages].float().permute(0, 2, 1, 3, 4).reshape(B * KV, np_ * P, D)
    v = s["v"][pages].float().permute(0, 2, 1, 4, 3).reshape(B * KV, np_ * P, D)
    q = s["q"].float()[padded].view(B, T, KV, G, D).permute(0, 2, 3, 1, 4).reshape(B * KV, G * T, D)
    a = (torch.bmm(q, k.transpose(1, 2).contiguous()) * s["scale"]).view(B, KV * G, T, np_ * P)
    lens, new = s["lens"].long(), s["new"].long()
    at = torch.arange(np_ * P, device=a.device)
    draft = at[None] - (lens - new)[:, None]   # place among the drafted keys, negative for the others
    if s["mask"] is None:
        see = draft[:, None, :] <= torch.arange(T, device=a.device)[None, :, None]
    else:
        words = s["mask"][padded]   # (B, T, words)
        j = draft.clamp(0, words.shape[2] * 32 - 1)
        word = torch.gather(words, 2, (j // 32)[:, None, :].expand(B, T, -1))
        see = ((word >> (j % 32).int()[:, None, :]) & 1 == 1) | (draft < 0)[:, None, :]
    see = (see & (at[None] < lens[:, None])[:, None, :])[:, None]
    a = torch.where(see, a, torch.full_like(a, -math.inf))
    o, lse = _weighted(a.view(B * KV, G * T, np_ * P), v)
    o = o.view(B, H, T, D).permute(0, 2, 1, 3)[seq, place]
    return o.to(s["q"].dtype), lse.view(B, H, T).permute(0, 2, 1)[seq, place]


def _weighted(a, v):
    """Softmax over the last axis of `a`, times v; a row that sees nothing gives zeros."""
    m = a.amax(-1, keepdim=True)
    m = torch.where(torch.isinf(m), torch.zeros_like(m), m)
    p = torch.exp(a - m)
    z = p.sum(-1, keepdim=True)
    o = torch.bmm(p, v) / torch.where(z == 0, torch.ones_like(z), z)
    return o, (m + torch.log(z)).squeeze(-1)


def _plain_sparse(s):
    KV, D, P, H, T, n = s["KV"], s["D"], s["P"], s["H"], s["max_new"], s["n"]
    G, B, nb = H // KV, s["B"], -(-s["max_len"] // P)
    seq, place, padded = _rows(s)
    N, dev = s["total"], s["k"].device
    q = s["q"].float().view(N, KV, G, D)
    # pooled queries: whole numbers on a power-of-two grid per group of heads
    a = q.abs().amax((2, 3))
    x = torch.frexp(a).exponent.clamp(min=-100)
    codes = torch.round(q * _pow2(6 - x)[:, :, None, None])
    pooled = torch.cat([codes.clamp(min=0).sum(2), codes.clamp(max=0).sum(2)], -1)   # (N, KV, 2 D)
    pages = s["table"][:, :nb].long().clamp(min=0)
    sums = s["summary"][pages].float().view(B, nb, KV, 2 * D).permute(0, 2, 3, 1).reshape(B * KV, 2 * D, nb)
    whole = torch.bmm(pooled[padded].permute(0, 2, 1, 3).reshape(B * KV, T, 2 * D), sums).view(B, KV, T, nb)
    step = s["step"][pages].permute(0, 2, 1)[:, :, None, :]
    score = torch.where(torch.isinf(step), step, whole * step).permute(0, 2, 1, 3)[seq, place]   # (N, KV, nb)
    # the first and the last blocks up to the query's own always, of the others the highest scores
    where = (s["lens"].long() - s["new"].long())[seq] + place
    last = where // P
    b = torch.arange(nb, device=dev)
    always = (b[None] < s["sink"]) | (b[None] > (last - s["recent"])[:, None])
    tier = torch.where(b[None] <= last[:, None], 1 + always.long(), torch.zeros_like(b[None]))[:, None].expand(N, KV, nb)
    by_score = torch.sort(score, dim=-1, descending=True, stable=True).indices
    by_tier = torch.sort(torch.gather(tier, 2, by_score), dim=-1, descending=True, stable=True)
    picks = torch.gather(by_score, 2, by_tier.indices)[..., :n]
    picks = torch.where(by_tier.values[..., :n] > 0, picks, torch.full_like(picks, nb))
    picks = torch.sort(picks, dim=-1).values
    picks = torch.where(picks < nb, picks, torch.full_like(picks, -1))
    if picks.shape[2] < n:
        picks = torch.cat([picks, picks.new_full((N, KV, n - picks.shape[2]), -1)], 2)
    # the picked pages
    page = s["table"][seq[:, None, None], picks.clamp(min=0)].long().clamp(min=0)
    head = torch.arange(KV, device=dev)[None, :, None]
    k = s["k"][page, head].float().view(N * KV, n * P, D)
    v = s["v"][page, head].float().transpose(3, 4).reshape(N * KV, n * P, D)
    at = (picks * P)[..., None] + torch.arange(P, device=dev)
    see = ((picks >= 0)[..., None] & (at <= where[:, None, None, None])).view(N * KV, 1, n * P)
    a = torch.bmm(q.reshape(N * KV, G, D), k.transpose(1, 2).contiguous()) * s["scale"]
    o, lse = _weighted(torch.where(see, a, torch.full_like(a, -math.inf)), v)
    return picks.int(), o.view(N, H, D).to(s["q"].dtype), lse.view(N, H)


def _plain_reserve(s):
    """Pages for the new tokens: fresh ones in the order of sequences, a shared last page is left for a copy."""
    P, dev = s["P"], s["k"].device
    lens, new, refs = s["lens"].long(), s["new"].long(), s["refs"]
    have, want = (lens + P - 1) // P, (lens + new + P - 1) // P
    rows = torch.arange(len(lens), device=dev)
    partial = (lens % P != 0) & (new > 0)
    tail = s["table"][rows, (lens // P).clamp(max=s["table"].shape[1] - 1)].long().clamp(min=0)
    earlier = (torch.tril(tail[:, None] == tail[None], -1) & partial[None]).sum(1)
    copy = partial & (refs[tail] - earlier > 1)
    first = have - copy.long()
    need = torch.where(new > 0, want - first, torch.zeros_like(want))
    offset = torch.cumsum(need, 0) - need
    free = torch.nonzero(refs == 0).squeeze(1)
    slot = torch.arange(s["table"].shape[1], device=dev)[None]
    fresh = (slot >= first[:, None]) & (slot < want[:, None]) & (new > 0)[:, None]
    pages = free[(offset[:, None] + slot - first[:, None]).clamp(0, len(free) - 1)]
    s["table"].copy_(torch.where(fresh, pages.int(), s["table"]))
    refs.index_add_(0, tail, -copy.int())
    refs.index_add_(0, pages.flatten(), fresh.flatten().int())
    s["lens"].copy_((lens + new).int())
    none = torch.full_like(tail, -1)
    return torch.where(copy, tail, none), torch.where(copy, s["table"][rows, (lens // P).clamp(max=slot.shape[1] - 1)].long(), none)


def _plain_copy(s, src, dst):
    src, dst = src[src >= 0], dst[src >= 0]
    for name in ("k", "v") + (("summary", "step") if s["summary"] is not None else ()):
        s[name][dst] = s[name][src]


def _plain_append(s):
    P = s["P"]
    seq, place, _ = _rows(s)
    at = (s["lens"].long() - s["new"].long())[seq] + place
    page = s["table"][seq, at // P].long()
    s["k"][page, :, at % P] = s["k_new"]
    s["v"][page, :, :, at % P] = s["v_new"]
    _plain_summary(s, s["lens"].long() - s["new"].long(), s["lens"].long())


def _plain_summary(s, begin, end):
    """Summaries of the pages that hold keys begin .. end - 1, over their keys before `end`."""
    if s["summary"] is None:
        return
    P = s["P"]
    slot = torch.arange(s["table"].shape[1], device=s["k"].device)[None]
    touched = torch.nonzero((slot >= (begin // P)[:, None]) & (slot * P < end[:, None]) & (begin < end)[:, None])
    page = s["table"][touched[:, 0], touched[:, 1]].long()
    filled = end[touched[:, 0]] - touched[:, 1] * P
    f = s["k"][page].float()
    there = (torch.arange(P, device=f.device)[None] < filled[:, None])[:, None, :, None]
    s["summary"][page], s["step"][page] = _codes_of(torch.where(there, f, torch.full_like(f, math.inf)).amin(2),
                                                    torch.where(there, f, torch.full_like(f, -math.inf)).amax(2))


def _plain_release(s, keep):
    P = s["P"]
    lens = s["lens"].long()
    left = torch.minimum(lens, keep.long())
    slot = torch.arange(s["table"].shape[1], device=lens.device)[None]
    gone = (slot >= ((left + P - 1) // P)[:, None]) & (slot < ((lens + P - 1) // P)[:, None])
    s["refs"].index_add_(0, s["table"].long().clamp(min=0).flatten(), -gone.flatten().int())
    s["table"].copy_(torch.where(gone, torch.full_like(s["table"], -1), s["table"]))
    s["lens"].copy_(left.int())


def _plain_fork(s):
    s["meta"].copy_(s["meta0"])
    parents, children = s["parents"].long(), s["children"].long()
    rows = s["table"][parents]
    s["table"][children] = rows
    s["lens"][children] = s["lens"][parents]
    held = torch.arange(rows.shape[1], device=rows.device)[None] < ((s["lens"][parents].long() + s["P"] - 1) // s["P"])[:, None]
    s["refs"].index_add_(0, rows.long().clamp(min=0).flatten(), held.flatten().int())
    _plain_copy(s, *_plain_reserve(s))
    _plain_append(s)
    return _cache(s)


def _plain_prompt(s):
    s["meta"].copy_(s["meta0"])
    _plain_reserve(s)
    _plain_append(s)
    return _cache(s)


def _plain_accept(s):
    s["meta"].copy_(s["meta0"])
    P = s["P"]
    _plain_reserve(s)
    _plain_append(s)
    j = torch.arange(s["picks"].shape[1], device=s["k"].device)[None]
    kept = torch.nonzero(j < s["counts"][:, None])
    seq = kept[:, 0]
    begin = s["base"].long()[seq]
    a, b = begin + s["picks"].long()[seq, kept[:, 1]], begin + kept[:, 1]
    pa, pb = s["table"][seq, a // P].long(), s["table"][seq, b // P].long()
    s["k"][pb, :, b % P] = s["k"][pa, :, a % P]
    s["v"][pb, :, :, b % P] = s["v"][pa, :, :, a % P]
    _plain_summary(s, s["base"].long(), s["base"].long() + s["counts"].long())
    _plain_release(s, s["left"])
    return _cache(s)


def _plain_compact(s):
    s["meta"].copy_(s["meta0"])
    _plain_release(s, s["left"])
    live = s["refs"] > 0
    at = torch.arange(len(live), device=live.device)
    low = at < live.sum()
    src, dst = torch.nonzero(live & ~low).squeeze(1), torch.nonzero(~live & low).squeeze(1)
    to = at.clone()
    to[src] = dst
    s["table"].copy_(torch.where(s["table"] >= 0, to[s["table"].long().clamp(min=0)].int(), s["table"]))
    s["refs"][dst] = s["refs"][src]
    s["refs"][src] = 0
    _plain_copy(s, src, dst)
    return _cache(s)


# ---- 64 bits ---------------------------------------------------------------------------------------------------------


def exact(case, seed):
    """Attention from its definition, sequence by sequence and key head by key head; copies have no rounding."""
    if case["op"] not in ("tree", "sparse"):
        return None
    s = prepare(case, seed)
    KV, D, P, H = s["KV"], s["D"], s["P"], s["H"]
    G = H // KV
    cu, lens = s["cu"].tolist(), s["lens"].tolist()
    table = s["table"].cpu().numpy()
    out = torch.zeros(s["total"], H, D, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["total"], H, dtype=torch.float64, device="cuda")
    picked = torch.full((s["total"], KV, case["n"]), -1, dtype=torch.int64, device="cuda") if case["op"] == "sparse" else None
    for b in range(s["B"]):
        L, t0, t1 = lens[b], cu[b], cu[b + 1]
        T, first = t1 - t0, lens[b] - (t1 - t0)
        pages = torch.from_numpy(table[b, :-(-L // P)].astype(np.int64)).cuda()
        key = torch.arange(L, device="cuda")
        if case["op"] == "tree" and s["mask"] is not None:
            bits = np.unpackbits(s["mask"][t0:t1].cpu().numpy().view(np.uint8), axis=1, bitorder="little")[:, :T]
            see_new = torch.from_numpy(bits.astype(bool)).cuda()
        else:
            see_new = torch.ones(T, T, dtype=torch.bool, device="cuda").tril()
        see = torch.cat([torch.ones(T, first, dtype=torch.bool, device="cuda"), see_new], 1)
        for h in range(KV):
            k = s["k"][pages, h].double().reshape(-1, D)[:L]
            v = s["v"][pages, h].double().transpose(1, 2).reshape(-1, D)[:L]
            q = s["q"][t0:t1, h * G:(h + 1) * G].double()
            seen = see
            if picked is not None:
                member = _exact_picks(case, q, k, torch.arange(first, L, device="cuda") // P)
                seen = see & member[:, key // P]
                for t in range(T):
                    blocks = torch.nonzero(member[t]).squeeze(1)
                    picked[t0 + t, h, :len(blocks)] = blocks
            for g in range(G):
                a = (q[:, g] @ k.T) * s["scale"]
                a = a.masked_fill(~seen, -math.inf)
                norm = torch.logsumexp(a, 1)
                lse[t0:t1, h * G + g] = norm
                out[t0:t1, h * G + g] = torch.exp(a - norm[:, None]) @ v
    return (out, lse) if picked is None else (picked, out, lse)


def _exact_picks(case, q, k, own_block):
    """Which blocks each query picks, (T, blocks): a block is in if fewer than the picks that are left go before it."""
    P, n = case["P"], case["n"]
    T, L = q.shape[0], k.shape[0]
    nb = -(-L // P)
    score = torch.zeros(T, nb, dtype=torch.float64, device=q.device)
    xq = torch.floor(torch.log2(q.abs().amax((1, 2)))) + 1
    c = torch.round(q * torch.exp2(6 - xq)[:, None, None])
    for b in range(L // P):   # a block that is not full is some query's last one or behind it
        kb = k[b * P:(b + 1) * P]
        grid = torch.exp2(torch.floor(torch.log2(kb.abs().max())) + 1 - 6)
        top, low = torch.ceil(kb.amax(0) / grid), torch.floor(kb.amin(0) / grid)
        score[:, b] = (c.clamp(min=0) @ top + c.clamp(max=0) @ low).sum(1) * grid
    at = torch.arange(nb, device=q.device)
    there = at[None] <= own_block[:, None]
    always = ((at[None] < case["sink"]) | (at[None] > (own_block - case["recent"])[:, None])) & there
    rest = there & ~always
    left = n - always.sum(1)
    ahead = torch.zeros(T, nb, dtype=torch.int64, device=q.device)
    for b in range(nb):
        before = (score > score[:, b:b + 1]) | ((score == score[:, b:b + 1]) & (at < b)[None])
        ahead[:, b] = (before & rest).sum(1)
    return always | (rest & (ahead < left[:, None]))
