"""Performance cases of attention with a sliding window, of a cache held in 4 bits and of the verification of drafted tokens.

A case is a dict of plain values; its "op" names the path:

* ``window`` -- ``tbn_window_attention``: attention over the paged cache (float32 or bfloat16) where a token sees the sequence's
  first keys and the last ones before it; one token per sequence, chunks of prompts, trees of drafted tokens;
* ``kv4``    -- ``tbn_kv4_attention``: attention over a cache of 4-bit keys and values, all keys (window 0) or a window of them;
* ``store``  -- ``tbn_kv4_append`` and ``tbn_kv4_read``: new keys and values enter the 4-bit cache; what they have become there is
  read back;
* ``verify`` -- ``tbn_verify``: drafted tokens are accepted or not by the target's probabilities, the draft's and given random
  numbers, and the token that follows is drawn.

Head layouts are 4096 = 32 x 128 with 8 key heads (the transformer layers of the benchmark) and 384 = 6 x 64 (the small vision
transformer), others are drawn.  Keys have a direction per channel and per page, as trained ones do; target and draft agree on
most tokens, as a draft model's do.

A 4-bit cache: a group is 32 neighbouring channels of one key (or value) of one head.  With a its largest magnitude, x is the
smallest whole number, -100 .. 125, with a <= 6 * 2^x (125 if there is none), and each element becomes the nearest of
0, 0.5, 1, 1.5, 2, 3, 4, 6 times 2^x with its sign (ties go to the code that is even: 0, 1, 2, 4).
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
        # one user's next token, a window of half a thousand keys: latency and launches
        dict(name="window_one_token", op="window", dt="bf16", B=1, T=1, ctx=2000, H=32, KV=8, D=128, P=64, sink=4, window=512, tree=False, rag=1),
        # a full decode batch over long histories, of which the last 4096 keys count
        dict(name="window_decode_batch", op="window", dt="bf16", B=64, T=1, ctx=16384, H=32, KV=8, D=128, P=64, sink=4, window=4096, tree=False, rag=2),
        # prompts in chunks of up to 2048 tokens
        dict(name="window_prompt_chunk", op="window", dt="bf16", B=2, T=2048, ctx=6000, H=32, KV=8, D=128, P=64, sink=4, window=1024, tree=False, rag=3),
        # trees of drafted tokens, float32, a key head for each query head, odd sizes
        dict(name="window_drafts_f32", op="window", dt="f32", B=7, T=13, ctx=1009, H=6, KV=6, D=64, P=32, sink=5, window=301, tree=True, rag=4),
        # one user's next token over a short 4-bit history
        dict(name="kv4_one_token", op="kv4", dt="bf16", B=1, T=1, ctx=513, H=32, KV=8, D=128, P=64, sink=0, window=0, tree=False, rag=5),
        # a full decode batch over long, ragged histories
        dict(name="kv4_decode_batch", op="kv4", dt="bf16", B=64, T=1, ctx=16384, H=32, KV=8, D=128, P=64, sink=0, window=0, tree=False, rag=6),
        # speculative decoding: trees of up to 26 drafted tokens
        dict(name="kv4_drafts", op="kv4", dt="bf16", B=16, T=26, ctx=4100, H=32, KV=8, D=128, P=64, sink=0, window=0, tree=True, rag=7),
        # a small decode batch, float32 queries, a window over the 4-bit history
        dict(name="kv4_window_f32", op="kv4", dt="f32", B=9, T=1, ctx=15000, H=6, KV=6, D=64, P=32, sink=4, window=5000, tree=False, rag=8),
        # the keys of one decoding step enter the cache
        dict(name="store_step", op="store", dt="bf16", B=64, T=1, ctx=4000, KV=8, D=128, P=64, rag=9),
        # eight prompts enter the cache
        dict(name="store_prompt", op="store", dt="bf16", B=8, T=4096, ctx=700, KV=8, D=128, P=64, rag=10),
        # the decoder's trees: best tokens and runners-up, no probabilities of the draft
        dict(name="verify_small_trees", op="verify", B=8, T=7, V=1024, kids=2, draft=False, rag=11),
        # a batch of chains of five sampled drafts behind the last token, a large vocabulary
        dict(name="verify_chains", op="verify", B=64, T=6, V=131072, kids=1, draft=True, rag=12),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    while True:
        op = rng.choice(["window", "window", "kv4", "kv4", "kv4", "store", "verify"])
        c = dict(op=op, rag=rng.randrange(1 << 30))
        if op == "verify":
            kids = rng.choice([1, 1, 2, 3])
            c.update(B=_log_int(rng, 1, 64), T=_log_int(rng, 2, 48), V=_log_int(rng, 64, 131072), kids=kids, draft=rng.random() < 0.6)
        else:
            KV, G = rng.choice([1, 2, 4, 6, 8]), rng.choice([1, 2, 4, 4, 5, 8])
            D = rng.choice([64, 64, 96, 128, 128, 128, 256]) if op != "window" else rng.choice([64, 64, 80, 128, 128, 128, 256])
            c.update(dt=rng.choice(["bf16", "bf16", "f32"]), KV=KV, D=D, P=rng.choice([32, 64, 64, 128]), B=_log_int(rng, 1, 64))
            if op == "store":
                c.update(T=_log_int(rng, 1, 4096), ctx=_log_int(rng, 1, 4000))
            else:
                T = rng.choice([1, 1, _log_int(rng, 2, 64), _log_int(rng, 2, 1024)])
                tree = 1 < T <= 64 and rng.random() < 0.6
                window = _log_int(rng, 64, 8192) if op == "window" or rng.random() < 0.4 else 0
                c.update(H=KV * G, T=T, ctx=_log_int(rng, 1, 131000), sink=rng.choice([0, 1, 4, 100]) if window else 0, window=window, tree=tree)
        if _fits(c):
            return c


def _fits(c):
    """No more than the largest listed cases, in bytes, operations and in what the plain form keeps."""
    w = work(c)
    if w["bytes"] > 1.3e9 or w["flops"] > 1.5e11:
        return False
    if c["op"] == "verify":
        return c["B"] * c["T"] * c["V"] <= 6e7
    keys = c["B"] * (c["ctx"] + c["T"])
    if keys * c["KV"] * c["D"] > 1.1e9:
        return False
    return c["op"] == "store" or keys * c["H"] * c["T"] <= 1.1e9


# ---- sizes of a case's sequences (from the case alone) ---------------------------------------------------------------------


def _ragged(case, most, salt):
    """Sizes between a quarter of `most` and `most` (the first one has it)."""
    rng = np.random.RandomState((case["rag"] * 7 + salt) % (1 << 31))
    v = rng.randint((most + 3) // 4, most + 1, case["B"])
    v[0] = most
    return v.astype(np.int64)


def _sizes(case):
    """Cached keys before the call and tokens of the call, for each sequence."""
    new = _ragged(case, case["T"], 2) if case["T"] > 1 else np.ones(case["B"], np.int64)
    return _ragged(case, case["ctx"], 1) if "ctx" in case else None, new


def _seen(case):
    """Keys that some token of a sequence sees, and pairs of a token and a key it sees (a tree's tokens: all before them)."""
    before, new = _sizes(case)
    if not case["window"]:
        return before + new, new * before + new * (new + 1) // 2
    s, w = case["sink"], case["window"]
    keys, pairs = np.zeros_like(before), np.zeros_like(before)
    for b in range(case["B"]):
        at = before[b] + np.arange(new[b])
        lo = np.maximum(at - w + 1, 0)
        first = np.minimum(s, lo)
        pairs[b] = (at - lo + 1 + first).sum()
        keys[b] = before[b] + new[b] - lo[0] + first[0]
    return keys, pairs


def work(case):
    before, new = _sizes(case)
    if case["op"] == "verify":
        # the row that is drawn from, the draft's where one was refused, one number for each drafted token
        rows = case["B"] * case["V"]
        return {"bytes": float(rows * 4 * (1.5 if case["draft"] else 1) + new.sum() * 20), "flops": float(rows * 2)}
    esz, KV, D = _ESZ[case["dt"]], case["KV"], case["D"]
    four = 2 * KV * (D / 2 + D / 32)   # bytes of one key and its value, all heads
    if case["op"] == "store":
        return {"bytes": float(new.sum() * (4 * KV * D * esz + 2 * four)), "flops": float(new.sum() * 4 * KV * D)}
    keys, pairs = _seen(case)
    row = four if case["op"] == "kv4" else 2 * KV * D * esz
    return {"bytes": float(keys.sum() * row + new.sum() * case["H"] * (2 * D * esz + 4)), "flops": float(4 * case["H"] * D * pairs.sum())}


# ---- inputs ----------------------------------------------------------------------------------------------------------------


def _ints(x):
    return torch.from_numpy(np.ascontiguousarray(x, np.int32)).cuda()


def _parents(case, new, rng):
    """For each sequence's tokens the place of the one they hang on, -1 for the first: at most `kids` on each."""
    rows = []
    for n in new:
        p, left = [-1], {0: case["kids"]}
        for i in range(1, int(n)):
            at = i - 1 if case["kids"] == 1 else rng.choice(sorted(left))
            left[at] = left.get(at, case["kids"]) - 1
            if left[at] == 0:
                del left[at]
            left[i] = case["kids"]
            p.append(int(at))
        rows.append(p)
    return rows


def _prepare_verify(case, seed):
    B, V = case["B"], case["V"]
    _, new = _sizes(case)
    rng = np.random.RandomState(seed % (1 << 31))
    parents = _parents(case, new, rng)
    N = int(new.sum())
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    logits = torch.randn(N, V, generator=g, device="cuda") * 3.0
    target = torch.softmax(logits, 1)
    logits += torch.randn(N, V, generator=g, device="cuda") * 0.7
    draft = torch.softmax(logits, 1)
    cu = np.concatenate([[0], np.cumsum(new)])
    above = torch.from_numpy(np.concatenate([np.maximum(p, 0) + a for p, a in zip(parents, cu)])).cuda()   # each token's parent's row
    if case["draft"]:   # drawn from the draft's probabilities
        noise = torch.rand(N, V, generator=g, device="cuda").clamp_(min=1e-30).log_().neg_()
        tokens = (draft[above] / noise).argmax(1)
    else:               # the best tokens and the runners-up
        nth, seen = np.zeros(N, np.int64), {}
        for i, a in enumerate(above.tolist()):
            if i not in set(cu[:-1].tolist()):
                nth[i] = seen.get(a, 0)
                seen[a] = nth[i] + 1
        best = draft.topk(int(nth.max()) + 1, 1).indices
        tokens = best[above, torch.from_numpy(nth).cuda()]
    return dict(case, target=target, draft_p=draft if case["draft"] else None, tokens=tokens.int(), u=torch.rand(N, generator=g, device="cuda"),
                parents=None if case["kids"] == 1 else _ints(np.concatenate(parents)), cu=_ints(cu), total=N, max_new=int(new.max()))


def _tables(case):
    """Page tables as a server has them: every sequence's pages anywhere in the pool, an eighth of it free."""
    B, P = case["B"], case["P"]
    before, new = _sizes(case)
    lens = before + new
    need = -(-lens // P)
    n_pages = int(need.sum() + need.sum() // 8 + 1)
    rng = np.random.RandomState((case["rag"] * 13 + 5) % (1 << 31))
    order = rng.permutation(n_pages)
    table, refs, at = np.full((B, int(need.max()) + 1), -1, np.int32), np.zeros(n_pages, np.int32), 0
    for s in range(B):
        table[s, :need[s]] = order[at:at + need[s]]
        at += need[s]
    refs[order[:at]] = 1
    return table, lens, refs, new


def _nibbles(x):
    """Codes and exponents (int32) of groups of 32 along the last axis."""
    f = x.float().unflatten(-1, (-1, 32))
    a = f.abs().amax(-1)
    m, e = torch.frexp(a)
    e = torch.where(a == 0, torch.full_like(e, -100), e - 3 + (m > 0.75).int()).clamp(-100, 125)
    y = torch.ldexp(f.abs(), -e.unsqueeze(-1))
    c = (y > 0.25).to(torch.uint8)
    for border, tie in ((0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False)):
        c += (y >= border) if tie else (y > border)
    return (c + torch.signbit(f).to(torch.uint8) * 8).flatten(-2), e


def _pack_pages(k, v, P):
    """Pages of keys and values (pages, heads, P, D) in the 4-bit cache's layout: codes of both, exponents of both."""
    n, KV, _, D = k.shape
    width = 4 if D <= 128 else 8

    def exponents(e):
        out = torch.zeros(n, KV, P, width, dtype=torch.int8, device=e.device)
        out[..., :D // 32] = e.to(torch.int8)
        return out

    kc, ke = _nibbles(k)
    vc, ve = _nibbles(v)
    kc = kc[..., 0::2] | (kc[..., 1::2] << 4)
    # value (32 b + 8 g + 2 j + i, 16 f + c) lies at [b][g][c][f][j], nibble i
    vc = vc.view(n, KV, P // 32, 4, 4, 2, D // 16, 16).permute(0, 1, 2, 3, 7, 6, 4, 5)
    vc = vc[..., 0] | (vc[..., 1] << 4)
    return kc.contiguous(), vc.contiguous(), exponents(ke), exponents(ve)


_GRID = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _unpack(s, pages):
    """Keys and values of these pages as the numbers they stand for, float32: (pages, heads, P, D) each."""
    D, P, KV = s["D"], s["P"], s["KV"]
    grid = torch.tensor(_GRID + [-x for x in _GRID], device=pages.device)
    n = pages.numel()

    def scaled(codes, exps):
        e = exps[pages.flatten()][..., :D // 32].int().unsqueeze(-1)
        return torch.ldexp(grid[codes.long()].unflatten(-1, (-1, 32)), e).flatten(-2)

    def split(c):
        return torch.stack([c & 15, c >> 4], -1)

    k = split(s["k"][pages.flatten()]).flatten(-2)
    v = split(s["v"][pages.flatten()]).permute(0, 1, 2, 3, 6, 7, 5, 4).reshape(n, KV, P, D)
    return scaled(k, s["ke"]), scaled(v, s["ve"])


def prepare(case, seed):
    if case["op"] == "verify":
        return _prepare_verify(case, seed)
    dt, KV, D, P, op, B = _DT[case["dt"]], case["KV"], case["D"], case["P"], case["op"], case["B"]
    table, lens, refs, new = _tables(case)
    n_pages = len(refs)
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    way = torch.randn(KV, 1, D, generator=g, device="cuda")

    def keys(n):
        k = torch.randn(n, KV, P, D, generator=g, device="cuda", dtype=dt)
        k += way.to(dt)
        k += torch.randn(n, KV, 1, D, generator=g, device="cuda", dtype=dt) * 0.5
        return k

    s = dict(case, table=_ints(table), lens=_ints(lens), refs=_ints(refs), status=_ints(np.zeros(1)), cu=_ints(np.concatenate([[0], np.cumsum(new)])),
             new=_ints(new), max_len=int(lens.max()), max_new=int(new.max()), total=int(new.sum()))
    N = s["total"]
    if op == "window":
        s["k"], s["v"] = keys(n_pages), torch.randn(n_pages, KV, D, P, generator=g, device="cuda", dtype=dt)
    else:
        width = 4 if D <= 128 else 8
        s["k"] = torch.empty(n_pages, KV, P, D // 2, dtype=torch.uint8, device="cuda")
        s["v"] = torch.empty(n_pages, KV, P // 32, 4, 16, D // 16, 4, dtype=torch.uint8, device="cuda")
        s["ke"], s["ve"] = torch.empty(n_pages, KV, P, width, dtype=torch.int8, device="cuda"), torch.empty(n_pages, KV, P, width, dtype=torch.int8, device="cuda")
        some = max(1, 50000000 // (KV * P * D))
        for i in range(0, n_pages, some):
            n = min(some, n_pages - i)
            for name, t in zip(("k", "v", "ke", "ve"), _pack_pages(keys(n), torch.randn(n, KV, P, D, generator=g, device="cuda", dtype=dt), P)):
                s[name][i:i + n] = t
    if op == "store":
        # the key and value part of a fused projection's output: tokens are further apart than KV * D
        s["kvnew"] = torch.randn(N, 3 * KV * D, generator=g, device="cuda", dtype=dt)
        s["k_new"], s["v_new"] = s["kvnew"][:, KV * D:2 * KV * D].unflatten(1, (KV, D)), s["kvnew"][:, 2 * KV * D:].unflatten(1, (KV, D))
        s["k_new"] += way.squeeze(1).to(dt)
        return s
    H = case["H"]
    s["qkv"] = torch.randn(N, (H + 2 * KV) * D, generator=g, device="cuda", dtype=dt) * 1.5
    s["q"] = s["qkv"][:, :H * D].unflatten(1, (H, D))
    s["scale"] = 1.0 / math.sqrt(D)
    s["mask"] = None
    if case["tree"]:   # each drafted token hangs on an earlier one or on the last cached one
        T = s["max_new"]
        rng = np.random.RandomState(seed % (1 << 31))
        see = np.zeros((B, T, -(-T // 32) * 32), np.uint8)
        for i in range(T):
            parent = rng.randint(-1, i, B) if i else np.full(B, -1)
            see[:, i] = np.where(parent[:, None] >= 0, see[np.arange(B), np.maximum(parent, 0)], 0)
            see[:, i, i] = 1
        rows = np.concatenate([see[b, :new[b]] for b in range(B)])
        s["mask"] = torch.from_numpy(np.packbits(rows, axis=1, bitorder="little").view(np.int32).copy()).cuda()
    return s


def run(s):
    if own:
        return _run_own(s)
    return {"window": _plain_attention, "kv4": _plain_attention, "store": _plain_store, "verify": _plain_verify}[s["op"]](s)


def _run_own(s):
    from paper_2407_12075_amd import kv
    op = s["op"]
    if op == "verify":
        return kv.tbn_verify(s["target"], s["tokens"], s["u"], s["cu"], s["max_new"], draft=s["draft_p"], parents=s["parents"])
    if "pool" not in s:   # the handles that a program keeps with its cache
        s["pool"] = kv.KVPool(s["k"], s["v"]) if op == "window" else kv.KV4Pool(s["k"], s["v"], s["ke"], s["ve"])
        s["index"] = kv.KVIndex(s["table"], s["lens"], s["refs"], s["status"], s["P"])
    pool, index = s["pool"], s["index"]
    if op == "store":
        kv.tbn_kv4_append(pool, index, s["k_new"], s["v_new"], s["cu"], s["max_new"])
        return kv.tbn_kv4_read(pool, index, s["cu"], s["max_new"], s["total"], s["k_new"].dtype)
    if op == "window":
        return kv.tbn_window_attention(s["q"], pool, index, s["cu"], s["max_new"], s["sink"], s["window"], mask=s["mask"], scale=s["scale"],
                                       max_len=s["max_len"])
    return kv.tbn_kv4_attention(s["q"], pool, index, s["cu"], s["max_new"], mask=s["mask"], n_sink=s["sink"], window=s["window"], scale=s["scale"],
                                max_len=s["max_len"])


# ---- the plain forms -------------------------------------------------------------------------------------------------------


def _rows(s):
    """For the call's tokens: sequence, place within its tokens; and the padded (B, T) indices of the tokens."""
    cu, dev = s["cu"].long(), s["cu"].device
    i = torch.arange(s["total"], device=dev)
    seq = (i[:, None] >= cu[None, 1:]).sum(1)
    padded = (cu[:-1, None] + torch.arange(s["max_new"], device=dev)).clamp(max=s["total"] - 1)
    return seq, i - cu[seq], padded


def _plain_attention(s):
    KV, D, P, H, T, B = s["KV"], s["D"], s["P"], s["H"], s["max_new"], s["B"]
    G, np_ = H // KV, -(-s["max_len"] // P)
    seq, place, padded = _rows(s)
    pages = s["table"][:, :np_].long().clamp(min=0)
    if s["op"] == "window":
        k = s["k"][pages].float().permute(0, 2, 1, 3, 4).reshape(B * KV, np_ * P, D)
        v = s["v"][pages].float().permute(0, 2, 1, 4, 3).reshape(B * KV, np_ * P, D)
    else:
        k, v = (t.view(B, np_, KV, P, D).permute(0, 2, 1, 3, 4).reshape(B * KV, np_ * P, D) for t in _unpack(s, pages))
    q = s["q"].float()[padded].view(B, T, KV, G, D).permute(0, 2, 3, 1, 4).reshape(B * KV, G * T, D)
    a = (torch.bmm(q, k.transpose(1, 2).contiguous()) * s["scale"]).view(B, KV * G, T, np_ * P)
    lens, new = s["lens"].long(), s["new"].long()
    at = torch.arange(np_ * P, device=a.device)
    first = (lens - new)[:, None]
    draft = at[None] - first   # place among the call's tokens, negative for the keys before them
    if s["mask"] is None:
        where = first + torch.arange(T, device=a.device)   # (B, T): the key of a token
        see = at <= where[:, :, None]
        if s["window"]:
            see &= (at < s["sink"]) | (at > where[:, :, None] - s["window"])
    else:
        words = s["mask"][padded]   # (B, T, words)
        j = draft.clamp(0, words.shape[2] * 32 - 1)
        word = torch.gather(words, 2, (j // 32)[:, None, :].expand(B, T, -1))
        hung = ((word >> (j % 32).int()[:, None, :]) & 1 == 1) & ((draft >= 0) & (draft < new[:, None]))[:, None, :]
        see = (draft < 0)[:, None, :].expand(B, T, -1)
        if s["window"]:   # a drafted token's place follows from the tokens above it
            where = first + hung.sum(2) - 1
            see = see & ((at < s["sink"]) | (at > where[:, :, None] - s["window"]))
        see = see | hung
    see = (see & (at[None] < lens[:, None])[:, None, :])[:, None]
    a = torch.where(see, a, torch.full_like(a, -math.inf)).view(B * KV, G * T, np_ * P)
    m = a.amax(-1, keepdim=True)
    m = torch.where(torch.isinf(m), torch.zeros_like(m), m)
    p = torch.exp(a - m)
    z = p.sum(-1, keepdim=True)
    o = torch.bmm(p, v) / torch.where(z == 0, torch.ones_like(z), z)
    lse = (m + torch.log(z)).squeeze(-1)
    o = o.view(B, H, T, D).permute(0, 2, 1, 3)[seq, place]
    return o.to(s["q"].dtype), lse.view(B, H, T).permute(0, 2, 1)[seq, place]


def _plain_store(s):
    """The words that the new keys share with older ones are taken from the cache and put back."""
    KV, D, P, dt = s["KV"], s["D"], s["P"], s["k_new"].dtype
    seq, place, _ = _rows(s)
    at = (s["lens"].long() - s["new"].long())[seq] + place
    page, row = s["table"][seq, at // P].long(), at % P
    width = s["ke"].shape[3]
    kc, ke = _nibbles(s["k_new"])
    vc, ve = _nibbles(s["v_new"])
    s["k"][page, :, row] = kc[..., 0::2] | (kc[..., 1::2] << 4)
    for name, e in (("ke", ke), ("ve", ve)):
        s[name][page, :, row] = torch.nn.functional.pad(e, (0, width - D // 32)).to(torch.int8)
    for i in (0, 1):   # even keys' nibbles, then the odd ones'
        mine = torch.nonzero(row % 2 == i).squeeze(1)
        p, r = page[mine], row[mine]
        c = vc[mine].view(-1, KV, D // 16, 16).transpose(2, 3)
        old = s["v"][p, :, r // 32, r // 8 % 4, :, :, r // 2 % 4]
        s["v"][p, :, r // 32, r // 8 % 4, :, :, r // 2 % 4] = (old & 0xF0) | c if i == 0 else (old & 0x0F) | (c << 4)
    grid = torch.tensor(_GRID + [-x for x in _GRID], device=page.device)
    k = s["k"][page, :, row]
    v = s["v"][page, :, row // 32, row // 8 % 4, :, :, row // 2 % 4].transpose(2, 3).reshape(-1, KV, D)
    v = torch.where((row % 2 == 0)[:, None, None], v & 15, v >> 4)
    out = []
    for c, e in ((torch.stack([k & 15, k >> 4], -1).flatten(-2), s["ke"]), (v, s["ve"])):
        e = e[page, :, row][..., :D // 32].int().unsqueeze(-1)
        out.append(torch.ldexp(grid[c.long()].unflatten(-1, (-1, 32)), e).flatten(-2).to(dt))
    return tuple(out)


def _plain_verify(s):
    """All sequences together, place by place: r is what is left of the target's row of a sequence's last accepted token, m its sum."""
    B, T, dev = s["B"], s["max_new"], s["u"].device
    cu = s["cu"].long()
    first, new = cu[:-1], cu[1:] - cu[:-1]
    b = torch.arange(B, device=dev)
    left = lambda row: s["target"][row].double().clamp(min=0)  # noqa: E731
    cur, r, m = torch.zeros_like(first), left(first), torch.ones(B, dtype=torch.float64, device=dev)
    picks = torch.full((B, T), -1, dtype=torch.int32, device=dev)
    picks[:, 0] = 0
    counts = torch.ones(B, dtype=torch.int32, device=dev)
    for j in range(1, T):
        row = (first + j).clamp(max=s["total"] - 1)
        parent = torch.full_like(cur, j - 1) if s["parents"] is None else s["parents"][row].long()
        asked = (j < new) & (parent == cur)
        tok, u = s["tokens"][row].long(), s["u"][row].double()
        above = (first + cur).clamp(max=s["total"] - 1)
        q = None if s["draft_p"] is None else s["draft_p"][above].double().clamp(min=0)
        here = r[b, tok]
        t = m if q is None else m * q[b, tok]
        yes = asked & (u * t < here)
        no = asked & ~yes
        if q is None:
            rest = r.clone()
            rest[b, tok] = 0
            sums = (m - here).clamp(min=0)
        else:
            rest = (r - m[:, None] * q).clamp(min=0)
            sums = rest.sum(1)
        r = torch.where(yes[:, None], left(row), torch.where(no[:, None], rest, r))
        m = torch.where(yes, torch.ones_like(m), torch.where(no, sums, m))
        cur = torch.where(yes, torch.full_like(cur, j), cur)
        picks[b, counts.long().clamp(max=T - 1)] = torch.where(yes, torch.full_like(counts, j), picks[b, counts.long().clamp(max=T - 1)])
        counts += yes.int()
    sums = torch.cumsum(r, 1)
    above = (sums > s["u"][first].double()[:, None] * sums[:, -1:]) & (r > 0)
    return picks, counts, above.int().argmax(1).int()


# ---- 64 bits ---------------------------------------------------------------------------------------------------------------


def _exact_values(codes, exps):
    """What 4-bit codes stand for: sign, two bits of exponent, one of mantissa."""
    c = codes.long()
    e, f = (c >> 1) & 3, (c & 1).double()
    x = torch.where(e == 0, f * 0.5, (1 + f * 0.5) * torch.exp2(e.double() - 1))
    return torch.where(c >= 8, -x, x) * torch.exp2(exps.double()).repeat_interleave(32, -1)


def _exact_quantized(x):
    """The nearest values of the grid, found among all of them."""
    f = x.double().unflatten(-1, (-1, 32))
    a = f.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(a.clamp(min=1e-300) / 6)).clamp(-100, 125)
    e = torch.where(6 * torch.exp2(e - 1) >= a, (e - 1).clamp(min=-100), e)
    e = torch.where(6 * torch.exp2(e) < a, (e + 1).clamp(max=125), e)
    y = f.abs() / torch.exp2(e)
    best, gap = torch.zeros_like(y), y.clone()
    for code, value in enumerate((0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0), 1):
        d = (y - value).abs()
        take = (d < gap) | ((d == gap) & (code % 2 == 0))
        best, gap = torch.where(take, torch.full_like(y, value), best), torch.where(take, d, gap)
    return (torch.sign(f) * best * torch.exp2(e)).flatten(-2)


def _exact_verify(s):
    """One sequence after another, along its tree."""
    picks = np.full((s["B"], s["max_new"]), -1, np.int32)
    counts, follows = np.zeros(s["B"], np.int32), np.zeros(s["B"], np.int32)
    cu, tokens, u = s["cu"].tolist(), s["tokens"].tolist(), s["u"].double().tolist()
    parents = None if s["parents"] is None else s["parents"].tolist()
    for b in range(s["B"]):
        t0, t1 = cu[b], cu[b + 1]
        up = [(i - 1 if parents is None else parents[t0 + i]) for i in range(t1 - t0)]
        path, at, moved = [0], 0, True
        while moved:
            moved = False
            row = s["target"][t0 + at].double()
            mass = 1.0
            for c in [i for i in range(t1 - t0) if i > at and up[i] == at]:
                tok = tokens[t0 + c]
                q = None if s["draft_p"] is None else s["draft_p"][t0 + at].double()
                if u[t0 + c] * (mass if q is None else mass * float(q[tok])) < float(row[tok]):
                    at, moved = c, True
                    path.append(c)
                    break
                if q is None:
                    mass = max(mass - float(row[tok]), 0.0)
                    row[tok] = 0.0
                else:
                    row = torch.relu(row - mass * q)
                    mass = float(row.sum())
        sums = torch.cumsum(row, 0)
        ahead = torch.nonzero(sums > u[t0] * float(sums[-1]))
        follows[b] = int(ahead[0])
        picks[b, :len(path)] = path
        counts[b] = len(path)
    return picks, counts, follows


def exact(case, seed):
    """Attention from its definition, sequence by sequence and key head by key head."""
    s = prepare(case, seed)
    if case["op"] == "verify":
        return tuple(torch.from_numpy(t).cuda() for t in _exact_verify(s))
    if case["op"] == "store":
        return _exact_quantized(s["k_new"]), _exact_quantized(s["v_new"])
    D, P, H, KV = s["D"], s["P"], s["H"], s["KV"]
    G = H // KV
    cu, lens = s["cu"].tolist(), s["lens"].tolist()
    table = s["table"].cpu().numpy()
    out = torch.zeros(s["total"], H, D, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["total"], H, dtype=torch.float64, device="cuda")
    for b in range(s["B"]):
        L, t0, t1 = lens[b], cu[b], cu[b + 1]
        T, first = t1 - t0, lens[b] - (t1 - t0)
        pages = torch.from_numpy(table[b, :-(-L // P)].astype(np.int64)).cuda()
        key = torch.arange(L, device="cuda")
        if s["mask"] is not None:
            bits = np.unpackbits(s["mask"][t0:t1].cpu().numpy().view(np.uint8), axis=1, bitorder="little")[:, :T]
            see_new = torch.from_numpy(bits.astype(bool)).cuda()
            depth = see_new.sum(1) - 1
        else:
            see_new = torch.ones(T, T, dtype=torch.bool, device="cuda").tril()
            depth = torch.arange(T, device="cuda")
        see = torch.cat([torch.ones(T, first, dtype=torch.bool, device="cuda"), see_new], 1)
        if s["window"]:
            far = (first + depth)[:, None] - key[None] >= s["window"]
            if s["mask"] is not None:
                far[:, first:] = False
            see &= ~(far & (key >= s["sink"])[None])
        for h in range(KV):
            if s["op"] == "window":
                k = s["k"][pages, h].double().reshape(-1, D)[:L]
                v = s["v"][pages, h].double().transpose(1, 2).reshape(-1, D)[:L]
            else:
                kc, vc = s["k"][pages, h], s["v"][pages, h]   # (pages, P, D / 2), (pages, P / 32, 4, 16, D / 16, 4)
                kc = torch.stack([kc % 16, kc // 16], -1).reshape(-1, D)
                vc = torch.stack([vc % 16, vc // 16], -1).permute(0, 1, 2, 5, 6, 4, 3).reshape(-1, D)
                k = _exact_values(kc, s["ke"][pages, h].reshape(len(pages) * P, -1)[:, :D // 32])[:L]
                v = _exact_values(vc, s["ve"][pages, h].reshape(len(pages) * P, -1)[:, :D // 32])[:L]
            for g in range(G):
                a = (s["q"][t0:t1, h * G + g].double() @ k.T) * s["scale"]
                a = a.masked_fill(~see, -math.inf)
                norm = torch.logsumexp(a, 1)
                lse[t0:t1, h * G + g] = norm
                out[t0:t1, h * G + g] = torch.exp(a - norm[:, None]) @ v
    return out, lse
