"""CPU oracle of the paged key/value cache and its attention: plain numpy, float64, one loop per definition of include/tbn.h.
Shares no code with the library.  bfloat16 data are float64 arrays that hold bfloat16 values."""
from __future__ import annotations

import math

import numpy as np


class Cache:
    """Bookkeeping as a list of pages per sequence, and the pages' contents."""

    def __init__(self, n_seqs, max_pages, n_pages, page, kv_heads=1, dim=8):
        self.page, self.max_pages, self.n_pages = page, max_pages, n_pages
        self.rows = [[] for _ in range(n_seqs)]
        self.lens = [0] * n_seqs
        self.refs = [0] * n_pages
        self.status = 0
        self.k = np.zeros((n_pages, kv_heads, page, dim))
        self.v = np.zeros((n_pages, kv_heads, dim, page))

    def reserve(self, n_new):
        """Pairs (source, target) per sequence; (-1, -1) where nothing is copied."""
        none = [(-1, -1)] * len(self.lens)
        if self.status:
            return none
        if any(n < 0 or -(-(l + n) // self.page) > self.max_pages for l, n in zip(self.lens, n_new)):
            self.status = 2
            return none
        free = [p for p in range(self.n_pages) if self.refs[p] == 0]
        refs, rows, pairs, lens = list(self.refs), [list(r) for r in self.rows], [], list(self.lens)
        for s, n in enumerate(n_new):
            pair = (-1, -1)
            if n > 0:
                want = -(-(lens[s] + n) // self.page)
                fresh = want - len(rows[s])
                shared = lens[s] % self.page != 0 and refs[rows[s][-1]] > 1
                if fresh + shared > len(free):
                    self.status = 1
                    return none
                if shared:
                    old = rows[s][-1]
                    refs[old] -= 1
                    rows[s][-1] = free.pop(0)
                    refs[rows[s][-1]] = 1
                    pair = (old, rows[s][-1])
                for _ in range(fresh):
                    rows[s].append(free.pop(0))
                    refs[rows[s][-1]] = 1
                lens[s] += n
            pairs.append(pair)
        self.refs, self.rows, self.lens = refs, rows, lens
        return pairs

    def fork(self, parents, children):
        n = len(self.lens)
        good = []
        for i, (a, b) in enumerate(zip(parents, children)):
            ok = 0 <= a < n and 0 <= b < n and b not in list(children)[:i] and b not in list(parents) and self.lens[b] == 0
            good.append(ok)
        for ok, a, b in zip(good, parents, children):
            if not ok:
                self.status = self.status or 2
                continue
            self.rows[b], self.lens[b] = list(self.rows[a]), self.lens[a]
            for p in self.rows[b]:
                self.refs[p] += 1

    def release(self, keep):
        for s, left in enumerate(keep):
            self.lens[s] = min(self.lens[s], max(left, 0))
            want = -(-self.lens[s] // self.page)
            for p in self.rows[s][want:]:
                self.refs[p] -= 1
            self.rows[s] = self.rows[s][:want]

    def compact(self):
        used = sum(r > 0 for r in self.refs)
        src = [p for p in range(used, self.n_pages) if self.refs[p] > 0]
        dst = [p for p in range(used) if self.refs[p] == 0]
        to = dict(zip(src, dst))
        for a, b in to.items():
            self.refs[a], self.refs[b] = 0, self.refs[a]
        self.rows = [[to.get(p, p) for p in r] for r in self.rows]
        return src, dst

    def copy(self, pairs):
        for a, b in pairs:
            if a >= 0 and b >= 0:
                self.k[b], self.v[b] = self.k[a], self.v[a]

    def put(self, s, at, k, v):
        """Key and value (kv_heads, dim) at place `at` of sequence s."""
        p, r = self.rows[s][at // self.page], at % self.page
        self.k[p, :, r], self.v[p, :, :, r] = k, v

    def append(self, s, k, v):
        """The last keys of a sequence, (n, kv_heads, dim)."""
        for i in range(len(k)):
            self.put(s, self.lens[s] - len(k) + i, k[i], v[i])

    def keep(self, s, base, picks):
        got = [self.key(s, base + p) for p in picks]
        for j, (k, v) in enumerate(got):
            self.put(s, base + j, k, v)

    def key(self, s, at):
        p, r = self.rows[s][at // self.page], at % self.page
        return self.k[p, :, r].copy(), self.v[p, :, :, r].copy()

    def keys(self, s):
        """(length, kv_heads, dim) keys and values of a sequence."""
        kv = [self.key(s, i) for i in range(self.lens[s])]
        h, d = self.k.shape[1], self.k.shape[3]
        return np.array([k for k, _ in kv]).reshape(-1, h, d), np.array([v for _, v in kv]).reshape(-1, h, d)


def exponent(a):
    return max(math.frexp(a)[1], -100) if a > 0 else -100


def summary(k):
    """Codes (2, dim) and step of the keys (rows, dim) that a page holds of one kv head."""
    if not np.isfinite(k).all():
        return np.zeros((2, k.shape[1]), np.int64), math.inf
    step = 2.0 ** (exponent(float(np.abs(k).max())) - 6)
    return np.stack([np.ceil(k.max(0) / step), np.floor(k.min(0) / step)]).astype(np.int64), step


def attention(q, k, v, see, scale):
    """One query row (dim) over keys (n, dim); see: which of them.  (out, lse).  Logits that are all -infinity have no weights: as if no key were seen."""
    see = np.asarray(see, bool)
    if not see.any():
        return np.zeros(v.shape[1]), -math.inf
    with np.errstate(invalid="ignore", over="ignore"):
        a = scale * (k[see] @ q)
        m = a.max()
        if m == -math.inf:
            return np.zeros(v.shape[1]), -math.inf
        p = np.exp(a - m)
        return (p[:, None] * v[see]).sum(0) / p.sum(), m if m == math.inf else m + math.log(p.sum())


def picks(q, codes, steps, own, n_select, n_sink, n_recent):
    """Blocks of one query and kv head: q (G, dim); codes (blocks, 2, dim), steps (blocks); own: the query's own block."""
    if own < 0:
        return []
    if own + 1 <= n_select:
        return list(range(own + 1))
    f = np.where(np.isfinite(q), q, 0.0)
    c = np.rint(f * 2.0 ** (6 - exponent(float(np.abs(f).max())))).astype(np.int64)
    forced = list(range(n_sink)) + list(range(own - n_recent + 1, own + 1))
    rest = []
    for b in range(n_sink, own - n_recent + 1):
        whole = int(np.maximum(c * codes[b, 0], c * codes[b, 1]).sum())
        rest.append((-(whole * steps[b] if math.isfinite(steps[b]) else math.inf), b))
    return sorted(forced + [b for _, b in sorted(rest)[:n_select - n_sink - n_recent]])
