"""CPU oracle of the cache held in 4 bits: numbers and layout as include/tbn.h defines them, plain numpy, float64.  Shares no code with the library."""
from __future__ import annotations

import numpy as np

VALUES = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
NO_NUMBER = -128


def exponent(a):
    """Least x, -100 .. 125, with a <= 6 * 2^x."""
    x = -100
    while x < 125 and a > 6 * 2.0 ** x:
        x += 1
    return x


def group(f):
    """Codes and exponent of 32 finite numbers."""
    x = exponent(np.abs(f).max())
    y = np.abs(f) / 2.0 ** x
    gap = np.abs(y[:, None] - VALUES[None])
    best = gap.min(1)
    codes = np.zeros(len(f), np.int64)
    for i in range(len(f)):
        nearest = [c for c in range(8) if gap[i, c] == best[i]]
        codes[i] = nearest[0] if len(nearest) == 1 else [c for c in nearest if c % 2 == 0][0]
    return codes + 8 * np.signbit(f), x


def quantize(k, v):
    """Keys and values (kv_heads, dim) of one token: codes and exponents of both."""
    H, D = k.shape
    out = [np.zeros((H, D), np.int64), np.zeros((H, D), np.int64), np.full((H, D // 32), NO_NUMBER), np.full((H, D // 32), NO_NUMBER)]
    for h in range(H):
        if not (np.isfinite(k[h]).all() and np.isfinite(v[h]).all()):
            continue
        for which, t in enumerate((k[h], v[h])):
            for c in range(D // 32):
                out[which][h, 32 * c:32 * c + 32], out[2 + which][h, c] = group(t[32 * c:32 * c + 32])
    return out


def numbers(codes, exps):
    """What codes (.., dim) with exponents (.., dim / 32) stand for."""
    codes, exps = np.asarray(codes), np.asarray(exps)
    f = VALUES[codes % 8] * np.where(codes >= 8, -1.0, 1.0)
    scale = np.where(exps == NO_NUMBER, np.nan, 2.0 ** exps.astype(np.float64))
    return f * np.repeat(scale, 32, axis=-1)


def key_byte(d):
    """Byte of a row of keys and half of it that hold channel d."""
    return d // 2, d % 2


def value_byte(row, d):
    """Place [b][g][n][f][j] of a page's values and half of that byte that hold channel d of a row."""
    return (row // 32, row % 32 // 8, d % 16, d // 16, row % 8 // 2), row % 2


def put(half, byte, code):
    """A byte with `code` in one of its halves."""
    return (byte & 0xF0) | code if half == 0 else (byte & 0x0F) | (code << 4)


def get(half, byte):
    return byte & 15 if half == 0 else byte >> 4


class Pool:
    """Arrays as the library has them, filled key by key."""

    def __init__(self, n_pages, kv_heads, dim, page, fill=None):
        e = 4 if dim <= 128 else 8
        rng = np.random.RandomState(fill)
        shapes = ((page, dim // 2), (page // 32, 4, 16, dim // 16, 4), (page, e), (page, e))
        self.k, self.v, self.k_exp, self.v_exp = (rng.randint(0, 256, (n_pages, kv_heads) + s).astype(np.uint8) for s in shapes)
        self.k_exp, self.v_exp = self.k_exp.view(np.int8), self.v_exp.view(np.int8)
        self.dim, self.page, self.kv_heads = dim, page, kv_heads

    def write(self, page, row, codes):
        """A token's codes and exponents, as quantize gives them."""
        kc, vc, ke, ve = codes
        for h in range(self.kv_heads):
            for d in range(self.dim):
                b, half = key_byte(d)
                self.k[page, h, row, b] = put(half, int(self.k[page, h, row, b]), int(kc[h, d]))
                at, half = value_byte(row, d)
                self.v[(page, h) + at] = put(half, int(self.v[(page, h) + at]), int(vc[h, d]))
            self.k_exp[page, h, row, :self.dim // 32] = ke[h]
            self.v_exp[page, h, row, :self.dim // 32] = ve[h]

    def read(self, page, row):
        """Codes and exponents of a token."""
        D = self.dim
        kc, vc = np.zeros((self.kv_heads, D), np.int64), np.zeros((self.kv_heads, D), np.int64)
        for h in range(self.kv_heads):
            for d in range(D):
                b, half = key_byte(d)
                kc[h, d] = get(half, int(self.k[page, h, row, b]))
                at, half = value_byte(row, d)
                vc[h, d] = get(half, int(self.v[(page, h) + at]))
        return kc, vc, self.k_exp[page, :, row, :D // 32].astype(np.int64), self.v_exp[page, :, row, :D // 32].astype(np.int64)
