"""CPU oracle of the verification of drafted tokens: one loop per rule of include/tbn.h, Python floats (binary64), sums exact but for one rounding.
Shares no code with the library."""
from __future__ import annotations

import math

import numpy as np


def clean(row):
    """Numbers above 0; all others count as 0."""
    row = np.asarray(row, np.float64)
    return np.where(row > 0, row, 0.0)


def draw(r, u):
    """First place whose prefix sum is above u * sum, else the last that is not 0; -1 without a positive finite sum."""
    total = math.fsum(r) if np.isfinite(r).all() else math.inf
    if not (0 < total < math.inf):
        return -1
    limit, s, last = u * total, 0.0, -1
    for v in np.nonzero(r)[0]:
        s += r[v]
        last = int(v)
        if s > limit:
            return int(v)
    return last


def verify(target, draft, tokens, parents, u):
    """One sequence: arrays of its T tokens (draft, parents: or None).  (accepted places, token that follows)."""
    T, V = np.asarray(target).shape
    x, path = 0, [0]
    while True:
        r, m, moved = clean(target[x]), 1.0, False
        for c in range(x + 1, T):
            if (c - 1 if parents is None else parents[c]) != x:
                continue
            t = int(tokens[c])
            known = 0 <= t < V
            here = r[t] if known else 0.0
            if draft is None:
                if float(u[c]) * m < here:
                    moved = True
                else:
                    if known:
                        r[t] = 0.0
                    m = max(m - here, 0.0)
            else:
                q = clean(draft[x])
                if float(u[c]) * (m * (q[t] if known else 0.0)) < here:
                    moved = True
                else:
                    r = np.maximum(r - m * q, 0.0)
                    m = math.fsum(r)
            if moved:
                x = c
                path.append(c)
                break
        if not moved:
            break
    token = draw(r, float(u[0]))
    return path, token if token >= 0 else draw(clean(target[x]), float(u[0]))
