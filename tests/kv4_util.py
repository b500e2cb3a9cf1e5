"""Caches in 4 bits for the tests: keys and values of known numbers in the library's layout, everything else of a pool random bytes."""
import numpy as np
import torch

from oracle import kv4_oracle as o4


def codes_of(rng, n, kv_heads, dim, no_number=0.0):
    """Codes and exponents of n tokens whose keys and values are of ordinary size: (n, kv_heads, dim) and (n, kv_heads, dim / 32), keys' and values'."""
    shape, groups = (n, kv_heads, dim), (n, kv_heads, dim // 32)
    kc, vc = rng.choice(16, shape, p=[.1, .1, .1, .08, .05, .04, .02, .01] * 2), rng.choice(16, shape)
    ke, ve = rng.randint(-2, 1, groups), rng.randint(-4, 0, groups)
    gone = rng.rand(n, kv_heads) < no_number
    ke[gone], ve[gone] = o4.NO_NUMBER, o4.NO_NUMBER
    return kc, vc, ke, ve


def place(pool, page, row, kc, vc, ke, ve):
    """Tokens at pages `page` and rows `row` (arrays of n) of a numpy pool, all at once."""
    D = pool.dim
    pool.k[page, :, row] = (kc[..., 0::2] | (kc[..., 1::2] << 4)).astype(np.uint8)
    pool.k_exp[page, :, row, :D // 32], pool.v_exp[page, :, row, :D // 32] = ke, ve
    d = np.arange(D)
    for half in (0, 1):
        mine = row % 2 == half
        p, r, c = page[mine], row[mine], vc[mine]
        h = np.arange(pool.kv_heads)
        at = (p[:, None, None], h[None, :, None], (r // 32)[:, None, None], (r % 32 // 8)[:, None, None], (d % 16)[None, None], (d // 16)[None, None],
              (r % 8 // 2)[:, None, None])
        old = pool.v[at]
        pool.v[at] = ((old & 0xF0) | c if half == 0 else (old & 0x0F) | (c << 4)).astype(np.uint8)


def make_cache4(kv, kv_heads, dim, page, lens, seed=0, max_pages=None, extra_pages=3, n_pages=None, no_number=0.0):
    """A pool of random bytes with the sequences' tokens in it, an index with pages anywhere, and the float64 numbers (length, kv_heads, dim)."""
    rng = np.random.RandomState(seed)
    need = [-(-l // page) for l in lens]
    n_pages = n_pages or sum(need) + extra_pages
    max_pages = max_pages or max(need + [1])
    order = rng.permutation(n_pages)
    host = o4.Pool(n_pages, kv_heads, dim, page, fill=seed + 1)
    table, refs = np.full((len(lens), max_pages), -7, np.int32), np.zeros(n_pages, np.int32)
    keys, values, at = [], [], 0
    for s, l in enumerate(lens):
        pages = order[at:at + need[s]]
        at += need[s]
        table[s, :need[s]], refs[pages] = pages, 1
        c = codes_of(rng, l, kv_heads, dim, no_number)
        if l:
            place(host, pages[np.arange(l) // page], np.arange(l) % page, *c)
        keys.append(o4.numbers(c[0], c[2]))
        values.append(o4.numbers(c[1], c[3]))
    pool = kv.KV4Pool(*(torch.from_numpy(t).cuda() for t in (host.k, host.v, host.k_exp, host.v_exp)))
    index = kv.kv_index(len(lens), max_pages, n_pages, page)
    index.table.copy_(torch.from_numpy(table))
    index.refs.copy_(torch.from_numpy(refs))
    index.lens.copy_(torch.tensor(lens, dtype=torch.int32))
    return pool, index, keys, values


def host_of(pool, like=None):
    """A numpy pool with the device's bytes."""
    host = o4.Pool(1, pool.kv_heads, pool.dim, pool.page)
    host.k, host.v, host.k_exp, host.v_exp = (t.cpu().numpy().copy() for t in (pool.k, pool.v, pool.k_exp, pool.v_exp))
    return host
