"""Caches for the tests of the attention over pages: the same keys and values in the library's tensors and as float64 arrays."""
import numpy as np
import torch

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def make_cache(kv, dt, kv_heads, dim, page, lens, seed=0, max_pages=None, extra_pages=3, n_pages=None, summary=False, garbage=float("nan"), far=False):
    """A pool whose every unused element is `garbage`, an index with pages anywhere in it (far: at its end), and float64 (length,
    kv_heads, dim) keys and values per sequence."""
    rng = np.random.RandomState(seed)
    need = [-(-l // page) for l in lens]
    n_pages = n_pages or sum(need) + extra_pages
    max_pages = max_pages or max(need + [1])
    order = rng.permutation(sum(need)) + (n_pages - sum(need)) if far else rng.permutation(n_pages)
    pool = kv.kv_pool(n_pages, kv_heads, dim, page, DT[dt], summary)
    index = kv.kv_index(len(lens), max_pages, n_pages, page)
    if not far:
        pool.k.fill_(garbage)
        pool.v.fill_(garbage)
    table = np.full((len(lens), max_pages), -7, np.int32)   # entries behind the last page are nobody's business
    refs = np.zeros(n_pages, np.int32)
    keys, values, at = [], [], 0
    for s, l in enumerate(lens):
        k = torch.from_numpy(rng.standard_normal((l, kv_heads, dim))).to(DT[dt])
        v = torch.from_numpy(rng.standard_normal((l, kv_heads, dim))).to(DT[dt])
        k += torch.from_numpy(rng.standard_normal((1, kv_heads, dim))).to(DT[dt])
        for b in range(need[s]):
            p = int(order[at])
            at += 1
            table[s, b] = p
            refs[p] = 1
            n = min(page, l - b * page)
            if far:
                pool.k[p].fill_(garbage)
                pool.v[p].fill_(garbage)
            pool.k[p, :, :n] = k[b * page:b * page + n].transpose(0, 1).cuda()
            pool.v[p, :, :, :n] = v[b * page:b * page + n].permute(1, 2, 0).cuda()
        keys.append(k.double().numpy())
        values.append(v.double().numpy())
    index.table.copy_(torch.from_numpy(table))
    index.refs.copy_(torch.from_numpy(refs))
    index.lens.copy_(torch.tensor(lens, dtype=torch.int32))
    return pool, index, keys, values


def make_queries(dt, counts, heads, dim, seed=1, scale=1.5, stride=None):
    """q (tokens, heads, dim) on the device, tokens `stride` elements apart; cu; float64 copy."""
    rng = np.random.RandomState(seed)
    n = sum(counts)
    x = torch.from_numpy(rng.standard_normal((n, heads, dim)) * scale).to(DT[dt])
    if stride is None:
        q = x.cuda()
    else:
        q = torch.full((n, stride), float("nan"), dtype=DT[dt]).cuda()
        q[:, :heads * dim] = x.reshape(n, -1).cuda()
        q = q[:, :heads * dim].unflatten(1, (heads, dim))
    cu = torch.from_numpy(np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)).cuda()
    return q, cu, x.double().numpy()


def pack_mask(see, words):
    """Rows of bits (tokens, any) to int32 (tokens, words)."""
    bits = np.zeros((see.shape[0], words * 32), np.uint8)
    bits[:, :see.shape[1]] = see
    return torch.from_numpy(np.packbits(bits, axis=1, bitorder="little").view(np.int32).copy()).cuda()


def tolerance(dt, values):
    """Largest error of an output element.  A weight e^(a - m) is off by the logit's error (sums of dim products of binary32: about
    1e-6 of a few units) and a few units of 2^-24, relative: 2e-5 of the largest |v| covers the weighted mean of them.  bfloat16
    adds 2^-9 for the rounded weights and 2^-9 for the rounded output, both at most of the largest |v|."""
    top = max([float(np.abs(v[np.isfinite(v)]).max()) for v in values if v.size and np.isfinite(v).any()] + [1e-30])
    return (2e-5 + (2.0 ** -8 if dt == "bf16" else 0.0)) * top


LSE_TOLERANCE = 5e-5   # absolute, on logits of at most about 30: the same errors of the logits, and the rounding of lse itself


def compare(out, lse, ref, ref_lse, tol):
    """NaN and infinities in the same places, everything else within tol."""
    out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    assert np.array_equal(np.isnan(out), np.isnan(ref))
    fine = np.isfinite(ref)
    assert np.array_equal(out[~fine & ~np.isnan(ref)], ref[~fine & ~np.isnan(ref)])
    if fine.any():
        err = np.abs(out[fine] - ref[fine]).max()
        assert err <= tol, f"error {err:.3e}, at most {tol:.3e}"
    assert np.array_equal(np.isneginf(lse), np.isneginf(ref_lse))
    fine = np.isfinite(ref_lse)
    if fine.any():
        err = np.abs(lse[fine] - ref_lse[fine]).max()
        assert err <= LSE_TOLERANCE, f"lse error {err:.3e}"
