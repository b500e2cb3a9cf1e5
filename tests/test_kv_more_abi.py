"""Refusals of attention with a window, of the cache in 4 bits and of the verification, on the CPU: validation runs before any device call."""
import ctypes

import pytest
import torch

from tests.test_kv_abi import FAKE, lib, structs  # noqa: F401  (lib is a fixture)

BIG = 1 << 40


def pool4(**changes):
    from paper_2407_12075_amd import kv
    return kv._Pool4(**{**dict(k=FAKE, v=FAKE, k_exp=FAKE, v_exp=FAKE, n_pages=10, kv_heads=2, dim=64, page=32), **changes})


def at(s):
    at.keep = getattr(at, "keep", []) + [s]
    return ctypes.addressof(s)


def window(lib, p, i, q=FAKE, stride=512, out=FAKE, cu=FAKE, total=5, most=3, heads=4, sink=1, size=9, mask=None, words=0, max_len=0, ws=FAKE, n=BIG):  # noqa: F811
    return lib.tbn_window_attention(q, stride, out, None, p, i, cu, total, most, heads, sink, size, mask, words, max_len, 1.0, ws, n, None)


def attend4(lib, p, i, q=FAKE, stride=512, dt=1, out=FAKE, cu=FAKE, total=5, most=3, heads=4, sink=1, size=0, mask=None, words=0, max_len=0, ws=FAKE, n=BIG):  # noqa: F811
    return lib.tbn_kv4_attention(q, stride, dt, out, None, p, i, cu, total, most, heads, sink, size, mask, words, max_len, 1.0, ws, n, None)


def calls4(lib, p, i):  # noqa: F811
    return {
        "append": lambda: lib.tbn_kv4_append(p, i, FAKE, 128, FAKE, 128, 0, FAKE, 5, 3, None),
        "read": lambda: lib.tbn_kv4_read(p, i, FAKE, FAKE, 0, FAKE, 5, 3, None),
        "keep": lambda: lib.tbn_kv4_keep(p, i, FAKE, FAKE, 2, FAKE, None),
        "attend": lambda: attend4(lib, p, i),
    }


@pytest.mark.parametrize("call", [window, attend4])
def test_queries(lib, call):  # noqa: F811
    pool, index = structs()
    p, i = at(pool if call is window else pool4()), at(index)
    for kw in (dict(q=None), dict(out=None), dict(cu=None)):
        assert call(lib, p, i, **kw) == 1, kw
    for kw in (dict(stride=255), dict(total=-1), dict(most=-1), dict(heads=3), dict(heads=0), dict(max_len=129), dict(max_len=-1), dict(mask=FAKE, words=0, size=3),
               dict(mask=FAKE, words=-1, size=3), dict(sink=-1, size=5), dict(size=-1), dict(mask=FAKE, words=1, size=2)):
        assert call(lib, p, i, **kw) == 2, kw
    for kw in (dict(heads=65538), dict(total=(1 << 30) + 1)):
        assert call(lib, p, i, **kw) == 3, kw
    assert call(lib, p, i, total=0, q=None, out=None, cu=None) == 0 and call(lib, p, i, most=0, q=None) == 0
    if call is window:
        assert call(lib, p, i, size=0) == 2
    else:
        assert call(lib, p, i, dt=2) == 3
    assert call(lib, None, i) == 1 and call(lib, p, None) == 1


def test_workspaces(lib):  # noqa: F811
    big, index = structs(index_max_pages=4000, index_n_seqs=1, pool_kv_heads=1, pool_dt=1)
    small = pool4(kv_heads=1)
    p, i, p4 = at(big), at(index), at(small)
    need = lib.tbn_window_attention_workspace_bytes(p, i, 1, 1, 4, 4, 100000, 0, 0)
    assert need > 0 and lib.tbn_window_attention_workspace_bytes(p, i, 1, 1, 4, 4, 64, 0, 0) == 0   # a short window is not split
    assert lib.tbn_window_attention_workspace_bytes(p, i, 1, 1, 4, 4, 0, 0, 0) == 0
    for ws, n in ((FAKE, need - 1), (None, need), (FAKE + 8, need)):
        assert window(lib, p, i, total=1, most=1, sink=4, size=100000, ws=ws, n=n) == 5
    need = lib.tbn_kv4_attention_workspace_bytes(p4, i, 1, 1, 1, 4, 0, 0, 0, 0)
    assert need > 0 and lib.tbn_kv4_attention_workspace_bytes(p4, i, 2, 1, 1, 4, 0, 0, 0, 0) == 0
    for ws, n in ((FAKE, need - 1), (None, need), (FAKE + 8, need)):
        assert attend4(lib, p4, i, total=1, most=1, ws=ws, n=n) == 5


@pytest.mark.parametrize("field,value,status", [
    ("k", None, 1), ("v", None, 1), ("k_exp", None, 1), ("v_exp", None, 1), ("n_pages", 0, 2), ("kv_heads", 0, 2), ("dim", 0, 2), ("page", 0, 2), ("dim", 48, 3),
    ("dim", 288, 3), ("page", 16, 3), ("kv_heads", 1025, 3), ("n_pages", 1 << 31, 3), ("k", FAKE + 8, 3), ("v", FAKE + 4, 3), ("k_exp", FAKE + 8, 3), ("v_exp", FAKE + 2, 3)])
def test_pool_in_4_bits_is_checked_everywhere(lib, field, value, status):  # noqa: F811
    p, i = at(pool4(**{field: value})), at(structs()[1])
    for name, call in calls4(lib, p, i).items():
        assert call() == status, name
        assert lib.tbn_last_error().decode().startswith("tbn_kv4_"), name
    assert lib.tbn_kv4_copy_pages(p, FAKE, FAKE, 2, None, None) == status


def test_pool_in_4_bits_and_index_agree(lib):  # noqa: F811
    i = at(structs()[1])
    for change in (dict(page=64), dict(n_pages=11)):
        for name, call in calls4(lib, at(pool4(**change)), i).items():
            assert call() == 2, name
    bad = at(structs(index_page=48)[1])
    for name, call in calls4(lib, at(pool4()), bad).items():
        assert call() == 3, name


def test_arguments_of_the_pages(lib):  # noqa: F811
    p, i = at(pool4()), at(structs()[1])
    assert lib.tbn_kv4_append(p, i, FAKE, 127, FAKE, 128, 0, FAKE, 5, 3, None) == 2
    assert lib.tbn_kv4_append(p, i, FAKE, 128, FAKE, 128, 2, FAKE, 5, 3, None) == 3
    assert lib.tbn_kv4_append(p, i, FAKE, 128, None, 128, 0, FAKE, 5, 3, None) == 1
    assert lib.tbn_kv4_append(p, i, FAKE, 128, FAKE, 128, 0, FAKE, -5, 3, None) == 2
    assert lib.tbn_kv4_append(p, i, None, 0, None, 0, 0, None, 0, 0, None) == 0
    assert lib.tbn_kv4_read(p, i, FAKE, FAKE, 0, None, 5, 3, None) == 1 and lib.tbn_kv4_read(p, i, FAKE, FAKE, 7, FAKE, 5, 3, None) == 3
    assert lib.tbn_kv4_read(p, i, FAKE, FAKE, 0, FAKE, 5, -1, None) == 2 and lib.tbn_kv4_read(p, i, None, None, 0, None, 0, 3, None) == 0
    assert lib.tbn_kv4_keep(p, i, FAKE, FAKE, -1, FAKE, None) == 2 and lib.tbn_kv4_keep(p, i, FAKE, None, 1, FAKE, None) == 1
    assert lib.tbn_kv4_copy_pages(p, FAKE, None, 1, None, None) == 1 and lib.tbn_kv4_copy_pages(p, FAKE, FAKE, -1, None, None) == 2
    assert lib.tbn_kv4_copy_pages(p, None, None, 0, None, None) == 0


def verify(lib, target=FAKE, ts=50, draft=FAKE, ds=50, tokens=FAKE, parents=None, u=FAKE, cu=FAKE, total=5, most=3, seqs=2, vocab=50, picks=FAKE, counts=FAKE, next_=FAKE,  # noqa: F811
           ws=FAKE, n=BIG):
    return lib.tbn_verify(target, ts, draft, ds, tokens, parents, u, cu, total, most, seqs, vocab, picks, counts, next_, ws, n, None)


def test_verify(lib):  # noqa: F811
    for kw in (dict(target=None), dict(tokens=None), dict(u=None), dict(cu=None), dict(picks=None), dict(counts=None), dict(next_=None)):
        assert verify(lib, **kw) == 1, kw
    for kw in (dict(ts=49), dict(ds=49), dict(total=-1), dict(most=-1), dict(seqs=0), dict(vocab=0), dict(ts=(1 << 40) + 1)):
        assert verify(lib, **kw) == 2, kw
    for kw in (dict(seqs=8193), dict(most=2049), dict(total=(1 << 30) + 1), dict(vocab=(1 << 28) + 1, ts=1 << 30, ds=1 << 30)):
        assert verify(lib, **kw) == 3, kw
    big = dict(vocab=100000, ts=100000, ds=100000)
    need = lib.tbn_verify_workspace_bytes(5, 3, 2, 100000)
    assert need > 0 and lib.tbn_verify_workspace_bytes(5, 3, 2, 0) == 0 and lib.tbn_verify_workspace_bytes(5, 3000, 2, 100000) == 0
    for ws, n in ((FAKE, need - 1), (None, need), (FAKE + 8, need)):
        assert verify(lib, ws=ws, n=n, **big) == 5


def test_queries_leave_the_last_error_alone(lib):  # noqa: F811
    assert verify(lib, cu=None) == 1
    text = lib.tbn_last_error()
    assert lib.tbn_kv4_attention_workspace_bytes(at(pool4(dim=48)), at(structs()[1]), 1, 5, 3, 4, 0, 0, 0, 0) == 0
    assert lib.tbn_window_attention_workspace_bytes(at(structs(pool_dim=12)[0]), at(structs()[1]), 5, 3, 4, 0, 5, 0, 0) == 0
    assert lib.tbn_verify_workspace_bytes(-1, 3, 2, 100000) == 0
    assert lib.tbn_last_error() == text


def test_binding_refuses_host_tensors():
    from paper_2407_12075_amd import kv
    z = torch.zeros
    with pytest.raises(ValueError):
        kv.KV4Pool(z(4, 2, 32, 16, dtype=torch.uint8), z(4, 2, 1, 4, 16, 2, 4, dtype=torch.uint8), z(4, 2, 32, 4, dtype=torch.int8), z(4, 2, 32, 4, dtype=torch.int8))
    with pytest.raises(ValueError):
        kv.KV4Pool(z(4, 2, 32, 16, dtype=torch.uint8), z(4, 2, 32, 16, dtype=torch.uint8), z(4, 2, 32, 4, dtype=torch.int8), z(4, 2, 32, 4, dtype=torch.int8))
    i = z(3, dtype=torch.int32)
    with pytest.raises(ValueError):
        kv.tbn_verify(z(2, 5), i, z(2), i, 2)


def rows_and_parts(lib, kind, T, window, n_seqs=1, heads=32, dim=128):  # noqa: F811
    """Stretches that a call's keys are split into, from the bytes of the workspace (0: not split)."""
    big = dict(n_pages=1 << 20, kv_heads=8, dim=dim, page=64)
    pool, index = structs(**{f"pool_{k}": v for k, v in big.items()}, pool_dt=1, index_page=64, index_n_pages=1 << 20, index_n_seqs=n_seqs, index_max_pages=2048)
    total = T * n_seqs
    if kind == "window":
        need = lib.tbn_window_attention_workspace_bytes(at(pool), at(index), total, T, heads, 4, window, 0, 20000)
    else:
        need = lib.tbn_kv4_attention_workspace_bytes(at(pool4(**big)), at(index), 1, total, T, heads, 4, window, 0, 20000)
    assert need % (total * heads * (dim + 4) * 4) == 0
    return need // (total * heads * (dim + 4) * 4)


def test_prompts_with_a_window_are_not_split(lib):  # noqa: F811
    """Rows fill the places: few keys stay whole once every CU has a tile of rows, many are split all the same."""
    for kind in ("window", "four"):
        assert [rows_and_parts(lib, kind, T, 1024) for T in (512, 700, 1024, 2048)] == [0] * 4
        assert rows_and_parts(lib, kind, 128, 4000) > 1 and rows_and_parts(lib, kind, 700, 16000) > 1
    # single tokens: one round of whole windows, two stretches beyond
    assert rows_and_parts(lib, "window", 1, 4096, n_seqs=64) == 0 and rows_and_parts(lib, "window", 1, 8000, n_seqs=80) == 2


def test_stretches_of_the_cache_in_4_bits(lib):  # noqa: F811
    """Short histories whole; one round of the places up to 1024 keys each; many sequences in stretches of about 1500 keys."""
    assert rows_and_parts(lib, "four", 1, 700) == 0
    assert 20 <= rows_and_parts(lib, "four", 1, 0) <= 96
    assert 11 <= rows_and_parts(lib, "four", 1, 0, n_seqs=64) <= 15
