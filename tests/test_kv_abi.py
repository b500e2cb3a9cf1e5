"""Refusals of the cache's entry points, on the CPU: validation runs before any device call and leaves everything alone."""
import ctypes

import pytest
import torch


@pytest.fixture(scope="module")
def lib():
    import os
    from paper_2407_12075_amd import build, tbn
    if not os.path.exists(build.LIB):
        build.build(verbose=False)
    return tbn.lib()


FAKE = 4096   # never dereferenced


def structs(**changes):
    from paper_2407_12075_amd import kv
    pool = dict(k=FAKE, v=FAKE, summary=FAKE, step=FAKE, n_pages=10, kv_heads=2, dim=64, page=32, dt=0)
    index = dict(table=FAKE, lens=FAKE, refs=FAKE, status=FAKE, n_pages=10, n_seqs=3, max_pages=4, page=32)
    for name, value in changes.items():
        part, field = name.split("_", 1)
        (pool if part == "pool" else index)[field] = value
    return kv._Pool(**pool), kv._Index(**index)


def refs(**changes):
    p, i = structs(**changes)
    refs.keep = (p, i)
    return ctypes.addressof(p), ctypes.addressof(i)


def calls(lib, p, i):
    """Every entry point with arguments that pass, but for what the structs hold; those with index only, pool only, both."""
    big = 1 << 30
    index_only = {
        "reserve": lambda: lib.tbn_kv_reserve(i, FAKE, FAKE, FAKE, FAKE, big, None),
        "fork": lambda: lib.tbn_kv_fork(i, FAKE, FAKE, 2, None),
        "release": lambda: lib.tbn_kv_release(i, FAKE, None),
        "compact": lambda: lib.tbn_kv_compact(i, FAKE, FAKE, FAKE, FAKE, big, None),
    }
    pool_only = {"copy_pages": lambda: lib.tbn_kv_copy_pages(p, FAKE, FAKE, 2, None, None)}
    both = {
        "append": lambda: lib.tbn_kv_append(p, i, FAKE, 128, FAKE, 128, FAKE, 5, 3, None),
        "keep": lambda: lib.tbn_kv_keep(p, i, FAKE, FAKE, 2, FAKE, None),
        "tree": lambda: lib.tbn_tree_attention(FAKE, 512, FAKE, FAKE, p, i, FAKE, 5, 3, 4, None, 0, 0, 1.0, FAKE, big, None),
        "select": lambda: lib.tbn_block_select(FAKE, 512, FAKE, p, i, FAKE, 5, 3, 4, 2, 0, 1, 0, FAKE, big, None),
        "attend": lambda: lib.tbn_block_attention(FAKE, 512, FAKE, FAKE, p, i, FAKE, 5, 3, 4, FAKE, 2, 1.0, FAKE, big, None),
    }
    return index_only, pool_only, both


@pytest.mark.parametrize("field,value,status", [
    ("table", None, 1), ("lens", None, 1), ("refs", None, 1), ("status", None, 1), ("n_seqs", 0, 2), ("max_pages", 0, 2), ("n_pages", 0, 2), ("page", 0, 2),
    ("page", 48, 3), ("page", 16, 3), ("n_seqs", 8193, 3), ("max_pages", 1 << 26, 3), ("n_pages", 1 << 31, 3)])
def test_index_is_checked_everywhere(lib, field, value, status):
    p, i = refs(**{f"index_{field}": value})
    index_only, _, both = calls(lib, p, i)
    for name, call in {**index_only, **both}.items():
        assert call() == status, name
        assert lib.tbn_last_error().decode().startswith("tbn_"), name


@pytest.mark.parametrize("field,value,status", [
    ("k", None, 1), ("v", None, 1), ("step", None, 1), ("summary", None, 1), ("n_pages", 0, 2), ("kv_heads", 0, 2), ("dim", 0, 2), ("page", 0, 2),
    ("dim", 12, 3), ("dim", 264, 3), ("page", 256, 3), ("kv_heads", 1025, 3), ("dt", 2, 3), ("k", FAKE + 8, 3), ("v", FAKE + 4, 3), ("summary", FAKE + 8, 3)])
def test_pool_is_checked_everywhere(lib, field, value, status):
    p, i = refs(**{f"pool_{field}": value})
    _, pool_only, both = calls(lib, p, i)
    for name, call in {**pool_only, **both}.items():
        assert call() == status, name


def test_pool_and_index_agree(lib):
    for change in (dict(pool_page=64), dict(pool_n_pages=11)):
        p, i = refs(**change)
        for name, call in calls(lib, p, i)[2].items():
            assert call() == 2, name


def test_null_structs(lib):
    p, i = refs()
    index_only, pool_only, both = calls(lib, None, None)
    for name, call in {**index_only, **pool_only, **both}.items():
        assert call() == 1, name
    for name, call in calls(lib, p, None)[2].items():
        assert call() == 1, name


def test_arguments(lib):
    p, i = refs()
    big = 1 << 30
    assert lib.tbn_kv_reserve(i, None, FAKE, FAKE, FAKE, big, None) == 1
    assert lib.tbn_kv_reserve(i, FAKE, FAKE, FAKE, None, big, None) == 5
    assert lib.tbn_kv_reserve(i, FAKE, FAKE, FAKE, FAKE, 43, None) == 5
    assert lib.tbn_kv_workspace_bytes(10, 3) == 44 and lib.tbn_kv_workspace_bytes(0, 3) == 0 and lib.tbn_kv_workspace_bytes(10, 9000) == 0
    assert lib.tbn_kv_fork(i, FAKE, FAKE, 4, None) == 2 and lib.tbn_kv_fork(i, FAKE, FAKE, -1, None) == 2
    assert lib.tbn_kv_fork(i, None, FAKE, 1, None) == 1 and lib.tbn_kv_fork(i, None, None, 0, None) == 0
    assert lib.tbn_kv_release(i, None, None) == 1
    assert lib.tbn_kv_compact(i, FAKE, FAKE, None, FAKE, big, None) == 1 and lib.tbn_kv_compact(i, FAKE, FAKE, FAKE, FAKE + 2, big, None) == 5
    assert lib.tbn_kv_copy_pages(p, FAKE, None, 1, None, None) == 1 and lib.tbn_kv_copy_pages(p, FAKE, FAKE, -1, None, None) == 2
    assert lib.tbn_kv_copy_pages(p, None, None, 0, None, None) == 0
    assert lib.tbn_kv_append(p, i, FAKE, 127, FAKE, 128, FAKE, 5, 3, None) == 2
    assert lib.tbn_kv_append(p, i, FAKE, 128, FAKE, 128, None, 5, 3, None) == 1
    assert lib.tbn_kv_append(p, i, FAKE, 128, FAKE, 128, FAKE, -1, 3, None) == 2
    assert lib.tbn_kv_append(p, i, None, 0, None, 0, None, 0, 0, None) == 0
    assert lib.tbn_kv_keep(p, i, FAKE, FAKE, -1, FAKE, None) == 2 and lib.tbn_kv_keep(p, i, FAKE, None, 1, FAKE, None) == 1
    assert lib.tbn_kv_keep(p, i, None, None, 0, None, None) == 0

    def tree(q=FAKE, stride=512, out=FAKE, cu=FAKE, total=5, most=3, heads=4, mask=None, words=0, max_len=0, ws=FAKE, size=big):
        return lib.tbn_tree_attention(q, stride, out, None, p, i, cu, total, most, heads, mask, words, max_len, 1.0, ws, size, None)
    assert tree(q=None) == 1 and tree(out=None) == 1 and tree(cu=None) == 1
    assert tree(stride=255) == 2 and tree(total=-1) == 2 and tree(most=-1) == 2 and tree(heads=3) == 2 and tree(heads=0) == 2
    assert tree(max_len=129) == 2 and tree(max_len=-1) == 2 and tree(mask=FAKE, words=0) == 2
    assert tree(total=0, q=None, out=None, cu=None) == 0 and tree(most=0, q=None) == 0
    need = lib.tbn_tree_attention_workspace_bytes(p, i, 5, 3, 4, 0)
    assert need == 0      # 128 keys: not split
    p2, i2 = refs(index_max_pages=400)
    need = lib.tbn_tree_attention_workspace_bytes(p2, i2, 5, 3, 4, 0)
    assert need > 0 and lib.tbn_tree_attention_workspace_bytes(p2, i2, 5, 3, 5, 0) == 0
    for ws, size in ((FAKE, need - 1), (None, need), (FAKE + 8, need)):
        assert lib.tbn_tree_attention(FAKE, 512, FAKE, None, p2, i2, FAKE, 5, 3, 4, None, 0, 0, 1.0, ws, size, None) == 5

    p, i = refs()

    def select(n=2, sink=0, recent=1, heads=4, picks=FAKE):
        return lib.tbn_block_select(FAKE, 64 * max(heads, 1), picks, p, i, FAKE, 5, 3, heads, n, sink, recent, 0, FAKE, big, None)
    assert select(n=0) == 2 and select(sink=-1) == 2 and select(recent=0) == 2 and select(sink=2) == 2 and select(n=4097) == 3
    assert select(heads=258) == 3 and select(picks=None) == 1
    q, j = refs(pool_summary=None, pool_step=None)
    assert lib.tbn_block_select(FAKE, 512, FAKE, q, j, FAKE, 5, 3, 4, 2, 0, 1, 0, FAKE, big, None) == 1
    p, i = refs()
    assert lib.tbn_block_attention(FAKE, 512, FAKE, None, p, i, FAKE, 5, 3, 4, None, 2, 1.0, FAKE, big, None) == 1
    assert lib.tbn_block_attention(FAKE, 512, FAKE, None, p, i, FAKE, 5, 3, 4, FAKE, 0, 1.0, FAKE, big, None) == 2
    assert lib.tbn_block_attention(FAKE, 512, FAKE, None, p, i, FAKE, 5, 3, 4, FAKE, 5000, 1.0, FAKE, big, None) == 3


def test_queries_leave_the_last_error_alone(lib):
    p, i = refs()
    assert lib.tbn_kv_release(i, None, None) == 1
    text = lib.tbn_last_error()
    bad, j = refs(pool_dim=12)
    assert lib.tbn_tree_attention_workspace_bytes(bad, j, 5, 3, 4, 0) == 0
    assert lib.tbn_block_select_workspace_bytes(bad, j, 5, 3, 4, 0) == 0
    assert lib.tbn_block_attention_workspace_bytes(bad, j, 5, 3, 4, 2) == 0
    assert lib.tbn_last_error() == text


def test_binding_refuses_host_tensors_and_wrong_shapes():
    from paper_2407_12075_amd import kv
    z = torch.zeros
    with pytest.raises(ValueError):
        kv.KVPool(z(4, 2, 32, 8), z(4, 2, 8, 32))
    with pytest.raises(ValueError):
        kv.KVPool(z(4, 2, 32, 8), z(4, 2, 32, 8))
    with pytest.raises(ValueError):
        kv.KVPool(z(4, 2, 32, 8), z(4, 2, 8, 32), summary=z(4, 2, 2, 8, dtype=torch.int8))
    i = lambda *s: z(s, dtype=torch.int32)  # noqa: E731
    with pytest.raises(ValueError):
        kv.KVIndex(i(2, 3), i(2), i(4), i(1), 32)
    with pytest.raises(ValueError):
        kv.KVIndex(i(2, 3), i(3), i(4), i(1), 32)
