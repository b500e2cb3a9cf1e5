"""Sizes of the attention's launches over the cache, on the CPU: what is beyond one launch is refused before anything is launched."""
import ctypes

from tests.test_kv_abi import FAKE, lib, structs  # noqa: F401  (lib is a fixture)


def test_more_workgroups_than_a_launch_has(lib):  # noqa: F811
    """2^30 queries in tiles of 8 and 1024 key heads are 2^37 workgroups, which end in 0 in 32 bits."""
    big = 1 << 62
    for dim, page, select in ((64, 64, 4), (128, 32, 100), (256, 128, 512)):
        p, i = structs(pool_kv_heads=1024, pool_dim=dim, pool_page=page, index_page=page, pool_dt=1)
        args = (ctypes.addressof(p), ctypes.addressof(i))
        n = 1 << 30
        assert lib.tbn_block_attention_workspace_bytes(*args, n, n, 4096, select) == 0   # queries share workgroups
        assert lib.tbn_block_attention(FAKE, 4096 * dim, FAKE, None, *args, FAKE, n, n, 4096, FAKE, select, 1.0, FAKE, big, None) == 3
        assert b"beyond one launch" in lib.tbn_last_error()


def parts(lib, total, max_q, n_seqs, dt=1, max_len=131000, heads=32):  # noqa: F811
    """Stretches that the keys of a sequence are split into, from the bytes of the workspace (0: not split)."""
    p, i = structs(pool_kv_heads=8, pool_dim=128, pool_page=64, index_page=64, pool_dt=dt, index_n_seqs=n_seqs, index_max_pages=2048, pool_n_pages=1 << 20, index_n_pages=1 << 20)
    need = lib.tbn_tree_attention_workspace_bytes(ctypes.addressof(p), ctypes.addressof(i), total, max_q, heads, max_len)
    assert need % (total * heads * (128 + 4) * 4) == 0
    return need // (total * heads * (128 + 4) * 4)


def test_keys_are_split_by_the_sequences_that_are_there(lib):  # noqa: F811
    """Places of the index that no token belongs to count for nothing."""
    for dt in (0, 1):
        for live, keys in ((1, 131000), (8, 9000), (3, 40000)):
            alone = parts(lib, live, 1, live, dt, keys)
            assert alone >= 4
            assert [parts(lib, live, 1, n, dt, keys) for n in (16, 64, 512, 8192)] == [alone] * 4
            # several tokens of each: never fewer than in an index that is full of them; bfloat16, some places: no fewer than half of the stretches
            alone = parts(lib, 26 * live, 26, live, dt, keys)
            assert all(parts(lib, 26 * live, 26, n, dt, keys) >= parts(lib, 26 * n, 26, n, dt, keys) for n in (16, 64, 512, 8192))
            assert dt == 0 or all(2 * parts(lib, 26 * live, 26, n, dt, keys) >= alone for n in (16, 64))
        # an index without idle places: as many as there are places, whether the drafts are of one length or ragged
        assert parts(lib, 16 * 26, 26, 16, dt) == parts(lib, 16 * 15, 26, 16, dt) > 1


def test_rounds_of_the_staged_kernel(lib):  # noqa: F811
    """Single tokens, 512 places for workgroups, 8 key heads: whole sequences that fill the places and are long are cut in two, fewer into as many as fit."""
    assert [parts(lib, 64, 1, 64, 1, n) for n in (3200, 4096, 4200, 16384)] == [0, 0, 2, 2]
    assert [parts(lib, 100, 1, 100, 1, n) for n in (2000, 6000)] == [0, 2]
    assert [parts(lib, n, 1, n, 1, 60000) for n in (16, 32)] == [4, 2]
