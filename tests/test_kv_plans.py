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
