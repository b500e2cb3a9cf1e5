"""Every call of the cache's binding takes a pool of its own kind and an index, on the CPU: the structs of both pools have one size and the same fields but for
the last, and the library cannot tell them apart."""
import ctypes

import pytest
import torch

from tests.test_kv_abi import FAKE, lib, structs  # noqa: F401  (lib is a fixture)
from tests.test_kv_more_abi import pool4


def held(kind, struct, **fields):
    """An object of the binding's class without tensors."""
    x = object.__new__(kind)
    x._c, x._at, x._gpu, x._ws, x.device = struct, ctypes.addressof(struct), 0, 0, torch.device("cuda", 0)
    x.__dict__.update(fields)
    return x


@pytest.fixture()
def objects(lib):  # noqa: F811
    from paper_2407_12075_amd import kv
    pool, index = structs()
    sizes = dict(n_pages=10, kv_heads=2, dim=64, page=32)
    return (held(kv.KVPool, pool, dtype=torch.float32, **sizes), held(kv.KV4Pool, pool4(), dtype=None, **sizes),
            held(kv.KVIndex, index, n_pages=10, n_seqs=3, max_pages=4, page=32))


def calls(pool, index):
    """Calls of a pool in the types of the inputs, of one in 4 bits, and of the index alone."""
    from paper_2407_12075_amd import kv
    i, q, k = torch.zeros(9, dtype=torch.int32), torch.zeros(5, 4, 64), torch.zeros(5, 2, 64)
    both = lambda p, x: {  # noqa: E731
        "append": lambda: kv.tbn_kv_append(p, x, k, k, i, 3), "keep": lambda: kv.tbn_kv_keep(p, x, i, i.view(3, 3), i), "copy_pages": lambda: kv.tbn_kv_copy_pages(p, i, i),
        "tree": lambda: kv.tbn_tree_attention(q, p, x, i, 3), "tree bytes": lambda: kv.tbn_tree_attention_workspace_bytes(q, p, x, 3),
        "window": lambda: kv.tbn_window_attention(q, p, x, i, 3, 1, 5), "window bytes": lambda: kv.tbn_window_attention_workspace_bytes(q, p, x, 3, 1, 5),
        "select": lambda: kv.tbn_block_select(q, p, x, i, 3, 2), "select bytes": lambda: kv.tbn_block_select_workspace_bytes(q, p, x, 3),
        "picked": lambda: kv.tbn_block_attention(q, p, x, i, 3, i), "picked bytes": lambda: kv.tbn_block_attention_workspace_bytes(q, p, x, 3, 2)}
    four = lambda p, x: {  # noqa: E731
        "append": lambda: kv.tbn_kv4_append(p, x, k, k, i, 3), "read": lambda: kv.tbn_kv4_read(p, x, i, 3, 5), "keep": lambda: kv.tbn_kv4_keep(p, x, i, i.view(3, 3), i),
        "copy_pages": lambda: kv.tbn_kv4_copy_pages(p, i, i), "attend": lambda: kv.tbn_kv4_attention(q, p, x, i, 3),
        "bytes": lambda: kv.tbn_kv4_attention_workspace_bytes(q, p, x, 3)}
    alone = {"reserve": lambda: kv.tbn_kv_reserve(index, i), "fork": lambda: kv.tbn_kv_fork(index, i, i), "release": lambda: kv.tbn_kv_release(index, i),
             "compact": lambda: kv.tbn_kv_compact(index)}
    return both(pool, index), four(pool, index), alone


def refused(all_calls, message):
    for name, call in all_calls.items():
        with pytest.raises(ValueError, match=message):
            call()
            pytest.fail(name)


def test_the_structs_cannot_be_told_apart():
    from paper_2407_12075_amd import kv
    assert ctypes.sizeof(kv._Pool) == ctypes.sizeof(kv._Pool4) and [f for f, _ in kv._Pool._fields_[4:8]] == [f for f, _ in kv._Pool4._fields_[4:8]]


def test_pools_of_the_other_kind(objects):
    pool, four, index = objects
    refused(calls(four, index)[0], "must be a KVPool, got KV4Pool")
    refused(calls(pool, index)[1], "must be a KV4Pool, got KVPool")


def test_pools_and_indices_change_places(objects):
    pool, four, index = objects
    refused(calls(index, pool)[0], "pool must be a KVPool, got KVIndex")
    refused(calls(index, four)[1], "pool must be a KV4Pool, got KVIndex")
    refused({k: c for k, c in calls(pool, four)[0].items() if k != "copy_pages"}, "index must be a KVIndex, got KV4Pool")
    refused({k: c for k, c in calls(four, pool)[1].items() if k != "copy_pages"}, "index must be a KVIndex, got KVPool")
    for x in (pool, four):
        refused(calls(None, x)[2], "index must be a KVIndex, got KV")


def test_classes_made_from_them_pass(objects):
    """What a program derives from a pool or an index is one: the call gets as far as its tensors, which live in host memory."""
    from paper_2407_12075_amd import kv
    pool, four, index = objects
    more = [type("Mine", (kind,), {}) for kind in (kv.KVPool, kv.KV4Pool, kv.KVIndex)]
    for x, kind in zip(objects, more):
        x.__class__ = kind
    q = torch.zeros(5, 4, 64)
    assert kv.tbn_tree_attention_workspace_bytes(q, pool, index, 3) == kv.tbn_kv4_attention_workspace_bytes(q, four, index, 3) == 0
    refused({k: c for k, c in calls(pool, index)[0].items() if "bytes" not in k}, "device tensor|must live on")
    refused({k: c for k, c in calls(four, index)[1].items() if k not in ("bytes", "read")}, "device tensor|must live on")
