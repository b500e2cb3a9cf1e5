"""The cache's calls through the extension module leave the interpreter to other threads while the library works: the library's entry points
are replaced by a function that waits, for a bounded time, until another Python thread has run.  Nothing is launched."""
import ctypes
import subprocess
import threading
import time

import pytest
import torch

pytestmark = pytest.mark.gpu

# 0 (TBN_OK) once `go` is set, 4 (TBN_ERR_DEVICE) if that takes two seconds
WAIT = r"""
#include <atomic>
#include <chrono>
#include <thread>
extern "C" {
std::atomic<int> inside{0}, go{0};
int wait_for_go() {
    const auto until = std::chrono::steady_clock::now() + std::chrono::seconds(2);
    inside = 1;
    while (!go && std::chrono::steady_clock::now() < until) std::this_thread::yield();
    return go ? 0 : 4;
}
}
"""

LAUNCHES = ("tbn_kv_reserve", "tbn_kv_fork", "tbn_kv_release", "tbn_kv_copy_pages", "tbn_kv_append", "tbn_kv_keep", "tbn_tree_attention", "tbn_block_select",
            "tbn_block_attention")


def test_other_threads_run_during_a_call(tmp_path, monkeypatch):
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2407_12075_amd import kv, tbn
    real = tbn.lib()
    host = tbn._host
    assert host is not None
    src, so = tmp_path / "wait.cpp", tmp_path / "wait.so"
    src.write_text(WAIT)
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", str(src), "-o", str(so)], check=True)
    wait = ctypes.CDLL(str(so))
    inside, go = ctypes.c_int.in_dll(wait, "inside"), ctypes.c_int.in_dll(wait, "go")

    ints = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    pool, index = kv.kv_pool(8, 1, 64, 32, torch.float32, summary=True), kv.kv_index(2, 4, 8, 32)
    q, new, cu, picks = (torch.zeros(2, 2, 64, device="cuda"), torch.zeros(2, 1, 64, device="cuda"), ints(0, 1, 2), torch.zeros(2, 1, 1, dtype=torch.int32, device="cuda"))
    calls = {
        "reserve": lambda: kv.tbn_kv_reserve(index, ints(1, 1)), "fork": lambda: kv.tbn_kv_fork(index, ints(0), ints(1)),
        "release": lambda: kv.tbn_kv_release(index, ints(0, 0)), "copy_pages": lambda: kv.tbn_kv_copy_pages(pool, ints(0), ints(1)),
        "append": lambda: kv.tbn_kv_append(pool, index, new, new, cu, 1), "keep": lambda: kv.tbn_kv_keep(pool, index, ints(0, 0), ints(0, 0).view(2, 1), ints(1, 1)),
        "tree": lambda: kv.tbn_tree_attention(q, pool, index, cu, 1), "select": lambda: kv.tbn_block_select(q, pool, index, cu, 1, 2),
        "picked": lambda: kv.tbn_block_attention(q, pool, index, cu, 1, picks),
    }
    assert len(calls) == len(LAUNCHES)
    torch.cuda.synchronize()

    class NoOtherWay:   # the wrappers' own path goes through ctypes and would not show it
        def __getattr__(self, name):
            f = getattr(real, name)
            assert name not in LAUNCHES, name
            return f

    names = [n for n in ("tbn_pack_workspace_bytes", "tbn_pack_tile", "tbn_linear_forward", "tbn_conv2d_forward", "tbn_sign_pack", "tbn_linear_coltiled_workspace_bytes",
                         "tbn_linear_coltiled_forward", "tbn_linear_forward_binact", "tbn_kv_workspace_bytes", "tbn_tree_attention_workspace_bytes",
                         "tbn_block_select_workspace_bytes", "tbn_block_attention_workspace_bytes") + LAUNCHES]
    address = lambda f: ctypes.cast(f, ctypes.c_void_p).value  # noqa: E731
    monkeypatch.setattr(tbn, "lib", lambda: NoOtherWay())
    try:
        host.init(tbn._raise, {n: address(wait.wait_for_go) if n in LAUNCHES else address(getattr(real, n)) for n in names})
        for name, call in calls.items():
            inside.value = go.value = 0

            def other():
                until = time.monotonic() + 10
                while not inside.value and time.monotonic() < until:
                    time.sleep(0.001)
                go.value = 1
            t = threading.Thread(target=other)
            t.start()
            call()   # raises where nobody set `go`
            t.join()
            assert inside.value, name
    finally:
        host.init(tbn._raise, {n: address(getattr(real, n)) for n in names})
    monkeypatch.undo()
    torch.cuda.synchronize()
    assert not index.lens.any() and not index.refs.any()
    kv.tbn_kv_release(index, ints(0, 0))   # the library's own again
    torch.cuda.synchronize()
