"""Calls on a stream that is not the current one: what a wrapper allocates for itself comes from the call's stream, so that neither a dropped
workspace nor a block that the current stream still uses is written by both."""
import pytest
import torch

from tests.kv_util import make_cache, make_queries

pytestmark = pytest.mark.gpu

H, KV, D, P = 8, 2, 64, 32


@pytest.fixture(scope="module")
def lib():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2407_12075_amd import kv, tbn
    tbn.lib()
    return tbn, kv


def ints(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def calls(tbn, kv):
    """Name -> call(**more) of every wrapper that allocates, each on tensors that are there already."""
    gen = torch.Generator().manual_seed(3)
    x = torch.randn(6, 128, generator=gen).cuda()
    w = torch.randn(64, 128, generator=gen).cuda()
    tile, alpha = tbn.tbn_pack_tile(w, 4)
    col_tile, col_alpha = tbn.tbn_pack_coltile(w, 4)
    image, cw = torch.randn(2, 8, 6, 6, generator=gen).cuda(), torch.randn(16, 8 * 9, generator=gen).cuda()
    c_tile, c_alpha = tbn.tbn_pack_tile(cw, 4)
    bits = tbn.tbn_sign_pack(x)
    pool, index, _, _ = make_cache(kv, "bf16", KV, D, P, [3000, 900], seed=12, summary=True)
    pool.summary.fill_(1)
    pool.step.fill_(1.0)
    q, cu, _ = make_queries("bf16", [1, 1], H, D)
    picks = kv.tbn_block_select(q, pool, index, cu, 1, 40)
    assert kv.tbn_tree_attention_workspace_bytes(q, pool, index, 1) and kv.tbn_block_attention_workspace_bytes(q, pool, index, 1, 40)
    table, lens, refs, status = (t.clone() for t in (index.table, index.lens, index.refs, index.status))
    back = lambda: [a.copy_(b) for a, b in zip((index.table, index.lens, index.refs, index.status), (table, lens, refs, status))]  # noqa: E731
    none = ints(0, 0)
    return back, {
        "pack_tile": lambda **m: tbn.tbn_pack_tile(w, 4, **m),
        "pack_coltile": lambda **m: tbn.tbn_pack_coltile(w, 4, **m),
        "linear": lambda **m: tbn.tbn_linear_forward(x, tile, alpha, 64, 4, **m),
        "linear_ws": lambda **m: tbn.tbn_linear_forward_ws(x, tile, alpha, 64, 4, None, **m),
        "coltiled": lambda **m: tbn.tbn_linear_coltiled_forward(x, col_tile, col_alpha, 64, 4, **m),
        "conv": lambda **m: tbn.tbn_conv2d_forward(image, c_tile, c_alpha, 16, 3, 3, 4, pad=(1, 1), **m),
        "sign_pack": lambda **m: tbn.tbn_sign_pack(x, **m),
        "binact": lambda **m: tbn.tbn_linear_forward_binact(bits, 128, tile, alpha, 64, 4, **m),
        "reserve": lambda **m: kv.tbn_kv_reserve(index, none, **m),
        "compact": lambda **m: kv.tbn_kv_compact(index, **m)[2],
        "tree": lambda **m: kv.tbn_tree_attention(q, pool, index, cu, 1, **m),
        "select": lambda **m: kv.tbn_block_select(q, pool, index, cu, 1, 40, **m),
        "picked": lambda **m: kv.tbn_block_attention(q, pool, index, cu, 1, picks, **m),
    }


def tensors(r):
    return list(r) if isinstance(r, tuple) else [r]


@pytest.mark.parametrize("form", ["stream", "handle"])
def test_memory_is_the_streams(lib, monkeypatch, form):
    back, every = calls(*lib)
    side = torch.cuda.Stream()
    given = side if form == "stream" else side.cuda_stream
    real, taken = torch.empty, []

    def empty(*args, **kw):
        taken.append(torch.cuda.current_stream().cuda_stream)
        return real(*args, **kw)
    for name, call in every.items():
        back()
        want = [t.clone() for t in tensors(call())]
        back()
        torch.cuda.synchronize()
        taken.clear()
        with monkeypatch.context() as m:
            m.setattr(torch, "empty", empty)
            got = call(stream=given)
        side.synchronize()
        assert taken and all(s == side.cuda_stream for s in taken), name
        assert all(torch.equal(a, b) for a, b in zip(tensors(got), want)), name
        # on the current stream, named or not, nothing changes
        back()
        taken.clear()
        with monkeypatch.context() as m:
            m.setattr(torch, "empty", empty)
            got = call(stream=torch.cuda.current_stream())
        assert all(s == torch.cuda.current_stream().cuda_stream for s in taken), name
        assert all(torch.equal(a, b) for a, b in zip(tensors(got), want)), name


def test_blocks_are_not_shared_with_the_current_stream(lib):
    """The other stream is late: the current one allocates and writes meanwhile.  Then the current one is late and drops blocks that it has yet to write."""
    back, every = calls(*lib)
    side = torch.cuda.Stream()
    for name in ("tree", "picked", "select", "reserve", "compact", "pack_tile", "coltiled"):
        call = every[name]
        back()
        want = [t.clone() for t in tensors(call())]
        back()
        sizes = [1 << s for s in range(9, 21)]
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(4_000_000)
        got = call(stream=side)
        for n in sizes * 2:
            torch.empty(n, dtype=torch.uint8, device="cuda").fill_(0xff)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(tensors(got), want)), name
        del got
        back()
        torch.cuda.synchronize()
        torch.cuda._sleep(4_000_000)
        blocks = [torch.empty(n, dtype=torch.uint8, device="cuda").fill_(0xff) for n in sizes * 2]
        del blocks
        got = call(stream=side)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(tensors(got), want)), name
