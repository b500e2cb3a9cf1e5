"""The newer calls through the extension module, through the wrappers' own code and bound once: one result; what the module does not take, the wrappers do."""
import numpy as np
import pytest
import torch

from tests.kv4_util import make_cache4
from tests.kv_util import make_cache, make_queries

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kv():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2407_12075_amd import kv as binding, tbn
    tbn.lib()
    assert tbn._host is not None
    return binding


def calls(kv):
    """Name -> a function that makes the call and returns all that it changed or gave back; every call begins from the same state."""
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    pool, index, _, _ = make_cache(kv, "bf16", 2, 64, 32, [70, 900], seed=1)
    four, index4, _, _ = make_cache4(kv, 2, 64, 32, [70, 900], seed=2)
    before = [t.clone() for t in (four.k, four.v, four.k_exp, four.v_exp)]
    q, cu, _ = make_queries("bf16", [3, 1], 8, 64, stride=8 * 64 + 3)
    mask = ints(1, 3, 5, 1).view(4, 1)
    new = torch.randn(4, 6, 64, device="cuda")
    probs = torch.softmax(torch.randn(4, 20000, device="cuda"), 1)
    draft = torch.softmax(torch.randn(4, 20000, device="cuda"), 1)
    tokens, u, parents = ints(0, 5, 6, 0), torch.rand(4, device="cuda"), ints(-1, 0, 0, -1)

    def reset():
        for t, b in zip((four.k, four.v, four.k_exp, four.v_exp), before):
            t.copy_(b)

    state = lambda _: [four.k, four.v, four.k_exp, four.v_exp]  # noqa: E731
    give = lambda r: list(r)  # noqa: E731
    return reset, {
        "window": (kv.tbn_window_attention, (q, pool, index, cu, 3, 4, 500), {}, give),
        "window, tree": (kv.tbn_window_attention, (q, pool, index, cu, 3, 4, 50), dict(mask=mask, scale=0.2, max_len=900), give),
        "four": (kv.tbn_kv4_attention, (q, four, index4, cu, 3), {}, give),
        "four, float32, window, tree": (kv.tbn_kv4_attention, (q.float(), four, index4, cu, 3), dict(mask=mask, n_sink=3, window=70, scale=0.2, max_len=900), give),
        "append": (kv.tbn_kv4_append, (four, index4, new[:, 1:3], new[:, 3:5], cu, 3), {}, state),
        "read": (kv.tbn_kv4_read, (four, index4, cu, 3, 4), {}, give),
        "read float32": (kv.tbn_kv4_read, (four, index4, cu, 3, 4, torch.float32), {}, give),
        "copy": (kv.tbn_kv4_copy_pages, (four, ints(1, 2, -1), ints(4, 0, 3)), {}, state),
        "copy some": (kv.tbn_kv4_copy_pages, (four, ints(1, 2), ints(4, 0), ints(1)), {}, state),
        "keep": (kv.tbn_kv4_keep, (four, index4, ints(60, 800), ints(1, 3, 5, 2, 9, 30).view(2, 3), ints(3, 2)), {}, state),
        "verify": (kv.tbn_verify, (probs, tokens, u, cu, 3), dict(draft=draft, parents=parents), give),
        "verify a chain": (kv.tbn_verify, (probs[:, :500], tokens, u, cu, 5), {}, give),
    }


def test_three_ways_one_result(kv, monkeypatch):
    from paper_2407_12075_amd import tbn
    reset, all_calls = calls(kv)
    for name, (fn, args, kw, after) in all_calls.items():
        reset()
        plain = [t.clone() for t in after(fn(*args, **kw))]
        reset()
        with monkeypatch.context() as m:
            m.setattr(tbn, "_host", None)
            wrapped = [t.clone() for t in after(fn(*args, **kw))]
        reset()
        bound = tbn.tbn_bind(fn, *args, **kw)
        for _ in range(2):
            reset()
            again = [t.clone() for t in after(bound())]
        torch.cuda.synchronize()
        for a, b, c in zip(plain, wrapped, again):
            assert torch.equal(a, b) and torch.equal(a, c), name


def test_the_module_takes_the_plain_form(kv, monkeypatch):
    """Without the wrappers' own way to the library every plain call still works."""
    from paper_2407_12075_amd import tbn
    reset, all_calls = calls(kv)
    monkeypatch.setattr(kv, "_call", None)
    for name, (fn, args, kw, after) in all_calls.items():
        fn(*args, **kw)
    torch.cuda.synchronize()


@pytest.mark.parametrize("own", [False, True])
def test_errors_are_the_librarys(kv, own, monkeypatch):
    from paper_2407_12075_amd import tbn
    if own:
        monkeypatch.setattr(tbn, "_host", None)
    _, all_calls = calls(kv)
    pool, index = all_calls["window"][1][1:3]
    q, four, index4, cu = all_calls["four"][1][:4]
    for call in (lambda: kv.tbn_window_attention(q[:, :3].contiguous(), pool, index, cu, 3, 0, 5), lambda: kv.tbn_window_attention(q, pool, index, cu, 3, 0, 0),
                 lambda: kv.tbn_kv4_attention(q, four, index4, cu, 3, max_len=10 ** 6), lambda: kv.tbn_verify(*all_calls["verify"][1][:4], 2049)):
        with pytest.raises(tbn.TbnError):
            call()


def test_no_tokens_at_all(kv):
    _, all_calls = calls(kv)
    four, index4 = all_calls["four"][1][1:3]
    none = torch.zeros(3, dtype=torch.int32, device="cuda")
    q = torch.zeros(0, 8, 64, dtype=torch.bfloat16, device="cuda")
    out, lse = kv.tbn_kv4_attention(q, four, index4, none, 0)
    assert out.shape == q.shape and lse.shape == (0, 8)
    k = torch.zeros(0, 2, 64, device="cuda")
    kv.tbn_kv4_append(four, index4, k, k, none, 0)
    a, b = kv.tbn_kv4_read(four, index4, none, 0, 0)
    assert a.shape == b.shape == (0, 2, 64)
    picks, counts, follows = kv.tbn_verify(torch.zeros(0, 9, device="cuda"), none[:0], torch.zeros(0, device="cuda"), none, 4)
    assert picks.tolist() == [[-1] * 4] * 2 and counts.tolist() == [0, 0] and follows.tolist() == [-1, -1]
    assert np.prod(picks.shape) == 8
