"""A window beyond 32 bits is no window; what has to be at least a number may be any."""
import math

import pytest
import torch

from tests.kv4_util import make_cache4
from tests.kv_util import compare, make_cache, make_queries, tolerance
from tests.test_kv_window_gpu import reference

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kv():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2407_12075_amd import kv as binding, tbn
    tbn.lib()
    return binding


@pytest.mark.parametrize("own", [False, True])
def test_large_integers(kv, own, monkeypatch):
    from paper_2407_12075_amd import tbn
    if own:
        monkeypatch.setattr(tbn, "_host", None)
    counts, far = [3, 1], 1 << 32
    pool, index, keys, values = make_cache(kv, "f32", 2, 64, 32, [400, 90], seed=7)
    four, index4, keys4, values4 = make_cache4(kv, 2, 64, 32, [400, 90], seed=8)
    q, cu, qs = make_queries("f32", counts, 8, 64)
    scale = 1 / math.sqrt(64)
    all_keys = reference(qs, keys, values, counts, 0, 1 << 30, None, scale)
    for most, sink, window in ((3, 0, far + 64), (far + 1, 0, far + 64), (3, far + 2, 5), (1 << 70, 0, 1 << 70)):
        compare(*kv.tbn_window_attention(q, pool, index, cu, most, sink, window), *all_keys, tolerance("f32", values))
        compare(*kv.tbn_kv4_attention(q, four, index4, cu, most, n_sink=sink, window=window), *reference(qs, keys4, values4, counts, 0, 1 << 30, None, scale), tolerance("f32", values4))
    compare(*kv.tbn_tree_attention(q, pool, index, cu, far + 1), *all_keys, tolerance("f32", values))
    for sink, window in ((-far + 1, 5), (0, -far + 5)):
        for call in (lambda: kv.tbn_window_attention(q, pool, index, cu, 3, sink, window), lambda: kv.tbn_kv4_attention(q, four, index4, cu, 3, n_sink=sink, window=window)):
            with pytest.raises(tbn.TbnError) as e:
                call()
            assert e.value.status == 2
    new = torch.randn(4, 2, 64, device="cuda")
    kv.tbn_kv4_append(four, index4, new, new, cu, far + 1)
    got, _ = kv.tbn_kv4_read(four, index4, cu, far + 1, 4, torch.float32)
    want = [t.clone() for t in (four.k, four.v, four.k_exp, four.v_exp)]
    kv.tbn_kv4_append(four, index4, new, new, cu, 3)
    assert all(torch.equal(a, b) for a, b in zip(want, (four.k, four.v, four.k_exp, four.v_exp)))
    assert torch.equal(got, kv.tbn_kv4_read(four, index4, cu, 3, 4, torch.float32)[0])
