"""Trees with a window whose sequences have more tokens than the call's max_q: the first max_q tokens of each are served as if there were no others, and
everything that lies behind them, the workspace's neighbours among it, stays as it is."""
import math

import pytest
import torch

from tests.kv4_util import make_cache4
from tests.kv_util import compare, make_cache, make_queries, tolerance
from tests.test_kv_attention_gpu import masks
from tests.test_kv_window_gpu import packed, reference

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kv():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2407_12075_amd import kv as binding, tbn
    tbn.lib()
    return binding


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("H,KV,D,P,seqs,most,sink,window", [
    (8, 2, 128, 64, [(4000, 900)], 2, 4, 2500),                    # few rows, keys in stretches
    (8, 2, 64, 32, [(300, 1500), (2000, 3)], 3, 70, 2000),
    (8, 1, 128, 64, [(5000, 700), (40, 5)], 20, 4, 3000),          # the kernels that stage keys
    (16, 1, 64, 128, [(6000, 600)], 12, 0, 2048),
    (4, 2, 64, 32, [(100, 90), (5, 2)], 7, 3, 7)])                 # not split
def test_more_tokens_than_max_q(kv, H, KV, D, P, seqs, most, sink, window, four, dt):
    counts = [n for _, n in seqs]
    lens = [p + n for p, n in seqs]
    pool, index, keys, values = make_cache4(kv, KV, D, P, lens, seed=H) if four else make_cache(kv, dt, KV, D, P, lens, seed=H, garbage=1.0)
    q, cu, qs = make_queries(dt, counts, H, D)
    served = [min(n, most) for n in counts]
    see = masks("tree", served, 3)
    starts = [sum(counts[:s]) for s in range(len(counts))]
    rows = torch.tensor([t + i for t, n in zip(starts, served) for i in range(n)])
    mask = torch.zeros(sum(counts), -(-most // 32), dtype=torch.int32, device="cuda")
    mask[rows.cuda()] = packed(see, served)
    scale = 1 / math.sqrt(D)
    kw = dict(n_sink=sink, window=window, mask=mask, scale=scale)
    fn = kv.tbn_kv4_attention if four else kv.tbn_window_attention
    need = (kv.tbn_kv4_attention_workspace_bytes if four else kv.tbn_window_attention_workspace_bytes)(q, pool, index, most, sink, window, masked=True)
    assert (need > 0) == (window > 100)
    room = torch.full((need + 4096,), 255, dtype=torch.uint8, device="cuda")   # parts that were read behind the workspace would be not-a-number
    out, lse = torch.full_like(q, 7.0), torch.full((sum(counts), H), 7.0, device="cuda")
    fn(q, pool, index, cu, most, out=out, lse=lse, workspace=room[:need] if need else None, **kw)
    ref = reference(qs[rows.numpy()], [k[:p + n] for k, (p, _), n in zip(keys, seqs, served)], [v[:p + n] for v, (p, _), n in zip(values, seqs, served)], served, sink, window, see, scale)
    compare(out[rows.cuda()], lse[rows.cuda()], *ref, tolerance(dt, values))
    others = torch.ones(sum(counts), dtype=torch.bool)
    others[rows] = False
    assert bool((out[others.cuda()] == 7).all()) and bool((lse[others.cuda()] == 7).all())
    assert bool((room[need:] == 255).all())
