"""Verifications of more tokens or sequences than there may be, on the CPU: the library's error, before any memory is asked for."""
import pytest
import torch

from tests.test_kv_abi import FAKE, lib  # noqa: F401  (lib is a fixture)


@pytest.mark.parametrize("most,seqs,vocab", [(2049, 2, 50), (1 << 30, 2, 50), (1 << 70, 3, 100000), (5, 8193, 50), (2048, 1 << 20, 100000)])
def test_nothing_is_allocated(lib, most, seqs, vocab, monkeypatch):  # noqa: F811
    from paper_2407_12075_amd import kv, tbn
    asked = []

    def empty(shape, *a, **kw):
        asked.append(shape)
        return torch.empty(0, dtype=torch.int32)

    monkeypatch.setattr(tbn, "_host", None)
    monkeypatch.setattr(kv, "_empty", empty)
    monkeypatch.setattr(kv, "_dev", lambda *a: FAKE)
    monkeypatch.setattr(kv, "_probabilities", lambda *a: (FAKE, vocab))
    monkeypatch.setattr(kv, "_stream", lambda s: None)
    target, i = torch.empty(5, 1).expand(5, vocab), torch.zeros(5, dtype=torch.int32)
    cu = torch.zeros(1, dtype=torch.int32).expand(seqs + 1)
    with pytest.raises(tbn.TbnError) as e:
        kv.tbn_verify(target, i, torch.zeros(5), cu, most)
    assert e.value.status == 3
    assert all(torch.Size([s] if isinstance(s, int) else s).numel() == 0 for s in asked), asked


def test_the_limits_are_the_librarys(lib):  # noqa: F811
    from paper_2407_12075_amd import kv
    ask = lambda most, seqs: lib.tbn_verify(None, 9, None, 9, None, None, None, None, 5, most, seqs, 9, None, None, None, None, 0, None)  # noqa: E731
    assert ask(kv.VERIFY_MAX_TOKENS, kv.MAX_SEQUENCES) == 1   # sizes pass, the pointers do not
    assert ask(kv.VERIFY_MAX_TOKENS + 1, kv.MAX_SEQUENCES) == ask(kv.VERIFY_MAX_TOKENS, kv.MAX_SEQUENCES + 1) == 3


@pytest.mark.gpu
@pytest.mark.parametrize("own", [False, True])
def test_on_the_gpu(own, monkeypatch):
    """2^30 places for each of two sequences would be 8 GiB."""
    from paper_2407_12075_amd import kv, tbn
    tbn.lib()
    if own:
        monkeypatch.setattr(tbn, "_host", None)
    p = torch.softmax(torch.randn(5, 50, device="cuda"), 1)
    i, cu = torch.zeros(5, dtype=torch.int32, device="cuda"), torch.tensor([0, 3, 5], dtype=torch.int32, device="cuda")
    u = torch.rand(5, device="cuda")
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.memory_allocated()
    for most, c in ((1 << 30, cu), (2049, cu), (3, torch.zeros(8194, dtype=torch.int32, device="cuda"))):
        with pytest.raises(tbn.TbnError) as e:
            kv.tbn_verify(p, i, u, c, most)
        assert e.value.status == 3
    assert torch.cuda.max_memory_allocated() < before + (1 << 20)
    replay = tbn.tbn_bind(kv.tbn_verify, p, i, u, cu, 1 << 30)   # marshalled all the same: the call raises
    with pytest.raises(tbn.TbnError):
        replay()
    assert kv.tbn_verify(p, i, u, cu, 2048)[0].shape == (2, 2048)
