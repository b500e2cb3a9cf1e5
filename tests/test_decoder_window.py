"""A tree of drafts that the model's window does not hold is refused before a key of it enters the cache."""
import pytest
import torch

from paper_2407_12075_amd.decoder import Decoder, DecoderConfig

SMALL = dict(layers=1, heads=2, kv_heads=1, dim=64, hidden=128, vocab=64, page=32, max_len=256, n_seqs=2)


@pytest.mark.parametrize("four_bit", [False, True])
def test_refused_before_anything(four_bit):
    model = object.__new__(Decoder)
    model.cfg, model.index, model.device = DecoderConfig(window=6, four_bit=four_bit, **SMALL), None, torch.device("cpu")
    with pytest.raises(ValueError, match="window of 6 .* tree of 7"):
        model.step(torch.zeros(2, dtype=torch.int64), depth=3)


@pytest.mark.gpu
@pytest.mark.parametrize("four_bit", [False, True])
def test_the_cache_stays_as_it_is(four_bit):
    model = Decoder(DecoderConfig(window=6, four_bit=four_bit, **SMALL))
    last = model.prompt(torch.arange(40, device="cuda"), 2)
    before = [t.clone() for t in (model.index.table, model.index.lens, model.index.refs)]
    for temperature in (0.0, 1.0):
        with pytest.raises(ValueError):
            model.step(last, depth=3, temperature=temperature)
    assert all(torch.equal(a, b) for a, b in zip(before, (model.index.table, model.index.lens, model.index.refs)))
    tokens, counts = model.step(last, depth=2)
    assert tokens.shape == (2, 3) and bool((model.index.lens == before[1] + counts).all())
    model.step(last, depth=0)
    model.check()
