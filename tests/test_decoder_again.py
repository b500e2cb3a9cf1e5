"""The example decoder with one prompt after another."""
import pytest
import torch


@pytest.mark.gpu
@pytest.mark.parametrize("copies,depth", [(1, 0), (3, 2)])
def test_a_second_prompt_begins_anew(copies, depth):
    from paper_2407_12075_amd import decoder
    torch.cuda.set_device(0)
    cfg = decoder.DecoderConfig(layers=2, heads=4, kv_heads=2, dim=32, hidden=256, vocab=256, page=32, max_len=256, n_seqs=4, dtype=torch.float32)
    prompts = [torch.randint(0, cfg.vocab, (n,), generator=torch.Generator().manual_seed(n)).cuda() for n in (90, 41, 90)]
    want = [decoder.Decoder(cfg, seed=3).generate(p, copies, 20, depth, 2) for p in prompts]
    model = decoder.Decoder(cfg, seed=3)
    assert [model.generate(p, copies, 20, depth, 2) for p in prompts] == want
    # after a text that was too long as well
    with pytest.raises(RuntimeError, match="longer than"):
        model.generate(prompts[0], copies, 300, depth, 2)
    assert model.generate(prompts[1], copies, 20, depth, 2) == want[1]
    lens = model.index.lens.tolist()
    assert sum(lens[copies:]) == 0 and int((model.index.refs > 0).sum()) <= sum(-(-n // cfg.page) for n in lens)
