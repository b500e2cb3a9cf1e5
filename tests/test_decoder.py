"""The example decoder against the same model in float64 without a cache, and its trees."""
import numpy as np
import pytest
import torch


def test_trees():
    from paper_2407_12075_amd import decoder
    assert decoder.tree_of(0) == ([-1], [0])
    parents, depths = decoder.tree_of(3)
    assert parents == [-1, 0, 0, 1, 1, 3, 3] and depths == [0, 1, 1, 2, 2, 3, 3]
    assert [r[0] for r in decoder.tree_mask(parents)] == [1, 3, 5, 11, 19, 43, 75]
    rows = decoder.tree_mask([-1] + list(range(39)))   # a chain of 40 fills the first word
    assert len(rows[0]) == 2 and rows[31] == [-1, 0] and rows[39] == [-1, 255]


class Exact:
    """The decoder's formulas in float64 over a whole text, weights materialised from the packed tiles."""

    def __init__(self, model):
        from oracle import tbn_oracle as orc
        self.cfg, self.specs = model.cfg, model.stack.specs
        self.w = [orc.materialise(t.cpu().numpy().view(np.uint32), a.cpu().numpy(), s.cin * s.cout, model.cfg.k).astype(np.float64).reshape(s.cout, s.cin)
                  for t, a, s in zip(model.stack.tiles, model.stack.alphas, self.specs)]
        self.embed, self.place = model.embed.double().cpu().numpy(), model.place.double().cpu().numpy()

    def linear(self, i, x):
        y = x @ self.w[i].T
        return np.maximum(y, 0) if self.specs[i].relu else y

    def logits(self, tokens):
        """Logits (tokens, vocab) and the keys and values of each layer (tokens, kv_heads, dim)."""
        c = self.cfg
        norm = lambda x: x / np.sqrt((x * x).mean(-1, keepdims=True) + 1e-6)  # noqa: E731
        x, cached, n = self.embed[tokens] + self.place[:len(tokens)], [], len(tokens)
        for i in range(c.layers):
            qkv = self.linear(4 * i, norm(x)).reshape(n, -1, c.dim)
            q, k, v = qkv[:, :c.heads], qkv[:, c.heads:c.heads + c.kv_heads], qkv[:, c.heads + c.kv_heads:]
            cached.append((k, v))
            out = np.zeros((n, c.heads, c.dim))
            for h in range(c.heads):
                a = q[:, h] @ k[:, h * c.kv_heads // c.heads].T / np.sqrt(c.dim)
                a = np.where(np.tri(n, dtype=bool), a, -np.inf)
                p = np.exp(a - a.max(1, keepdims=True))
                out[:, h] = p @ v[:, h * c.kv_heads // c.heads] / p.sum(1, keepdims=True)
            x = x + self.linear(4 * i + 1, out.reshape(n, -1))
            x = x + self.linear(4 * i + 3, self.linear(4 * i + 2, norm(x)))
        return self.linear(4 * c.layers, norm(x)), cached


def cached_rows(model, layer, seq):
    n, page = int(model.index.lens[seq]), model.cfg.page
    rows = model.index.table[seq, :-(-n // page)].long()
    k = model.pools[layer].k[rows].permute(0, 2, 1, 3).flatten(0, 1)[:n]
    v = model.pools[layer].v[rows].permute(0, 3, 1, 2).flatten(0, 1)[:n]
    return k.cpu(), v.cpu()


# Each layer's kernels are within 1e-5 of the largest value in float32; nine layers and two attentions in a row, whose norms may
# amplify what came before, stay within 100 times that.
TOL = 1e-3


@pytest.mark.gpu
@pytest.mark.parametrize("depth,n_select", [(0, 0), (1, 2), (3, 2), (3, 64)])
def test_texts_are_the_whole_models(depth, n_select):
    from paper_2407_12075_amd import decoder
    torch.cuda.set_device(0)
    cfg = decoder.DecoderConfig(layers=2, heads=4, kv_heads=2, dim=32, hidden=256, vocab=256, page=32, max_len=512, n_seqs=4, dtype=torch.float32)
    model = decoder.Decoder(cfg, seed=3)
    prompt = torch.randint(0, cfg.vocab, (141,), generator=torch.Generator().manual_seed(5))
    steps = []
    real = model.step
    model.step = lambda *a, **kw: steps.append(real(*a, **kw)) or steps[-1]
    texts = model.generate(prompt.cuda(), 3, 40, depth, n_select)
    exact = Exact(model)
    assert all(len(t) >= 40 for t in texts) and len({t[0] for t in texts}) == 3
    for s, text in enumerate(texts):
        whole = prompt.tolist() + text
        logits, cached = exact.logits(whole[:-1])
        size = np.abs(logits).max()
        for i in range(1, len(text)):
            row = logits[len(prompt) + i - 1]
            assert row[text[i]] >= row.max() - TOL * size, (s, i)
        assert int(model.index.lens[s]) == len(whole) - 1   # the last token's key is not there yet
        for layer in range(cfg.layers):
            for got, want in zip(cached_rows(model, layer, s), cached[layer]):
                assert np.abs(got.double().numpy() - want).max() <= TOL * np.abs(want).max(), (s, layer)
    if n_select == 64:   # drafts by the whole model: all but ties are right
        assert np.mean([c.float().mean().item() for _, c in steps]) > 3.5

    # what was shared is stored once: whole pages of the prompt, and what each has of its own
    lens = model.index.lens[:3].tolist()
    full = len(prompt) // cfg.page
    assert int((model.index.refs > 0).sum()) == full + sum(-(-n // cfg.page) - full for n in lens)
    before = {(layer, s): cached_rows(model, layer, s) for layer in range(cfg.layers) for s in (0, 2)}
    model.end(1)
    used = full + sum(-(-lens[s] // cfg.page) - full for s in (0, 2))
    assert (model.index.refs > 0).nonzero().flatten().tolist() == list(range(used)) and int(model.index.lens[1]) == 0
    for (layer, s), was in before.items():
        for a, b in zip(cached_rows(model, layer, s), was):
            assert torch.equal(a, b)


@pytest.mark.gpu
def test_a_full_pool_is_told():
    from paper_2407_12075_amd import decoder
    torch.cuda.set_device(0)
    cfg = decoder.DecoderConfig(layers=1, heads=2, kv_heads=1, dim=32, hidden=64, vocab=64, page=32, max_len=64, n_seqs=2, dtype=torch.float32)
    model = decoder.Decoder(cfg)
    with pytest.raises(RuntimeError, match="longer than"):
        model.generate(torch.zeros(40, dtype=torch.int64, device="cuda"), 2, 8, depth=20)
