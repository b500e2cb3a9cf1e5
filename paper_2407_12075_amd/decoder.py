"""A small decoder on the library: every projection is a tiled-bit layer (``stack.py``), keys and values live in the paged
cache (``kv.py``), and its operators run together as a server would use them:

* a prompt is run once and forked, so that all its continuations share its pages until they write to one of them;
* each step drafts a few tokens per sequence with attention over picked blocks only, gives their keys back, and has the whole
  model judge the drafts and their runners-up as a tree in one pass;
* the keys of the accepted path move together, the others are given back; a sequence that has ended frees its pages, and
  compaction brings the rest to the front of the pool.

What is emitted is what the whole model picks (its highest logit) after each prefix: drafts change the speed only.  Weights
are synthetic; embeddings, norms, residual sums and the choice of tokens are PyTorch's, everything else is the library's.  At this
size the host's launches set the pace (127 steps without drafts in 79 - 89 ms, 66 steps of four passes with them in 194 - 197 ms): what the
example shows is how the calls fit together, and that drafts save steps, not that they pay.

    python -m paper_2407_12075_amd.decoder          # tokens per second with and without drafts on cuda:0
"""
from __future__ import annotations

import json
import time
from dataclasses import dataclass
from typing import List, Optional, Tuple

import torch

from . import kv, tbn
from .stack import LayerSpec, TiledStack


@dataclass
class DecoderConfig:
    layers: int = 4
    heads: int = 8
    kv_heads: int = 2
    dim: int = 64
    hidden: int = 2048
    vocab: int = 1024
    k: int = 4                       # tiles per layer
    page: int = 64
    max_len: int = 4096
    n_seqs: int = 8
    dtype: torch.dtype = torch.bfloat16

    @property
    def width(self) -> int:
        return self.heads * self.dim


def tree_of(depth: int) -> Tuple[List[int], List[int]]:
    """A root and, per depth, the best token and its runner-up, both below the best one above: parents and depths of the nodes."""
    parents, depths = [-1], [0]
    for d in range(depth):
        main = 2 * d - 1 if d else 0
        parents += [main, main]
        depths += [d + 1, d + 1]
    return parents, depths


def tree_mask(parents: List[int]) -> List[List[int]]:
    """What tbn_tree_attention takes: bit j of row i is set where j is i or above it."""
    words = (len(parents) + 31) // 32
    rows: List[List[int]] = []
    for i, p in enumerate(parents):
        row = list(rows[p]) if p >= 0 else [0] * words
        row[i // 32] |= 1 << (i % 32)
        rows.append(row)
    return [[w - (1 << 32) if w >> 31 else w for w in row] for row in rows]


class Decoder:
    """The model, one pool of pages per layer, and the index that they share."""

    def __init__(self, cfg: DecoderConfig, seed: int = 0, device: str = "cuda"):
        self.cfg, self.device = cfg, torch.device(device)
        w = cfg.width
        specs: List[LayerSpec] = []
        for _ in range(cfg.layers):
            specs += [LayerSpec(w, (cfg.heads + 2 * cfg.kv_heads) * cfg.dim), LayerSpec(w, w), LayerSpec(w, cfg.hidden, relu=True), LayerSpec(cfg.hidden, w)]
        self.stack = TiledStack(specs + [LayerSpec(w, cfg.vocab)], cfg.k, seed=seed, device=device)
        gen = torch.Generator().manual_seed(seed)
        self.embed = torch.randn(cfg.vocab, w, generator=gen).to(device, cfg.dtype)
        self.max_pages = -(-cfg.max_len // cfg.page)
        self.place = (0.5 * torch.randn(self.max_pages * cfg.page, w, generator=gen)).to(device, cfg.dtype)
        n_pages = cfg.n_seqs * self.max_pages
        self.pools = [kv.kv_pool(n_pages, cfg.kv_heads, cfg.dim, cfg.page, cfg.dtype, summary=True, device=device) for _ in range(cfg.layers)]
        self.index = kv.kv_index(cfg.n_seqs, self.max_pages, n_pages, cfg.page, device=device)
        self.steps = 0   # of generate()

    def _linear(self, i: int, x: torch.Tensor) -> torch.Tensor:
        s = self.stack.specs[i]
        return tbn.tbn_linear_forward(x, self.stack.tiles[i], self.stack.alphas[i], s.cout, self.stack.k, flags=tbn.TBN_FLAG_RELU if s.relu else 0)

    @staticmethod
    def _norm(x: torch.Tensor) -> torch.Tensor:
        f = x.float()
        return (f * torch.rsqrt(f.square().mean(-1, keepdim=True) + 1e-6)).to(x.dtype)

    def forward(self, tokens: torch.Tensor, places: torch.Tensor, counts: torch.Tensor, max_new: int, mask: Optional[torch.Tensor] = None,
                n_select: int = 0) -> torch.Tensor:
        """Logits of `tokens` (all sequences', one after another; counts int32 of each), whose keys join the cache.  n_select: attention
        over that many picked blocks of each query instead of all."""
        cfg, index = self.cfg, self.index
        cu = torch.nn.functional.pad(counts.cumsum(0, dtype=torch.int32), (1, 0))
        src, dst = kv.tbn_kv_reserve(index, counts)
        x = self.embed[tokens] + self.place[places.clamp(max=self.place.shape[0] - 1)]   # beyond: reserve has said no, check() raises
        q_end, k_end = cfg.heads, cfg.heads + cfg.kv_heads
        for i, pool in enumerate(self.pools):
            kv.tbn_kv_copy_pages(pool, src, dst)
            qkv = self._linear(4 * i, self._norm(x)).view(-1, cfg.heads + 2 * cfg.kv_heads, cfg.dim)
            kv.tbn_kv_append(pool, index, qkv[:, q_end:k_end], qkv[:, k_end:], cu, max_new)
            if n_select:
                picks = kv.tbn_block_select(qkv[:, :q_end], pool, index, cu, max_new, n_select)
                out, _ = kv.tbn_block_attention(qkv[:, :q_end], pool, index, cu, max_new, picks)
            else:
                out, _ = kv.tbn_tree_attention(qkv[:, :q_end], pool, index, cu, max_new, mask=mask)
            x = x + self._linear(4 * i + 1, out.view(-1, cfg.width))
            x = x + self._linear(4 * i + 3, self._linear(4 * i + 2, self._norm(x)))
        return self._linear(4 * cfg.layers, self._norm(x)).float()

    def check(self) -> None:
        """Raises where a step found the pool full or a sequence too long; waits for the GPU."""
        st = int(self.index.status.item())
        if st:
            raise RuntimeError("the cache is full" if st == kv.TBN_KV_FULL else "a sequence is longer than the cache allows")

    def prompt(self, tokens: torch.Tensor, copies: int) -> torch.Tensor:
        """Runs a prompt as sequence 0 and forks it into the sequences below `copies`; each begins with another of the best first
        tokens, which are returned (int64, copies) and whose keys are not in the cache yet.  What the cache held is given back first."""
        n = tokens.numel()
        kv.tbn_kv_release(self.index, torch.zeros_like(self.index.lens))
        self.index.status.zero_()
        counts = torch.zeros(self.cfg.n_seqs, dtype=torch.int32, device=self.device)
        counts[0] = n
        logits = self.forward(tokens, torch.arange(n, device=self.device), counts, n)
        if copies > 1:
            children = torch.arange(1, copies, dtype=torch.int32, device=self.device)
            kv.tbn_kv_fork(self.index, torch.zeros_like(children), children)
        return logits[-1].topk(copies).indices

    def step(self, last: torch.Tensor, depth: int = 0, n_select: int = 4) -> Tuple[torch.Tensor, torch.Tensor]:
        """One step of the sequences below last.numel(), each of which ends with a token whose key is not in the cache yet.  Drafts `depth`
        tokens (0: none).  Returns (tokens (sequences, depth + 1), counts): what follows `last`, of which counts are emitted."""
        cfg, index, dev = self.cfg, self.index, self.device
        n = last.numel()
        live = torch.zeros(cfg.n_seqs, dtype=torch.int32, device=dev)
        live[:n] = 1
        base = index.lens.clone()
        first = base[:n].long()
        nodes, draft = [last], last
        for d in range(depth):
            logits = self.forward(draft, first + d, live, 1, n_select=n_select)
            best = logits.topk(2, 1).indices
            nodes += [best[:, 0], best[:, 1]]
            draft = best[:, 0]
        if depth:
            kv.tbn_kv_release(index, base)
        parents, depths = tree_of(depth)
        size = len(parents)
        tree = torch.stack(nodes, 1)
        mask = torch.tensor(tree_mask(parents), dtype=torch.int32, device=dev).repeat(n, 1) if depth else None
        places = first[:, None] + torch.tensor(depths, device=dev)
        choice = self.forward(tree.flatten(), places.flatten(), live * size, size, mask=mask).argmax(1).view(n, size)
        # down the tree, as long as the model's choice is one of the drafts
        at = torch.zeros(n, dtype=torch.int64, device=dev)
        going = torch.ones(n, dtype=torch.bool, device=dev)
        emitted, picks, counts = [choice[:, 0]], [at], torch.ones(n, dtype=torch.int32, device=dev)
        for d in range(depth):
            wanted = choice.gather(1, at[:, None])[:, 0]
            main = going & (wanted == tree[:, 2 * d + 1])
            side = going & ~main & (wanted == tree[:, 2 * d + 2])
            at = torch.where(main, 2 * d + 1, torch.where(side, 2 * d + 2, at))
            counts += (main | side).int()
            picks.append(torch.where(main | side, at, size))   # behind the last pick: not looked at
            emitted.append(choice.gather(1, at[:, None])[:, 0])
            going = main
        if depth:
            kept = torch.zeros(cfg.n_seqs, depth + 1, dtype=torch.int32, device=dev)
            kept[:n] = torch.stack(picks, 1)
            many = torch.zeros(cfg.n_seqs, dtype=torch.int32, device=dev)
            many[:n] = counts
            for pool in self.pools:
                kv.tbn_kv_keep(pool, index, base, kept, many)
            kv.tbn_kv_release(index, base + many)
        return torch.stack(emitted, 1), counts

    def end(self, seq: int) -> None:
        """Frees a sequence's pages and moves the others' to the front of the pool."""
        keep = self.index.lens.clone()
        keep[seq] = 0
        kv.tbn_kv_release(self.index, keep)
        src, dst, count = kv.tbn_kv_compact(self.index)
        for pool in self.pools:
            kv.tbn_kv_copy_pages(pool, src, dst, count)

    def generate(self, prompt: torch.Tensor, copies: int, n_new: int, depth: int = 0, n_select: int = 4) -> List[List[int]]:
        """`copies` continuations of at least n_new tokens each (the first of them chosen by prompt(), the others as the model wants)."""
        last = self.prompt(prompt, copies)
        texts = [[t] for t in last.tolist()]
        self.steps = 0
        while min(len(t) for t in texts) < n_new:
            self.steps += 1
            tokens, counts = self.step(last, depth, n_select)
            last = tokens.gather(1, counts[:, None].long() - 1)[:, 0]
            for t, row, m in zip(texts, tokens.tolist(), counts.tolist()):
                t += row[:m]
        self.check()
        return texts


def main() -> None:
    cfg = DecoderConfig()
    prompt = torch.randint(0, cfg.vocab, (2000,), generator=torch.Generator().manual_seed(1)).cuda()
    copies, n_new, texts = 8, 128, {}
    for depth in (0, 3):
        for timed in (False, True):
            model = Decoder(cfg)
            torch.cuda.synchronize()
            t = time.perf_counter()
            texts[depth] = model.generate(prompt, copies, n_new, depth)
            torch.cuda.synchronize()
            t = time.perf_counter() - t
        print(json.dumps({"example": "decoder", "copies": copies, "prompt": prompt.numel(), "drafted_depth": depth, "tokens": sum(map(len, texts[depth])), "steps": model.steps,
                          "ms": round(1e3 * t, 2), "tokens_per_s": round(sum(map(len, texts[depth])) / t),
                          "pages_in_use": int((model.index.refs > 0).sum()), "data": "synthetic", "dtype": str(cfg.dtype)}), flush=True)


if __name__ == "__main__":
    main()
