"""Scoring prompts in pieces over a paged cache, and training on their tokens.

A small decoder whose queries and keys are normed per head and rotated by a scaled rotation, with key heads
that query heads share.  Prompts of different lengths go through the cache a piece of each at a time: the
pages of the new tokens are planned on the GPU, their queries and keys normed and rotated in one pass, their
rows written, the pieces read against everything before them, and every token's log probability taken with the
row's entropy and its likeliest alternatives.  The same model trains on whole sequences through the autograd
wrappers of the same operators.  Random weights: what it shows is the path.

    python examples/prompt_scoring.py [--prompts 6] [--piece 48] [--top 3]
"""
from __future__ import annotations

import argparse
import math
import os
import sys
from dataclasses import dataclass

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2608_20172_gb300 import binding  # noqa: E402


@dataclass(frozen=True)
class Config:
    vocab: int = 500
    layers: int = 2
    H: int = 4       # query heads
    Hk: int = 2      # key/value heads
    d: int = 64
    width: int = 128
    lam: float = 0.5
    context: int = 64      # the context that the rotation was made for,
    longer: float = 8.0    # and how many times as long it is stretched
    dtype: torch.dtype = torch.bfloat16


class Scorer:
    """Pre-norm decoder of Relation layers with normed and rotated queries and keys."""

    def __init__(self, cfg: Config, seed: int = 0, device="cuda"):
        self.cfg = cfg
        g = torch.Generator().manual_seed(seed)
        w = lambda *s: (torch.randn(s, generator=g) / math.sqrt(s[0])).to(device, cfg.dtype)  # noqa: E731
        self.embed = torch.randn((cfg.vocab, cfg.width), generator=g).to(device, cfg.dtype)
        self.head = w(cfg.width, cfg.vocab) * 3
        self.layers = [{"p1": w(cfg.width, cfg.H * cfg.d), "p2": w(cfg.width, cfg.Hk * cfg.d),
                        "info": w(cfg.width, cfg.Hk * cfg.d), "out": w(cfg.H * cfg.d, cfg.width),
                        "w1": (1 + 0.1 * torch.randn(cfg.d, generator=g)).to(device),
                        "w2": (1 + 0.1 * torch.randn(cfg.d, generator=g)).to(device)}
                       for _ in range(cfg.layers)]
        self.rotary = binding.rotary(cfg.d, layout="half", scaling="yarn", factor=cfg.longer,
                                     context=cfg.context, device=device)

    def parameters(self):
        return [self.embed, self.head] + [t for layer in self.layers for t in layer.values()]

    def projections(self, layer, x):
        c = self.cfg
        h = torch.nn.functional.rms_norm(x, (c.width,))
        return [(h @ layer[n]).view(*x.shape[:-1], H, c.d)
                for n, H in (("p1", c.H), ("p2", c.Hk), ("info", c.Hk))]

    def logits(self, x):
        return torch.nn.functional.rms_norm(x, (self.cfg.width,)) @ self.head

    def whole(self, tokens):
        """Logits [B, T, vocab] of whole sequences [B, T], differentiable."""
        c, G = self.cfg, self.cfg.H // self.cfg.Hk
        x = self.embed[tokens]
        for layer in self.layers:
            p1, p2, info = self.projections(layer, x)
            q, k = binding.NormRopeFunction.apply(p1, p2, layer["w1"], layer["w2"], self.rotary)
            k, v = (t.repeat_interleave(G, 2) for t in (k, info))
            y = binding.RelationFunction.apply(q, k, v, torch.tensor(c.lam))
            x = x + y.flatten(-2) @ layer["out"]
        return self.logits(x)

    def loss(self, tokens, weights, entropy: float = 0.0):
        """-sum of the tokens' weighted log probabilities given those before them, less `entropy` times the
        rows' entropies."""
        logits = self.whole(tokens)[:, :-1].reshape(-1, self.cfg.vocab)
        logp, h, _ = binding.LogprobsFunction.apply(logits, tokens[:, 1:].reshape(-1).int())
        return -(logp * weights[:, 1:].reshape(-1)).sum() - entropy * h.sum()


class Pieces:
    """Requests that come to the model's paged cache a piece at a time."""

    def __init__(self, model: Scorer, batch: int, n_pages: int, page_size: int, max_rows: int):
        c, dev = model.cfg, model.embed.device
        self.model, self.batch, self.page = model, batch, page_size
        shape = (c.layers, n_pages, page_size, c.Hk, c.d)
        self.k, self.v = (torch.zeros(shape, dtype=c.dtype, device=dev) for _ in range(2))
        i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device=dev)  # noqa: E731
        self.table = i32(batch, -(-max_rows // page_size))
        self.free = torch.arange(n_pages, dtype=torch.int32, device=dev)
        self.free_state = torch.tensor([0, n_pages], dtype=torch.int32, device=dev)
        self.lengths, self.status = i32(batch), i32(1)

    def step(self, tokens, counts):
        """Logits [N, vocab] of the requests' next tokens [N] (counts int32 [batch] of them, in the requests'
        order; what is left of the buffer is padding), and the step's plan."""
        model, c = self.model, self.model.cfg
        plan = binding.page_plan(self.lengths, counts, self.table, self.free, self.free_state, self.page,
                                 tokens.numel(), dev_status=self.status)
        self.lengths, self.free_state = plan.lengths, plan.free_state
        x = model.embed[tokens]
        for i, layer in enumerate(model.layers):
            p1, p2, info = model.projections(layer, x)
            q, k = binding.norm_rope(p1, p2, model.rotary, plan.positions, layer["w1"], layer["w2"])
            binding.cache_append(None, k, info, None, None, plan.slots, self.k[i], self.v[i], rope_base=0.0,
                                 dev_status=self.status)
            y, _ = binding.paged_chunk(q, self.k[i], self.v[i], self.table, plan.starts, plan.positions, c.lam,
                                       dev_status=self.status)
            x = x + y.flatten(-2) @ layer["out"]
        return model.logits(x), plan


def score(pieces: Pieces, prompts, piece: int, top: int = 0):
    """Per prompt its tokens' log probabilities given those before them (from the second on), the entropies
    there, and the `top` likeliest tokens with their log probabilities; `piece` tokens of each at a time."""
    dev = pieces.table.device
    at = [0] * len(prompts)
    out = [[] for _ in prompts]
    while any(a < len(p) for a, p in zip(at, prompts)):
        take = [min(piece, len(p) - a) for a, p in zip(at, prompts)]
        cut = [p[a:a + n] for a, n, p in zip(at, take, prompts)]
        # a row's given token is the prompt's next one, none for its last
        given = [torch.cat([p[a + 1:a + n + 1], p.new_full((int(a + n == len(p)) if n else 0,), -1)])
                 for a, n, p in zip(at, take, prompts)]
        counts = torch.tensor(take, dtype=torch.int32, device=dev)
        logits, _ = pieces.step(torch.cat(cut), counts)
        r = binding.logprobs(logits, torch.cat(given).int(), top=top, dev_status=pieces.status)
        for rows, all_rows in zip(out, zip(*(t.split(take) for t in r if t is not None))):
            rows.append(all_rows)
        at = [a + n for a, n in zip(at, take)]
    if int(pieces.status):
        raise binding.RelationError(int(pieces.status), "score")
    joined = [[torch.cat(t)[:-1] for t in zip(*rows)] for rows in out]
    return [[t for i, t in enumerate(rows) if i != 2] for rows in joined]  # (without logz)


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--prompts", type=int, default=6)
    ap.add_argument("--piece", type=int, default=48)
    ap.add_argument("--top", type=int, default=3)
    a = ap.parse_args()
    model = Scorer(Config())
    g = torch.Generator().manual_seed(1)
    lengths = torch.randint(2, 400, (a.prompts,), generator=g).tolist()
    prompts = [torch.randint(0, model.cfg.vocab, (n,), generator=g).cuda() for n in lengths]
    pieces = Pieces(model, a.prompts, n_pages=sum(-(-n // 16) for n in lengths), page_size=16,
                    max_rows=max(lengths))
    with torch.no_grad():
        for p, rows in zip(prompts, score(pieces, prompts, a.piece, a.top)):
            logp, entropy = rows[:2]
            hits = (rows[2] == p[1:, None]).any(1).float().mean() if a.top else float("nan")
            print(f"{len(p):4d} tokens: perplexity {float(torch.exp(-logp.mean())):9.1f}, mean entropy "
                  f"{float(entropy.mean()):.3f}, among the {a.top} likeliest {float(hits):.1%}")
    for t in model.parameters():
        t.requires_grad_()
    batch = torch.randint(0, model.cfg.vocab, (2, 65), generator=g).cuda()
    loss = model.loss(batch, torch.ones((2, 65), device="cuda"), entropy=0.01)
    loss.backward()
    size = math.sqrt(sum(float(t.grad.float().square().sum()) for t in model.parameters()))
    print(f"training step on {batch.numel()} tokens: loss {float(loss.detach()):.1f}, gradient norm {size:.2f}")


if __name__ == "__main__":
    main()
