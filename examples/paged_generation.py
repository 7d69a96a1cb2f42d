"""Text generation with a small Full Relation decoder over a paged cache.

Requests of different lengths share one pool of pages.  A prompt is prefilled with the ordinary
forward and its keys and information states written to the request's pages; from then on every step
plans the pages of the new tokens on the GPU, writes their rows, reads each request's last row over
its pages and draws the next tokens.  A request that has its tokens gives its pages back and the next
one takes its place.  Random weights (there is no checkpoint here): what it shows is the serving path.

    python examples/paged_generation.py [--requests 12] [--batch 4] [--tokens 24] [--greedy]
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
    vocab: int = 1000
    layers: int = 4
    H: int = 8
    d: int = 48
    lam: float = 0.5
    rope_base: float = 1.0e4

    @property
    def width(self) -> int:
        return self.H * self.d


def rms_norm(x):
    return (x.float() * torch.rsqrt(x.float().square().mean(-1, keepdim=True) + 1e-6)).to(x.dtype)


class Decoder:
    """Pre-norm decoder: projections, Relation with RoPE and Givens mixing, output projection, FFN."""

    def __init__(self, cfg: Config, seed: int = 0, device="cuda"):
        self.cfg = cfg
        g = torch.Generator().manual_seed(seed)
        w = lambda *s: (torch.randn(s, generator=g) / math.sqrt(s[0])).to(  # noqa: E731
            device, torch.bfloat16)
        D = cfg.width
        self.embed = torch.randn((cfg.vocab, D), generator=g).to(device, torch.bfloat16)
        self.head = w(D, cfg.vocab) * 4
        self.layers = [{"p1": w(D, D), "p2": w(D, D), "info": w(D, D), "out": w(D, D),
                        "up": w(D, 4 * D), "down": w(4 * D, D),
                        "theta": (torch.randn(cfg.H // 2, generator=g) * 0.5).to(device),
                        "pairing": i % 2} for i in range(cfg.layers)]

    def projections(self, layer, x):
        h = rms_norm(x)
        return [(h @ layer[n]).view(*x.shape[:-1], self.cfg.H, self.cfg.d)
                for n in ("p1", "p2", "info")]

    def after(self, layer, x, y):
        x = x + y.reshape(x.shape) @ layer["out"]
        return x + torch.nn.functional.silu(rms_norm(x) @ layer["up"]) @ layer["down"]

    def logits(self, x):
        return (rms_norm(x) @ self.head).float()

    def prefill(self, tokens, layer_rows=None):
        """Logits [T, vocab] of one sequence; layer_rows(i, k, v) receives every layer's rows."""
        x = self.embed[tokens][None]
        for i, layer in enumerate(self.layers):
            q, k, v = binding.layer_prep(*self.projections(layer, x), layer["theta"],
                                         layer["pairing"], self.cfg.rope_base)
            if layer_rows is not None:
                layer_rows(i, k[0], v[0])
            y, _ = binding.fwd(q, k, v, self.cfg.lam)
            x = self.after(layer, x, y)
        return self.logits(x[0])


class Server:
    """A batch of `batch` requests over `n_pages` pages of `page_size` rows."""

    def __init__(self, model: Decoder, batch: int, n_pages: int, page_size: int, max_rows: int):
        cfg, dev = model.cfg, model.embed.device
        self.model, self.batch, self.page = model, batch, page_size
        shape = (cfg.layers, n_pages, page_size, cfg.H, cfg.d)
        self.k, self.v = (torch.zeros(shape, dtype=torch.bfloat16, device=dev) for _ in range(2))
        i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device=dev)  # noqa: E731
        self.table = i32(batch, -(-max_rows // page_size))
        self.free = torch.arange(n_pages, dtype=torch.int32, device=dev)
        self.free_state = torch.tensor([0, n_pages], dtype=torch.int32, device=dev)
        self.lengths, self.status = i32(batch), i32(1)
        self.last = torch.zeros(batch, dtype=torch.int64, device=dev)  # the requests' last tokens

    def plan(self, counts, n_tokens):
        p = binding.page_plan(self.lengths, counts, self.table, self.free, self.free_state, self.page,
                              n_tokens, dev_status=self.status)
        self.lengths, self.free_state = p.lengths, p.free_state
        return p

    def admit(self, row: int, prompt):
        """Prefill a prompt into batch row `row`; returns the logits of its last token."""
        counts = torch.zeros(self.batch, dtype=torch.int32)
        counts[row] = len(prompt)
        p = self.plan(counts.to(self.table.device), len(prompt))

        def rows(i, k, v):  # rotated and mixed already
            binding.cache_append(None, k, v, None, None, p.slots, self.k[i], self.v[i],
                                 rope_base=0.0, dev_status=self.status)

        return self.model.prefill(prompt, rows)[-1]

    def finish(self, rows):
        """The requests in these batch rows have ended: their pages go back."""
        counts = torch.zeros(self.batch, dtype=torch.int32)
        counts[list(rows)] = -1
        self.plan(counts.to(self.table.device), 1)

    def step(self, counts):
        """One decoding step: counts int32 [batch], 1 for the rows that continue and 0 for idle ones.
        Returns logits [batch, vocab] (of idle rows: without meaning)."""
        model, cfg = self.model, self.model.cfg
        p = self.plan(counts, self.batch)
        at = torch.arange(self.batch, device=counts.device)
        row = torch.searchsorted(p.starts[1:], at.int(), right=True).clamp(max=self.batch - 1)
        token = p.starts[:-1].long().clamp(max=self.batch - 1)  # a row's place among the tokens
        x = model.embed[self.last[row]]
        for i, layer in enumerate(model.layers):
            q = binding.cache_append(*model.projections(layer, x), layer["theta"], p.positions,
                                     p.slots, self.k[i], self.v[i], layer["pairing"], cfg.rope_base,
                                     dev_status=self.status)
            y, _ = binding.paged_decode(q[token], self.k[i], self.v[i], self.table, p.lengths, cfg.lam,
                                        dev_status=self.status)
            x = model.after(layer, x, y[row])
        return model.logits(x)[token]


def generate(server: Server, prompts, n_tokens: int, *, seed: int = 0, temperature: float = 0.8,
             top_k: int = 50, top_p: float = 0.95):
    """n_tokens tokens after each prompt; returns the sequences in the prompts' order."""
    dev, B = server.table.device, server.batch
    g = torch.Generator(device=dev).manual_seed(seed)
    par = {"temperature": torch.full((B,), temperature, device=dev),
           "top_k": torch.full((B,), top_k, dtype=torch.int32, device=dev),
           "top_p": torch.full((B,), top_p, device=dev)}
    draw = lambda logits: binding.sample(  # noqa: E731
        logits, torch.rand(B, generator=g, device=dev), dev_status=server.status, **par)[0]
    waiting, out, active = list(range(len(prompts))), [None] * len(prompts), {}
    while waiting or active:
        for row in range(B):
            if row not in active and waiting:
                n = waiting.pop(0)
                logits = server.admit(row, prompts[n])
                server.last[row] = draw(logits.expand(B, -1).contiguous())[row]
                active[row] = n
                out[n] = prompts[n].tolist() + [int(server.last[row])]
        done = [r for r, n in active.items() if len(out[n]) - len(prompts[n]) >= n_tokens]
        if done:
            server.finish(done)
            for r in done:
                del active[r]
            continue
        counts = torch.zeros(B, dtype=torch.int32)
        counts[list(active)] = 1
        token = draw(server.step(counts.to(dev)))
        server.last = token.long().clamp(min=0)
        for r, t in enumerate(token.tolist()):
            if r in active:
                out[active[r]].append(t)
    if int(server.status):
        raise binding.RelationError(int(server.status), "generate")
    return out


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--requests", type=int, default=12)
    ap.add_argument("--batch", type=int, default=4)
    ap.add_argument("--tokens", type=int, default=24)
    ap.add_argument("--greedy", action="store_true")
    a = ap.parse_args()
    model = Decoder(Config())
    rows = 200 + a.tokens
    server = Server(model, a.batch, n_pages=a.batch * -(-rows // 16), page_size=16, max_rows=rows)
    g = torch.Generator().manual_seed(1)
    prompts = [torch.randint(0, model.cfg.vocab, (int(torch.randint(1, 200, (1,), generator=g)),),
                             generator=g).cuda() for _ in range(a.requests)]
    out = generate(server, prompts, a.tokens, temperature=0.0 if a.greedy else 0.8)
    for p, s in zip(prompts, out):
        print(f"{len(p):4d} prompt tokens -> {s[len(p):]}")
    print(f"free pages: {int(server.free_state[1])} of {server.free.numel()}")


if __name__ == "__main__":
    main()
