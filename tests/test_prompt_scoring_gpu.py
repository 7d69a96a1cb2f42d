"""Norm with rotation, the cache's write, chunks and log probabilities together, as examples/prompt_scoring.py
uses them: pieces of any length give the whole sequence's scores, and the gradients are those of the formulas."""
import math
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import prompt_scoring as ex  # noqa: E402
from paper_2608_20172_gb300 import binding  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    binding.load()


def prompts_of(lengths, vocab, seed=0):
    g = torch.Generator().manual_seed(seed)
    return [torch.randint(0, vocab, (n,), generator=g).to(DEV) for n in lengths]


def plain_logits(model, tokens):
    """The model in fp64 from elementary operations, [T, vocab], differentiable in the model's parameters."""
    c, f8 = model.cfg, torch.float64
    T, G = len(tokens), c.H // c.Hk
    norm = lambda x: x / torch.sqrt(x.square().mean(-1, keepdim=True) + torch.finfo(c.dtype).eps)  # noqa: E731
    f = model.rotary.freqs
    a = torch.arange(T, device=DEV, dtype=f8)[:, None, None] * f
    cos, sin = torch.cos(a) * model.rotary.scale, torch.sin(a) * model.rotary.scale

    def turned(x, w):
        n = x / torch.sqrt(x.square().mean(-1, keepdim=True) + 1e-6) * w.to(f8)
        x0, x1 = n[..., :c.d // 2], n[..., c.d // 2:]
        return torch.cat((x0 * cos - x1 * sin, x0 * sin + x1 * cos), -1)

    x = model.embed.to(f8)[tokens]
    i = torch.arange(T, device=DEV)
    for layer in model.layers:
        h = norm(x)
        p1, p2, info = ((h @ layer[n].to(f8)).view(T, H, c.d)
                        for n, H in (("p1", c.H), ("p2", c.Hk), ("info", c.Hk)))
        q, k = turned(p1, layer["w1"]), turned(p2, layer["w2"]).repeat_interleave(G, 1)
        v = info.repeat_interleave(G, 1)
        U = torch.einsum("thd,jhd->htj", q, k) / math.sqrt(c.d)
        R = U * torch.sigmoid(U) - c.lam * torch.log(i + 1.0)[:, None]
        R = torch.where(i[:, None] == i, torch.sigmoid(U / 2), R)
        F = torch.softmax(R.masked_fill(i[None, :] > i[:, None], -math.inf), -1)
        x = x + torch.einsum("htj,jhd->thd", F, v).flatten(-2) @ layer["out"].to(f8)
    return norm(x) @ model.head.to(f8)


def test_pieces_give_the_formulas_scores():
    """In fp32 against fp64: logits of about 3 whose sums of up to 256 terms, over two layers, are off by some
    hundred roundings of 2^-24 of their size: 1e-4 is ten times that."""
    model = ex.Scorer(ex.Config(dtype=torch.float32))
    prompts = prompts_of([150, 2, 77, 31], model.cfg.vocab)
    logits = [plain_logits(model, p) for p in prompts]
    for piece in (1000, 48, 7):
        pieces = ex.Pieces(model, 4, 24, 16, 160)
        got = ex.score(pieces, prompts, piece, top=4)
        for p, z, (logp, entropy, tokens, top) in zip(prompts, logits, got):
            want = torch.log_softmax(z[:-1], -1)
            assert torch.allclose(logp.double(), want.gather(1, p[1:, None])[:, 0], atol=1e-4, rtol=0)
            assert torch.allclose(entropy.double(), -(want.exp() * want).sum(-1), atol=1e-4, rtol=0)
            best = want.sort(-1, descending=True).values[:, :4]
            assert torch.allclose(top.double(), best, atol=1e-4, rtol=0)
            assert torch.allclose(want.gather(1, tokens.long()), best, atol=2e-4, rtol=0)


def test_bf16_pieces_of_any_length_agree():
    """The same rows through chunks of other lengths: P and Y are rounded to bf16 (2^-8 of their size) in each of
    two layers, so that logits of about 3 differ by a few hundredths."""
    model = ex.Scorer(ex.Config())
    prompts = prompts_of([300, 40], model.cfg.vocab, 1)
    scores = []
    for piece in (1000, 37, 1):
        scores.append(ex.score(ex.Pieces(model, 2, 40, 16, 320), prompts, piece))
        for (a, h), (b, k) in zip(scores[0], scores[-1]):
            assert float((a - b).abs().max()) < 0.15 and float((h - k).abs().max()) < 0.15


def test_gradients_are_the_formulas():
    """fp32 through the wrappers against autograd through the fp64 formulas, every parameter: roundings of sums of
    up to some thousand terms, 1e-4 of the largest entry."""
    model = ex.Scorer(ex.Config(dtype=torch.float32))
    tokens = torch.stack(prompts_of([33, 33], model.cfg.vocab, 2))
    weights = torch.rand((2, 33), generator=torch.Generator().manual_seed(3)).to(DEV)
    params = model.parameters()
    for t in params:
        t.requires_grad_()
    got = torch.autograd.grad(model.loss(tokens, weights, entropy=0.1), params)
    want_loss = 0.0
    for b in range(2):
        logp = torch.log_softmax(plain_logits(model, tokens[b])[:-1], -1)
        chosen = logp.gather(1, tokens[b, 1:, None])[:, 0]
        want_loss = want_loss - (chosen * weights[b, 1:].double()).sum() + 0.1 * (logp.exp() * logp).sum()
    for g, w in zip(got, torch.autograd.grad(want_loss, params)):
        assert float((g.double() - w.double()).abs().max()) <= 1e-4 * float(w.abs().max()) + 1e-9


def test_step_in_a_graph():
    """A whole step captured once serves steps of other counts and lengths: no length is on the host."""
    model = ex.Scorer(ex.Config())
    prompts = prompts_of([90, 200, 17], model.cfg.vocab, 4)
    N = 64
    eager, graphed = (ex.Pieces(model, 3, 30, 16, 256) for _ in range(2))
    tokens = torch.zeros(N, dtype=torch.int64, device=DEV)
    counts = torch.zeros(3, dtype=torch.int32, device=DEV)
    lengths, state = graphed.lengths, graphed.free_state
    with torch.no_grad():
        graphed.step(tokens, counts)  # (first calls outside the capture)
        graphed.lengths, graphed.free_state = lengths, state
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out, plan = graphed.step(tokens, counts)
            lengths.copy_(plan.lengths)
            state.copy_(plan.free_state)
        at = [0, 0, 0]
        for take in ([40, 20, 4], [1, 50, 13], [30, 0, 0], [19, 45, 0], [0, 64, 0]):
            new = torch.cat([p[a:a + n] for p, a, n in zip(prompts, at, take)])
            tokens.zero_()
            tokens[:len(new)] = new
            counts.copy_(torch.tensor(take, dtype=torch.int32))
            want, _ = eager.step(tokens, counts)
            graph.replay()
            torch.cuda.synchronize()
            n = sum(take)
            assert torch.equal(out[:n], want[:n]) and torch.equal(lengths, eager.lengths)
            at = [a + n for a, n in zip(at, take)]
    assert int(eager.status) == int(graphed.status) == 0


def test_main_runs(monkeypatch, capsys):
    monkeypatch.setattr(sys, "argv", ["prompt_scoring.py", "--prompts", "3", "--piece", "33"])
    ex.main()
    text = capsys.readouterr().out
    assert text.count("perplexity") == 3 and "gradient norm" in text
