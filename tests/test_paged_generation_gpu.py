"""The serving path as a whole (examples/paged_generation.py): steps over the paged cache give the
logits of the whole sequence recomputed, pages come back, and a step replays from a CUDA graph.

Bound on the logits: two paths of four bf16 layers, equal in exact arithmetic; every layer rounds its
activations to bf16 a few times (2^-8 each) with independent errors, so that logits of norm about
sqrt(width) may differ by a few percent of their spread: 6 % of the largest."""
import os
import sys

import pytest
import torch

from paper_2608_20172_gb300 import binding

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                                "examples"))
import paged_generation as pg  # noqa: E402

pytestmark = pytest.mark.gpu
BOUND = 0.06


@pytest.fixture(scope="module")
def model():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    binding.load()
    return pg.Decoder(pg.Config(vocab=300, layers=4, H=4, d=48))


def prompts_of(model, lengths, seed=1):
    g = torch.Generator().manual_seed(seed)
    return [torch.randint(0, model.cfg.vocab, (n,), generator=g).cuda() for n in lengths]


def near(a, b):
    assert (a - b).abs().max() <= BOUND * b.abs().max(), (a - b).abs().max()


@pytest.mark.parametrize("page", [1, 16, 24])
def test_steps_equal_the_whole_sequence(model, page):
    lengths = [1, 7, 130, 33]
    prompts = prompts_of(model, lengths)
    server = pg.Server(model, 4, n_pages=4 * -(-170 // page), page_size=page, max_rows=170)
    seqs = [p.tolist() for p in prompts]
    for row, p in enumerate(prompts):
        near(server.admit(row, p), model.prefill(p)[-1])
    g = torch.Generator().manual_seed(3)
    for step in range(20):
        counts = torch.ones(4, dtype=torch.int32)
        if step % 3 == 1:
            counts[step % 4] = 0  # a row that waits
        new = torch.randint(0, model.cfg.vocab, (4,), generator=g)
        server.last = new.cuda()
        logits = server.step(counts.cuda())
        for row in range(4):
            if counts[row]:
                seqs[row].append(int(new[row]))
                near(logits[row], model.prefill(torch.tensor(seqs[row]).cuda())[-1])
    assert int(server.status) == 0
    assert server.lengths.tolist() == [len(s) for s in seqs]


def test_generation_serves_more_requests_than_rows(model):
    prompts = prompts_of(model, [5, 60, 1, 17, 90, 33, 2], seed=4)
    server = pg.Server(model, 3, n_pages=3 * 8, page_size=16, max_rows=128)
    out = pg.generate(server, prompts, 20)
    assert [len(s) for s in out] == [len(p) + 20 for p in prompts]
    assert all(s[:len(p)] == p.tolist() for s, p in zip(out, prompts))
    assert all(0 <= t < model.cfg.vocab for s in out for t in s)
    assert int(server.free_state[1]) == 24  # every page came back
    # the same seed draws the same tokens, whatever pages the requests lie in
    again = pg.Server(model, 3, n_pages=40, page_size=16, max_rows=128)
    assert pg.generate(again, prompts, 20) == out


def test_step_in_a_graph(model):
    """A captured step, replayed with other lengths, tokens and pages, equals eager steps."""
    prompts = prompts_of(model, [30, 1, 64], seed=5)
    eager, graphed = (pg.Server(model, 3, n_pages=40, page_size=16, max_rows=128) for _ in range(2))
    for s in (eager, graphed):
        for row, p in enumerate(prompts):
            s.admit(row, p)
        s.last = torch.tensor([1, 2, 3]).cuda()
    counts = torch.ones(3, dtype=torch.int32).cuda()
    lengths, state = graphed.lengths.clone(), graphed.free_state.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graphed.lengths, graphed.free_state = lengths, state
        graphed.step(counts)  # (the same inputs below: what it writes is written alike)
    torch.cuda.current_stream().wait_stream(side)
    graphed.lengths, graphed.free_state = lengths, state
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        logits = graphed.step(counts)
        token = binding.sample(logits, torch.full((3,), 0.5, device="cuda"))[0]
        graphed.last.copy_(token)
        lengths.copy_(graphed.lengths)
        state.copy_(graphed.free_state)
    for _ in range(25):
        graph.replay()
        want = eager.step(counts)
        tok = binding.sample(want, torch.full((3,), 0.5, device="cuda"))[0]
        torch.cuda.synchronize()
        assert torch.equal(logits, want) and torch.equal(token, tok)
        eager.last = tok.long()
    assert torch.equal(lengths, eager.lengths) and torch.equal(state, eager.free_state)
    assert int(graphed.status) == 0
