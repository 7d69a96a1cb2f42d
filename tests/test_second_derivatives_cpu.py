"""The autograd wrappers give first derivatives; a second one is an error, not a part that is missing.  CPU only:
plain stand-ins take the place of the library's calls."""
import pytest
import torch

from paper_2608_20172_gb300 import binding


def relation_fwd(q, k, v, lam, tau_s, kernel="auto"):
    return q * k + lam * v, q.sum()


def relation_bwd(q, k, v, y, dy, logz, lam, tau_s, kernel="auto"):
    return dy * k, dy * q, lam * dy, (dy * v).sum()


def norm_rope(p1, p2, rotary, positions, w1, w2, *, norm, eps):
    return p1 * p1 * w1, None if p2 is None else p2 * p2 * w2


def norm_rope_grad(dq, dk, p1, p2, rot, positions, w1, w2, *, norm, eps, weights):
    both = [(2 * p * w * g, (g * p * p).sum(0)) if p is not None else (None, None)
            for g, p, w in ((dq, p1, w1), (dk, p2, w2))]
    return both[0][0], both[1][0], both[0][1], both[1][1]


def logprobs(logits, targets, *, temperature=None):
    z = logits.logsumexp(1)
    return binding.Logprobs(logits[torch.arange(len(logits)), targets.long()] - z, z * 0, z, None, None)


def logprobs_grad(logits, targets, logz, entropy, dlogprob, dentropy, dlogz, *, temperature=None):
    p = (logits - logz[:, None]).exp()
    return torch.nn.functional.one_hot(targets.long(), logits.shape[1]) * dlogprob[:, None] + \
        p * (dlogz - dlogprob)[:, None]


@pytest.fixture(autouse=True)
def stand_ins(monkeypatch):
    for name, f in (("fwd", relation_fwd), ("bwd", relation_bwd), ("norm_rope", norm_rope),
                    ("norm_rope_grad", norm_rope_grad), ("logprobs", logprobs), ("logprobs_grad", logprobs_grad)):
        monkeypatch.setattr(binding, name, f)


def leaves(*shapes):
    g = torch.Generator().manual_seed(0)
    return [torch.randn(s, generator=g).requires_grad_() for s in shapes]


def relation():
    q, k, v, lam = leaves((2, 3), (2, 3), (2, 3), ())
    return (q, k, v, lam), binding.RelationFunction.apply(q, k, v, lam)


def rope():
    p1, p2, w1, w2 = leaves((2, 3), (2, 3), (3,), (3,))
    q, k = binding.NormRopeFunction.apply(p1, p2, w1, w2, None)
    return (p1, p2, w1, w2), q + k


def rope_queries():
    p1, w1 = leaves((2, 3), (3,))
    return (p1, w1), binding.NormRopeFunction.apply(p1, None, w1, None, None)[0]


def scores():
    (x,) = leaves((4, 5))
    logp, _, logz = binding.LogprobsFunction.apply(x, torch.tensor([0, 1, 2, 4], dtype=torch.int32))
    return (x,), logp + 0.5 * logz


WRAPPERS = [relation, rope, rope_queries, scores]


@pytest.mark.parametrize("f", WRAPPERS)
@pytest.mark.parametrize("outer", [lambda y: y.sum(), lambda y: y.square().sum()])
def test_a_second_derivative_is_an_error(f, outer):
    """A gradient penalty, of a loss that is linear in the outputs (its gradients' own inputs are constants) and
    of one that is not."""
    inputs, y = f()
    loss = outer(y)
    grads = torch.autograd.grad(loss, inputs, create_graph=True)
    assert all(g.requires_grad for g in grads)
    penalty = sum(g.square().sum() for g in grads)
    with pytest.raises(RuntimeError, match="second derivatives"):
        (loss + penalty).backward()


@pytest.mark.parametrize("f", WRAPPERS)
def test_first_derivatives_are_as_before(f):
    inputs, y = f()
    want = torch.autograd.grad(y.square().sum(), inputs, retain_graph=True)
    with_graph = torch.autograd.grad(y.square().sum(), inputs, create_graph=True)
    for a, b in zip(want, with_graph):
        assert torch.equal(a, b) and not a.requires_grad
    y.square().sum().backward()
    assert all(torch.equal(t.grad, a) and not t.grad.requires_grad for t, a in zip(inputs, want))


def test_inputs_that_need_no_gradient():
    q, k, v, _ = leaves((2, 3), (2, 3), (2, 3), ())
    k, v = k.detach(), v.detach()
    y = binding.RelationFunction.apply(q, k, v, torch.tensor(0.5))
    (g,) = torch.autograd.grad(y.sum(), q, create_graph=True)
    assert torch.equal(g, k)
    with pytest.raises(RuntimeError, match="second derivatives"):
        g.square().sum().backward()
