"""The autograd wrappers under create_graph: the same first derivatives, an error for a second one."""
import pytest
import torch

from paper_2608_20172_gb300 import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    binding.load()


def leaves(*shapes):
    g = torch.Generator(device=DEV).manual_seed(0)
    return [torch.randn(s, generator=g, device=DEV).requires_grad_() for s in shapes]


def relation():
    q, k, v = leaves((1, 9, 2, 32), (1, 9, 2, 32), (1, 9, 2, 32))
    lam = torch.tensor(0.5, device=DEV, requires_grad=True)
    return (q, k, v, lam), binding.RelationFunction.apply(q, k, v, lam)


def rope():
    p1, p2, w1, w2 = leaves((9, 4, 32), (9, 2, 32), (32,), (32,))
    q, k = binding.NormRopeFunction.apply(p1, p2, w1, w2, binding.rotary(32))
    return (p1, p2, w1, w2), q[:, :2] + k


def scores():
    (x,) = leaves((4, 50))
    targets = torch.tensor([0, 49, -1, 3], dtype=torch.int32, device=DEV)
    return (x,), sum(binding.LogprobsFunction.apply(x, targets))


@pytest.mark.parametrize("f", [relation, rope, scores])
@pytest.mark.parametrize("linear", [True, False])
def test_first_derivatives_and_no_second_ones(f, linear):
    inputs, y = f()
    loss = y.sum() if linear else y.square().sum()
    want = torch.autograd.grad(loss, inputs, retain_graph=True)
    grads = torch.autograd.grad(loss, inputs, create_graph=True)
    assert all(torch.equal(a, b) and b.requires_grad for a, b in zip(want, grads))
    with pytest.raises(RuntimeError, match="second derivatives"):
        (loss + sum(g.square().sum() for g in grads)).backward()
