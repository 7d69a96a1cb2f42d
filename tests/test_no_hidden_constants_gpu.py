"""Learned temperatures and frequencies, of which the library has no gradients: a backward that wants one is
refused, any other gives what it gives for constants."""
import pytest
import torch

from paper_2608_20172_gb300 import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_temperature_and_frequencies():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    x = torch.randn(4, 50, device=DEV).requires_grad_()
    targets = torch.tensor([0, 49, -1, 3], dtype=torch.int32, device=DEV)
    t = torch.full((4,), 0.7, device=DEV)
    f = lambda t: sum(o.sum() for o in binding.LogprobsFunction.apply(x, targets, t))  # noqa: E731
    (want,) = torch.autograd.grad(f(t), x)
    t.requires_grad_()
    (got,) = torch.autograd.grad(f(t), x)
    assert torch.equal(got, want)
    with pytest.raises(ValueError, match="temperature"):
        f(t).backward()
    p = torch.randn(5, 2, 32, device=DEV).requires_grad_()
    freqs = binding.rotary(32, device=DEV).freqs
    f = lambda q: binding.NormRopeFunction.apply(p, None, None, None, binding.Rotary(q))[0].square().sum()  # noqa: E731
    (want,) = torch.autograd.grad(f(freqs), p)
    freqs.requires_grad_()
    (got,) = torch.autograd.grad(f(freqs), p)
    assert torch.equal(got, want)
    with pytest.raises(ValueError, match="frequencies"):
        f(freqs).backward()
