"""An input whose gradient the autograd wrappers do not have is no constant for them: asked for it, they say so.
CPU only: plain stand-ins take the place of the library's calls."""
import pytest
import torch

from paper_2608_20172_gb300 import binding
from tests.test_second_derivatives_cpu import leaves, stand_ins  # noqa: F401

TARGETS = torch.tensor([0, 1, 2, 4], dtype=torch.int32)


def test_a_temperature_that_is_learned():
    (x,) = leaves((4, 5))
    t = torch.ones(4, requires_grad=True)
    for call in (lambda y: y.backward(), lambda y: torch.autograd.grad(y, (x, t)),
                 lambda y: torch.autograd.grad(y, t)):
        with pytest.raises(ValueError, match="temperature"):
            call(binding.LogprobsFunction.apply(x, TARGETS, t)[0].sum())
    # not asked for: as ever
    want = torch.autograd.grad(binding.LogprobsFunction.apply(x, TARGETS, t.detach())[0].sum(), x)
    got = torch.autograd.grad(binding.LogprobsFunction.apply(x, TARGETS, t)[0].sum(), x)
    assert torch.equal(got[0], want[0])
    with torch.no_grad():
        assert not binding.LogprobsFunction.apply(x, TARGETS, t)[0].requires_grad


def test_frequencies_that_are_learned():
    p1, w1 = leaves((2, 4), (4,))
    freqs = torch.ones(2, dtype=torch.float64, requires_grad=True)
    with pytest.raises(ValueError, match="frequencies"):
        binding.NormRopeFunction.apply(p1, None, w1, None, binding.Rotary(freqs))[0].sum().backward()
    (got,) = torch.autograd.grad(binding.NormRopeFunction.apply(p1, None, w1, None, binding.Rotary(freqs))[0].sum(),
                                 p1)
    p1.grad = None  # (the refused backward may have come this far)
    binding.NormRopeFunction.apply(p1, None, w1, None, binding.Rotary(freqs.detach()))[0].sum().backward()
    assert torch.equal(p1.grad, got)
    with torch.no_grad():
        binding.NormRopeFunction.apply(p1, None, w1, None, binding.Rotary(freqs))
