"""A call runs on the current device's streams: operands on another device are refused before anything
is launched.  CPU only, with the stand-ins of test_call_streams_cpu.py (operands on cuda:0)."""
import pytest
import torch

from paper_2608_20172_gb300 import binding
from tests.test_call_streams_cpu import calls, on_gpu, streams  # noqa: F401


@pytest.mark.parametrize("name", sorted(calls()))
@pytest.mark.parametrize("given", [None, 100, 7])
def test_operands_off_the_current_device(streams, name, given, monkeypatch):  # noqa: F811
    call = calls()[name]
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    with pytest.raises(ValueError, match="current device"):
        call(stream=given)
    assert "args" not in vars(binding._lib)  # nothing was launched


def test_calls_without_allocations(streams, monkeypatch):  # noqa: F811
    x, f = (on_gpu(torch.zeros((1, 8, 2, 64), dtype=t)) for t in (torch.bfloat16, torch.float32))
    m, z = on_gpu(torch.zeros((1, 2, 8))), on_gpu(torch.zeros((1, 2, 8, 64)))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    with pytest.raises(ValueError, match="current device"):
        binding.state_merge((m, m, z), (m, m, z))
    with pytest.raises(ValueError, match="current device"):
        binding.bwd_no_alloc(x, x, x, x, x, f, 0.5, dq=x, dk=x, dv=x, dlambda=f)
    assert "args" not in vars(binding._lib)
