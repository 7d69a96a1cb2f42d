"""dev_status is written by the kernels: a call refuses one that is not an int32 of its operands' device
before it launches anything.  CPU only, with the stand-ins of test_call_streams_cpu.py."""
import pytest
import torch

from paper_2608_20172_gb300 import binding
from tests.test_call_streams_cpu import calls, on_gpu, streams  # noqa: F401

WITH_STATUS = sorted(set(calls()) - {"state_finish", "layer_prep", "layer_grad"})
EMPTY = on_gpu(torch.zeros(0, dtype=torch.int32))
WIDE, FLOAT = on_gpu(torch.zeros(1, dtype=torch.int64)), on_gpu(torch.zeros(1))
HOST = torch.zeros(1, dtype=torch.int32)


@pytest.mark.parametrize("name", WITH_STATUS)
@pytest.mark.parametrize("bad", [HOST, WIDE, FLOAT, EMPTY], ids=["host", "int64", "float", "empty"])
def test_bad_status_is_refused(streams, name, bad):  # noqa: F811
    with pytest.raises(ValueError):
        calls()[name](dev_status=bad)
    assert "args" not in vars(binding._lib)  # nothing was launched


@pytest.mark.parametrize("name", WITH_STATUS)
def test_good_status_is_passed_on(streams, name):  # noqa: F811
    status = on_gpu(torch.zeros(3, dtype=torch.int32))[1:]
    calls()[name](dev_status=status)
    assert status.data_ptr() in binding._lib.args


def test_self_test_and_fixed_scratch(streams):  # noqa: F811
    x, f = (on_gpu(torch.zeros((1, 8, 2, 64), dtype=t)) for t in (torch.bfloat16, torch.float32))
    for bad in (HOST, WIDE, EMPTY):
        with pytest.raises(ValueError):
            binding.selftest_wait_timeout(bad)
        with pytest.raises(ValueError):
            binding.bwd_no_alloc(x, x, x, x, x, f, 0.5, dq=x, dk=x, dv=x, dlambda=f, dev_status=bad)
    assert "args" not in vars(binding._lib)
