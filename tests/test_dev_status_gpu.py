"""dev_status of the serving calls: the native calls leave one that the kernels may not write to the
binding, which refuses it; one in pinned host memory goes its way."""
import pytest
import torch

from paper_2608_20172_gb300 import binding
from tests.test_native_calls_gpu import (DEV, decode_args, native, plan_args, sample_args,  # noqa: F401
                                         token_args)

pytestmark = pytest.mark.gpu


def calls():
    (x, u), kw = sample_args()
    return {"page_plan": lambda s: binding.page_plan(*plan_args(), dev_status=s),
            "cache_append": lambda s: binding.cache_append(*token_args(), dev_status=s),
            "paged_decode": lambda s: binding.paged_decode(*decode_args(), dev_status=s),
            "sample": lambda s: binding.sample(x, u, dev_status=s, **kw)}


@pytest.mark.parametrize("name", ["page_plan", "cache_append", "paged_decode", "sample"])
def test_refused(native, name):  # noqa: F811
    call = calls()[name]
    for bad in (torch.zeros(1, dtype=torch.int32), torch.zeros(1, dtype=torch.int64, device=DEV),
                torch.zeros(0, dtype=torch.int32, device=DEV), torch.zeros(1, device=DEV)):
        with pytest.raises(ValueError):
            call(bad)


def test_native_declines(native):  # noqa: F811
    (x, u), _ = sample_args()
    for bad in (torch.zeros(1, dtype=torch.int32), torch.zeros(1, dtype=torch.int64, device=DEV),
                torch.zeros(0, dtype=torch.int32, device=DEV)):
        assert native.page_plan(*plan_args(), bad) is None
        assert native.cache_append(*token_args(), 0, 1e4, bad) is None
        assert native.paged_decode(*decode_args(), 2.0, bad) is None
        assert native.sample(x, u, None, None, None, None, bad) is None


def test_written(native):  # noqa: F811
    """A bad temperature is reported on the device, past a view's offset, and in pinned host memory."""
    (x, u), _ = sample_args()
    cold = torch.full((3,), -1.0, device=DEV)
    for status in (torch.zeros(3, dtype=torch.int32, device=DEV)[1:],
                   torch.zeros(1, dtype=torch.int32).pin_memory()):
        binding.sample(x, u, temperature=cold, dev_status=status)
        torch.cuda.synchronize()
        assert int(status[0].item()) == binding.ERR_INVALID_ARG
