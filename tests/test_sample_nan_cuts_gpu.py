"""relation_sample with NaN cuts: a NaN top_p or min_p keeps every token, as without the cut."""
import pytest
import torch

from paper_2608_20172_gb300 import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("V,dtype", [(300, torch.float32), (40000, torch.float32), (9000, torch.bfloat16)])
@pytest.mark.parametrize("top_k", [None, 50])
def test_nan_cut_is_no_cut(V, dtype, top_k):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    binding.load()
    g = torch.Generator(device=DEV).manual_seed(V)
    x = torch.randn((64, V), generator=g, device=DEV).to(dtype)
    u = torch.rand(64, generator=g, device=DEV)
    nan = torch.full((64,), float("nan"), device=DEV)
    k = None if top_k is None else torch.full((64,), top_k, dtype=torch.int32, device=DEV)
    want = binding.sample(x, u, top_k=k)
    assert want[0].unique().numel() > 8
    for kw in (dict(top_p=nan), dict(min_p=nan), dict(top_p=nan, min_p=nan)):
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        got = binding.sample(x, u, top_k=k, dev_status=status, **kw)
        assert int(status.item()) == 0
        for a, b in zip(got, want):
            assert torch.equal(a, b)
