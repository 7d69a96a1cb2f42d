"""The serving calls in native code (csrc/torch_calls.cpp) and in Python: the same results, and the
native ones decline what the binding has to look at."""
import pytest
import torch

from paper_2608_20172_gb300 import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def native():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    m = binding._native()
    assert m is not binding._NoCalls, "relation_calls.so is not built"
    return m


def plan_args():
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    return [i32([5, 0, 30]), i32([1, 7, -1]), i32([[3, -1, -1], [-1, -1, -1], [4, 5, -1]]),
            torch.arange(6, dtype=torch.int32, device=DEV), i32([2, 3]), 16, 9]


def token_args(layout="nhd"):
    g = torch.Generator(device=DEV).manual_seed(1)
    x = [torch.randn((9, 4, 64), generator=g, device=DEV, dtype=torch.bfloat16) for _ in range(3)]
    kp, vp = (torch.zeros((6, 16, 4, 64), device=DEV, dtype=torch.bfloat16) for _ in range(2))
    return x + [torch.rand(2, generator=g, device=DEV), torch.arange(9, dtype=torch.int32, device=DEV),
                torch.arange(9, device=DEV) * 3, kp, vp]


def decode_args():
    g = torch.Generator(device=DEV).manual_seed(2)
    kp, vp = (torch.randn((6, 16, 2, 64), generator=g, device=DEV, dtype=torch.bfloat16)
              for _ in range(2))
    table = torch.tensor([[0, 1, 2], [3, 4, 5]], dtype=torch.int32, device=DEV)
    return [torch.randn((2, 4, 64), generator=g, device=DEV, dtype=torch.bfloat16), kp, vp, table,
            torch.tensor([40, 7], dtype=torch.int32, device=DEV), 0.5]


def sample_args():
    g = torch.Generator(device=DEV).manual_seed(3)
    return [torch.randn((3, 500), generator=g, device=DEV), torch.rand(3, generator=g, device=DEV)], {
        "temperature": torch.full((3,), 0.8, device=DEV),
        "top_k": torch.full((3,), 20, dtype=torch.int32, device=DEV),
        "top_p": torch.full((3,), 0.9, device=DEV)}


def outputs(out):
    return [out] if isinstance(out, torch.Tensor) else list(out)


def test_native_and_python_agree(native, monkeypatch):
    def both(call, make, kw=None):
        got = []
        for m in (native, binding._NoCalls):
            monkeypatch.setattr(binding, "_calls", m)
            status = torch.zeros(1, dtype=torch.int32, device=DEV)
            args = make()
            out = call(*args, dev_status=status, **(kw or {}))
            got.append((type(out), outputs(out) + [a for a in args if isinstance(a, torch.Tensor)] +
                        [status]))
        assert got[0][0] is got[1][0]
        for a, b in zip(got[0][1], got[1][1]):
            assert a.dtype == b.dtype and a.shape == b.shape and a.stride() == b.stride()
            assert torch.equal(a, b)

    both(binding.page_plan, plan_args)
    both(binding.cache_append, token_args)
    both(binding.paged_decode, decode_args)
    args, kw = sample_args()
    both(binding.sample, lambda: args, kw)
    both(binding.sample, lambda: args)


def test_native_takes_the_common_calls(native):
    a = plan_args()
    assert len(native.page_plan(*a, None)) == 5
    t = token_args()
    assert native.cache_append(*t, 0, 1e4, None).shape == (9, 4, 64)
    assert native.cache_append(*t[:3], None, *t[4:], 1, 10000, None) is not None
    assert len(native.paged_decode(*decode_args(), 2.0, None)) == 2
    (x, u), kw = sample_args()
    assert len(native.sample(x, u, kw["temperature"], kw["top_k"], kw["top_p"], None, None)) == 3


def test_native_declines(native):
    a = plan_args()
    for i, bad in ((0, a[0].cpu()), (1, a[1][:2]), (2, a[2].T), (3, a[3].long()), (4, a[4][:1]),
                   (5, 16.0), (6, 0), (6, -1), (6, 1 << 40), (0, None), (0, 3)):
        b = list(a)
        b[i] = bad
        assert native.page_plan(*b, None) is None, i
    t = token_args()
    for i, bad in ((0, t[0].float()), (1, t[1][:8]), (2, t[2].cpu()), (3, t[3].double()), (4, t[4][:3]),
                   (5, t[5].int()), (6, t[6][:2]), (7, t[7].float()), (0, None),
                   (0, t[0].transpose(0, 1).contiguous().transpose(0, 1))):
        b = list(t)
        b[i] = bad
        assert native.cache_append(*b, 0, 1e4, None) is None, i
    assert native.cache_append(*t, 2, 1e4, None) is None  # (refused by the library)
    d = decode_args()
    for i, bad in ((0, d[0].float()), (0, d[0][:, :3]), (1, d[1][:2]), (3, d[3].long()), (4, d[4][:1]),
                   (5, "x"), (5, float("nan"))):
        b = list(d)
        b[i] = bad
        assert native.paged_decode(*b, 2.0, None) is None, i
    (x, u), kw = sample_args()
    for args in ((x.T, u, None, None, None, None, None), (x.double(), u, None, None, None, None, None),
                 (x, u[:2], None, None, None, None, None), (x, u, u[:1], None, None, None, None),
                 (x, u, None, u, None, None, None), (x[0], u, None, None, None, None, None),
                 (x, u)):
        assert native.sample(*args) is None


def test_views_and_parameters_go_the_other_way():
    """A strided query, a Parameter and a non-contiguous table still work through the binding."""
    d = decode_args()
    want = binding.paged_decode(*d)
    wide = torch.zeros((2, 4, 80), device=DEV, dtype=torch.bfloat16)
    wide[:, :, :64] = d[0]
    got = binding.paged_decode(wide[:, :, :64], *d[1:])
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    t = token_args()
    want = binding.cache_append(*t)
    t[3] = torch.nn.Parameter(t[3])
    assert torch.equal(binding.cache_append(*t), want)


def test_current_stream_is_used(native):
    """Calls made under another stream follow what that stream does before them."""
    d = decode_args()
    want = binding.paged_decode(*d)[0]
    side = torch.cuda.Stream()
    k = torch.empty_like(d[1])
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
        k.copy_(d[1])
        got = binding.paged_decode(d[0], k, *d[2:])[0]
    side.synchronize()
    assert torch.equal(got, want)
