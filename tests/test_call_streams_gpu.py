"""Calls with stream= on the GPU: what they allocate stays theirs while the stream is still waiting, and
results keep their memory until the caller's stream has read them."""
import pytest
import torch

from paper_2608_20172_gb300 import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
WAIT = 20_000_000  # clocks: about 10 ms, far more than the host needs for what follows


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    binding.load()


def make():
    g = torch.Generator(device=DEV).manual_seed(5)
    r = lambda *s, dtype=torch.bfloat16: torch.randn(s, generator=g, device=DEV).to(dtype)  # noqa: E731
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    kp, vp, q = r(600, 16, 2, 64), r(600, 16, 2, 64), r(4, 8, 64)
    table = torch.arange(600, dtype=torch.int32, device=DEV).view(4, 150)
    lengths = i32([2400, 900, 1, 1777])
    kc, vc, long = r(4, 640, 8, 64), r(4, 640, 8, 64), i32([640, 3, 77, 500])
    x, u = r(5, 9000, dtype=torch.float32), torch.rand(5, generator=g, device=DEV)
    top_p = torch.full((5,), 0.9, device=DEV)
    toks, theta = [r(9, 2, 64) for _ in range(3)], torch.rand(1, generator=g, device=DEV)
    pos, slots = i32(list(range(9))), torch.arange(9, device=DEV) * 3
    k2, v2 = torch.zeros_like(kp), torch.zeros_like(vp)
    x4 = [r(1, 300, 2, 64) for _ in range(3)]
    return {
        "paged_decode": lambda **k: binding.paged_decode(q, kp, vp, table, lengths, 0.5, **k),
        "decode": lambda **k: binding.decode(q, kc, vc, long, 0.5, **k),
        "sample": lambda **k: binding.sample(x, u, top_p=top_p, **k),
        "cache_append": lambda **k: binding.cache_append(*toks, theta, pos, slots, k2, v2, **k),
        "fwd": lambda **k: binding.fwd(*x4, 0.5, **k),
    }


def flat(out):
    return [out] if isinstance(out, torch.Tensor) else list(out)


@pytest.mark.parametrize("raw", [False, True])
@pytest.mark.parametrize("name", ["paged_decode", "decode", "sample", "cache_append", "fwd"])
def test_nothing_else_gets_the_memory_meanwhile(name, raw):
    call = make()[name]
    want = [t.clone() for t in flat(call())]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(WAIT)
    got = flat(call(stream=side.cuda_stream if raw else side))
    sizes = [1 << n for n in range(9, 23)] + [t.numel() * t.element_size() for t in got]
    size = binding.paged_decode_workspace_size(torch.empty((4, 8, 64), device=DEV),
                                               torch.empty((1, 16, 2, 64), device=DEV))
    junk = [torch.full((n,), 0xff, dtype=torch.uint8, device=DEV) for n in sizes + [size] * 4]
    torch.cuda.synchronize()
    del junk
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_a_result_waits_for_its_reader():
    call = make()["paged_decode"]
    want = call()[0].clone()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    y = call(stream=side)[0]
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda._sleep(WAIT)
    seen = y.clone()
    del y
    with torch.cuda.stream(side):
        junk = [torch.full_like(want, 7.0) for _ in range(8)]
    torch.cuda.synchronize()
    del junk
    assert torch.equal(seen, want)


def test_the_default_stream_by_number():
    """Stream 0 from under another one: its memory, in its order."""
    call = make()["paged_decode"]
    want = call()[0].clone()
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        got = call(stream=0)[0]
    torch.cuda.synchronize()
    assert torch.equal(got, want)
