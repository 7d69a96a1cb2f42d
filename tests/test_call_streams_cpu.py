"""A call with stream= allocates what it was not given in that stream's memory: scratch that goes back
to the allocator when the call returns is then reused in the stream's order, and an output waits for
the caller's stream as well before its memory is used again.  CPU only: stand-ins for the library, for
CUDA tensors and for the allocator's streams."""
import contextlib
from types import SimpleNamespace

import pytest
import torch

from paper_2608_20172_gb300 import binding

HERE = SimpleNamespace(cuda_stream=100)
F32, BF16, I32, I64 = torch.float32, torch.bfloat16, torch.int32, torch.int64


class OnGpu(torch.Tensor):
    """A CPU tensor that says it lives on cuda:0, with the stream whose memory it came from."""
    is_cuda = property(lambda self: True)
    device = property(lambda self: torch.device("cuda", 0))

    def get_device(self):
        return 0

    def record_stream(self, stream):
        self.__dict__.setdefault("recorded", []).append(stream.cuda_stream)


def on_gpu(t):
    return t.as_subclass(OnGpu)


class Library:
    """Every function succeeds; the pointers of the last call."""

    def __getattr__(self, name):
        def call(*args):
            if name.endswith("workspace_size"):
                return 64
            self.args = args
            return binding.OK
        return call


@pytest.fixture
def streams(monkeypatch):
    now = [HERE]
    made = []

    @contextlib.contextmanager
    def under(stream):
        now.append(stream)
        yield
        now.pop()

    def allocator(make):
        def f(*args, **kw):
            kw.pop("device", None)
            t = on_gpu(make(*args, **kw))
            t.owner = now[-1].cuda_stream
            made.append(t)
            return t
        return f

    plain = {n: getattr(torch, n) for n in ("empty", "empty_strided")}
    for n, make in plain.items():
        monkeypatch.setattr(torch, n, allocator(make))
    monkeypatch.setattr(torch, "empty_like", allocator(
        lambda t: plain["empty_strided"](t.size(), t.stride(), dtype=t.dtype)))
    monkeypatch.setattr(torch.cuda, "stream", under)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *_: now[-1])
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)

    def external(ptr, device=None):
        assert ptr != 0  # (torch takes 0 for a stream of its own choice)
        return SimpleNamespace(cuda_stream=ptr)
    monkeypatch.setattr(torch.cuda, "ExternalStream", external)
    monkeypatch.setattr(torch.cuda, "default_stream", lambda device=None: SimpleNamespace(cuda_stream=0))
    monkeypatch.setattr(binding, "_raw_stream", lambda device: now[-1].cuda_stream)
    monkeypatch.setattr(binding, "_calls", binding._NoCalls)
    monkeypatch.setattr(binding, "_lib", Library())
    return made


def calls():
    t = lambda *s, dtype=BF16: on_gpu(torch.zeros(s, dtype=dtype))  # noqa: E731
    x, f = t(2, 8, 4, 64), t(2, 8, 4, 64, dtype=F32)
    cut = on_gpu(torch.zeros((2, 8, 4, 80), dtype=BF16))[..., :64]
    wide = t(4, dtype=F32)[::2]  # theta that a call lays out anew
    m, z = t(2, 4, 8, dtype=F32), t(2, 4, 8, 64, dtype=F32)
    pages, tok = t(6, 16, 4, 64), t(3, 4, 64)
    i, table, u = t(2, dtype=I32), t(2, 3, dtype=I32), t(2, dtype=F32)
    b = binding
    return {
        "fwd": lambda **k: b.fwd(x, x, x, 0.5, **k),
        "fwd of a view": lambda **k: b.fwd(cut, cut, cut, 0.5, **k),
        "fwd_flow": lambda **k: b.fwd_flow(x, x, x, 0.5, **k),
        "linear_fwd": lambda **k: b.linear_fwd(x, x, x, f, **k),
        "fwd_state": lambda **k: b.fwd_state(x, x, x, True, **k),
        "state_finish": lambda **k: b.state_finish(x, x, x, (m, m, z), 0.5, **k),
        "linear_fwd_ws": lambda **k: b.linear_fwd_ws(x, x, x, f, **k),
        "linear_bwd": lambda **k: b.linear_bwd(x, x, x, f, x, **k),
        "layer_prep": lambda **k: b.layer_prep(x, x, x, wide, **k),
        "layer_grad": lambda **k: b.layer_grad(x, x, x, x, wide, **k),
        "decode": lambda **k: b.decode(x[:, 0], x, x, i, 0.5, **k),
        "page_plan": lambda **k: b.page_plan(i, i, table, t(6, dtype=I32), i, 16, 5, **k),
        "cache_append": lambda **k: b.cache_append(tok, tok, tok, u, t(3, dtype=I32), t(3, dtype=I64),
                                                   pages, pages, **k),
        "paged_decode": lambda **k: b.paged_decode(tok[:2], pages, pages, table, i, 0.5, **k),
        "sample": lambda **k: b.sample(t(2, 50), u, **k),
        "bwd": lambda **k: b.bwd(x, x, x, x, x, m, 0.5, **k),
    }


def flat(out):
    return [t for o in out for t in flat(o)] if isinstance(out, (tuple, list)) else [out]


@pytest.mark.parametrize("name", sorted(calls()))
@pytest.mark.parametrize("given,owner", [(SimpleNamespace(cuda_stream=8), 8), (8, 8), (0, 0), (1, 0)])
def test_allocations_belong_to_the_given_stream(streams, name, given, owner):
    copies = []
    contiguous = OnGpu.contiguous

    def contiguous_here(t):
        copies.append(torch.cuda.current_stream().cuda_stream)
        return contiguous(t)
    OnGpu.contiguous = contiguous_here
    try:
        out = flat(calls()[name](stream=given))
    finally:
        OnGpu.contiguous = contiguous
    assert streams and out
    assert {t.owner for t in streams} == {owner} and set(copies) <= {owner}
    for t in out:  # the caller's stream uses it after this one
        assert HERE.cuda_stream in t.__dict__.get("recorded", ()), name
    assert binding._lib.args[-1] == getattr(given, "cuda_stream", given)


@pytest.mark.parametrize("name", sorted(calls()))
@pytest.mark.parametrize("given", [None, HERE, HERE.cuda_stream])
def test_the_current_stream_needs_nothing_more(streams, name, given, monkeypatch):
    def never(*_):
        raise AssertionError("no other stream is entered")
    monkeypatch.setattr(torch.cuda, "stream", never)
    calls()[name](stream=given)
    assert {t.owner for t in streams} == {HERE.cuda_stream}
    assert not any("recorded" in t.__dict__ for t in streams)
    assert binding._lib.args[-1] == HERE.cuda_stream


def test_given_buffers_are_not_touched(streams):
    t = lambda *s, dtype=BF16: on_gpu(torch.zeros(s, dtype=dtype))  # noqa: E731
    q, pages = t(2, 4, 64), t(6, 16, 4, 64)
    out, logz, ws = t(2, 4, 64), t(2, 4, dtype=F32), t(64, dtype=torch.uint8)
    got = binding.paged_decode(q, pages, pages, t(2, 3, dtype=I32), t(2, dtype=I32), 0.5, out=out,
                               logz=logz, workspace=ws, stream=7)
    assert got[0] is out and got[1] is logz and not streams
    assert "recorded" not in out.__dict__ and binding._lib.args[-1] == 7
