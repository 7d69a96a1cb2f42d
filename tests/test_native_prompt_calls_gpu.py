"""norm_rope, paged_chunk and logprobs, and the gradients, in native code and in Python: the same results, and
the native ones decline what the binding has to look at."""
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


def rand(*shape, dtype=torch.float32, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return torch.randn(shape, generator=g, device=DEV).to(dtype)


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def rope_args(view=False):
    both = rand(9, 6, 64, dtype=torch.bfloat16)
    p = (both[:, :4], both[:, 4:]) if view else (both[:, :4].contiguous(), both[:, 4:].contiguous())
    return [*p, binding.rotary(32, layout="half"), i32([3, 4, 5, -1, 0, 1, 2, 900, 901]), rand(64), rand(64)]


def chunk_args():
    k, v = (rand(6, 16, 2, 64, dtype=torch.bfloat16, seed=s) for s in (1, 2))
    return [rand(7, 4, 64, dtype=torch.bfloat16), k, v, i32([[0, 1, 2], [3, 4, 5]]), i32([0, 5, 6]),
            i32([20, 21, 22, 23, 24, 40, -1]), 0.5]


def logit_args():
    return [rand(5, 700), i32([3, -1, 699, 0, 7])]


def grad_args():
    x, t = logit_args()
    r = binding.logprobs(x, t)
    return [x, t, r.logz, r.entropy, rand(5, seed=3), None, rand(5, seed=4)]


CALLS = [("norm_rope", rope_args, {}), ("norm_rope", lambda: rope_args(True), {}),
         ("norm_rope", lambda: [rope_args()[0], None, None], {}),
         ("norm_rope", rope_args, dict(norm=False)), ("norm_rope", rope_args, dict(eps=0.5)),
         ("norm_rope_grad", lambda: [*(x.clone() for x in rope_args()[:2]), *rope_args()], {}),
         ("norm_rope_grad", lambda: [rope_args()[0], None, rope_args()[0], None, *rope_args()[2:]],
          dict(weights=False)),
         ("paged_chunk", chunk_args, {}), ("paged_chunk", chunk_args, dict(tau_s=1.5)),
         ("logprobs", logit_args, {}), ("logprobs", logit_args, dict(top=4)),
         ("logprobs", logit_args, dict(temperature=torch.full((5,), 0.7))),
         ("logprobs_grad", grad_args, {}), ("logprobs_grad", grad_args, dict(temperature=torch.full((5,), 0.7)))]


@pytest.mark.parametrize("name,make,kw", CALLS)
def test_native_and_python_agree(native, monkeypatch, name, make, kw):
    kw = {k: v.to(DEV) if isinstance(v, torch.Tensor) else v for k, v in kw.items()}
    taken, got = [], []
    real = getattr(native, name)
    spy = type("Spy", (binding._NoCalls,), {name: staticmethod(lambda *a: taken.append(real(*a)) or taken[-1])})
    for m in (spy, binding._NoCalls):
        monkeypatch.setattr(binding, "_calls", m)
        out = getattr(binding, name)(*make(), **kw)
        got.append([out] if isinstance(out, torch.Tensor) else list(out))
    assert taken[0] is not None  # the native call took it
    for a, b in zip(*got):
        assert (a is None) == (b is None)
        if a is not None:
            assert a.dtype == b.dtype and a.shape == b.shape and a.stride() == b.stride() and torch.equal(a, b)


def test_native_declines(native):
    p1, p2, rot, pos, w1, w2 = rope_args()
    args = lambda **kw: [v for v in {**dict(p1=p1, p2=p2, f=rot.freqs, layout=1, scale=1.0, pos=pos, w1=w1,  # noqa: E731
                                            w2=w2, norm=1, eps=1e-6), **kw}.values()]
    assert native.norm_rope(*args()) is not None
    for kw in (dict(p1=p1.half()), dict(p1=p1.cpu()), dict(p2=p2[:3]), dict(p2=p2.float()), dict(f=rot.freqs.float()),
               dict(layout=2), dict(pos=pos.long()), dict(pos=pos[:2]), dict(w1=w1[:9]), dict(norm=True),
               dict(eps=-1.0), dict(eps=None), dict(p1=p1.transpose(1, 2)), dict(p1="x")):
        assert native.norm_rope(*args(**kw)) is None, kw
    c = [*chunk_args(), 2.0, None]
    assert native.paged_chunk(*c) is not None
    for i, bad in ((0, c[0].float()), (0, c[0][..., :32]), (2, c[2][:, :8]), (3, c[3].t()), (4, c[4].long()),
                   (4, c[4][:1]), (5, c[5][:3]), (6, "x"), (7, 0.0), (8, torch.zeros(1, device=DEV))):
        assert native.paged_chunk(*c[:i], bad, *c[i + 1:]) is None, i
    x, t = logit_args()
    assert native.logprobs(x, t, None, 3, None) is not None
    for bad in ((x.t(), t, None, 3, None), (x, t.long(), None, 3, None), (x, t, None, 33, None),
                (x, t, None, -1, None), (x, t, t, 3, None), (x.half(), t, None, 3, None), (x, t, None, 3)):
        assert native.logprobs(*bad) is None
    g = grad_args()
    assert native.logprobs_grad(*g, None) is not None
    assert native.logprobs_grad(*g[:2], g[2].double(), *g[3:], None) is None


def test_refusals_reach_the_caller():
    """What the native call declines is refused by the binding, with its words."""
    p1, p2, rot, pos, w1, w2 = rope_args()
    with pytest.raises(ValueError, match="positions"):
        binding.norm_rope(p1, p2, rot, pos[:3])
    with pytest.raises(binding.RelationError, match="UNSUPPORTED"):
        binding.logprobs(*logit_args(), top=33)
    c = chunk_args()
    with pytest.raises(ValueError, match="starts"):
        binding.paged_chunk(*c[:4], c[4].long(), *c[5:])
