"""relation_norm_rope and its gradient against the definition in 64 bits: types, layouts of the pairs, parts
of a head, odd widths, strides, far positions, padding, in place, streams, capture, autograd."""
import numpy as np
import pytest
import torch

from paper_2608_20172_gb300 import binding
from tests import norm_rope_util as nu

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    binding.load()


def half_step(dtype):
    return torch.finfo(dtype).eps / 2 if dtype is BF16 else 2.0 ** -24


class Case:
    """Inputs of one call, on the GPU and as fp64 arrays."""

    def __init__(self, N, H, Hk, d, d_rot, layout, dtype, *, seed=0, pad=0, reach=5000, scale=1.1, norm=True,
                 eps=1e-6, head_major=False, weights=True):
        rng = np.random.default_rng(seed)
        self.norm, self.eps, self.half, self.scale, self.dtype = norm, eps, layout == "half", scale, dtype
        self.put = lambda a, H: self.strided(a, H, d, pad, head_major)
        self.pos = rng.integers(0, reach, N).astype(np.int32)
        if N > 3:
            self.pos[2] = -1
        self.positions = torch.from_numpy(self.pos).to(DEV)
        self.freqs = 1e4 ** (-np.arange(d_rot // 2) / max(1, d_rot // 2))
        self.rotary = binding.Rotary(torch.from_numpy(self.freqs).to(DEV), layout, scale) if d_rot else None
        self.x, self.dy, self.w, self.tx, self.tdy, self.tw = [], [], [], [], [], []
        for H in (H, Hk) if Hk else (H,):
            t = [self.put(torch.from_numpy(rng.standard_normal((N, H, d)) * k).to(dtype), H) for k in (2.0, 1.0)]
            w = (1 + 0.3 * rng.standard_normal(d)).astype(np.float32) if weights else np.ones(d, np.float32)
            self.tx.append(t[0])
            self.tdy.append(t[1])
            self.x.append(t[0].double().cpu().numpy())
            self.dy.append(t[1].double().cpu().numpy())
            self.w.append(w.astype(np.float64))
            self.tw.append(torch.from_numpy(w).to(DEV) if weights else None)
        if not Hk:
            self.tx.append(None), self.tdy.append(None), self.tw.append(None)

    @staticmethod
    def strided(t, H, d, pad, head_major):
        N = t.shape[0]
        if head_major:
            out = torch.full((H, N, d + pad), 7.0, dtype=t.dtype, device=DEV).transpose(0, 1)[..., :d]
        else:
            out = torch.full((N, H, d + pad), 7.0, dtype=t.dtype, device=DEV)[..., :d]
        return out.copy_(t)

    def forward(self, **kw):
        return binding.norm_rope(*self.tx, self.rotary, self.positions, *self.tw, norm=self.norm, eps=self.eps,
                                 **kw)

    def backward(self, **kw):
        return binding.norm_rope_grad(*self.tdy, *self.tx, self.rotary, self.positions, *self.tw,
                                      norm=self.norm, eps=self.eps, **kw)

    def check(self, outs):
        step = half_step(self.dtype)
        for x, w, got in zip(self.x, self.w, outs):
            want, tol = nu.norm_rope(x, w, self.pos, self.freqs if self.rotary else np.zeros(0), self.half,
                                     self.scale, self.norm, self.eps)
            err = np.abs(got.double().cpu().numpy() - want)
            assert (err <= step * np.abs(want) * 1.01 + tol + 1e-37).all(), float((err - tol).max())

    def check_grad(self, outs):
        step = half_step(self.dtype)
        for i, (x, dy, w) in enumerate(zip(self.x, self.dy, self.w)):
            dx, dw, tol, wtol = nu.norm_rope_grad(dy, x, w, self.pos, self.freqs if self.rotary else np.zeros(0),
                                                  self.half, self.scale, self.norm, self.eps)
            err = np.abs(outs[i].double().cpu().numpy() - dx)
            assert (err <= step * np.abs(dx) * 1.01 + tol + 1e-37).all(), float((err - tol).max())
            if outs[2 + i] is not None:
                err = np.abs(outs[2 + i].double().cpu().numpy() - dw)
                assert (err <= wtol + 2.0 ** -24 * np.abs(dw)).all(), float((err - wtol).max())


SHAPES = [  # N, H, Hk, d, d_rot
    (1, 1, 1, 64, 64), (1, 12, 12, 64, 64), (5, 8, 2, 128, 128), (33, 4, 4, 128, 64), (7, 3, 1, 80, 40),
    (9, 2, 2, 96, 32), (6, 4, 1, 256, 256), (3, 2, 1, 8, 8), (4, 5, 5, 48, 12), (17, 2, 1, 72, 36),
    (3, 2, 2, 33, 10), (2, 1, 1, 1, 0), (5, 2, 2, 2, 2), (4, 3, 3, 255, 254), (130, 16, 0, 64, 16),
    (6, 2, 1, 64, 0), (700, 2, 1, 32, 32)]


@pytest.mark.parametrize("layout", ["interleaved", "half"])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N,H,Hk,d,d_rot", SHAPES)
def test_forward_and_gradient(N, H, Hk, d, d_rot, layout, dtype):
    c = Case(N, H, Hk, d, d_rot, layout, dtype)
    c.check(c.forward())
    c.check_grad(c.backward())


@pytest.mark.parametrize("layout", ["interleaved", "half"])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("kw", [dict(pad=8), dict(pad=1), dict(head_major=True), dict(norm=False),
                                dict(weights=False), dict(norm=False, weights=False), dict(eps=0.5),
                                dict(reach=2 ** 31 - 1), dict(scale=-0.7)])
def test_forms(kw, dtype, layout):
    c = Case(19, 6, 2, 64, 32, layout, dtype, seed=1, **kw)
    c.check(c.forward())
    c.check_grad(c.backward(weights=kw.get("weights", True)))


@pytest.mark.parametrize("layout", ["interleaved", "half"])
def test_batch_without_positions(layout):
    """[B, T, H, d] with positions 0 .. T - 1 in every sequence, both from one projection's columns."""
    rng = np.random.default_rng(5)
    B, T, H, Hk, d = 3, 21, 4, 2, 64
    both = torch.from_numpy(rng.standard_normal((B, T, H + Hk, d))).to(BF16).to(DEV)
    rotary = binding.rotary(d, layout=layout, scaling="yarn", factor=4.0, context=16)
    q, k = binding.norm_rope(both[:, :, :H], both[:, :, H:], rotary)
    pos = np.tile(np.arange(T, dtype=np.int32), B)
    for got, x in ((q, both[:, :, :H]), (k, both[:, :, H:])):
        assert got.shape == x.shape and got.stride() == x.stride()
        n = x.double().cpu().numpy().reshape(B * T, -1, d)
        want, tol = nu.norm_rope(n, np.ones(d), pos, rotary.freqs.cpu().numpy(), layout == "half",
                                 rotary.scale, True, 1e-6)
        err = np.abs(got.double().cpu().numpy().reshape(want.shape) - want)
        assert (err <= 2.0 ** -8 * 1.01 * np.abs(want) + tol).all()


@pytest.mark.parametrize("d,pad", [(64, 0), (33, 0)])
def test_in_place_and_neighbours(d, pad):
    c = Case(11, 3, 1, d, 32, "half", F32, pad=3)
    want, wide = c.forward(), [t.as_strided((t.shape[0], t.shape[1], d + 3), t.stride()) for t in c.tx]
    kept = c.tx[0].clone(), c.tx[1].clone()
    grads = c.backward()
    dp1, dp2, *_ = binding.norm_rope_grad(*c.tdy, *c.tx, c.rotary, c.positions, *c.tw, eps=c.eps)
    c.forward(out=tuple(c.tx))
    for got, w, t in zip(c.tx, want, wide):
        assert torch.equal(got, w) and (t[..., d:] == 7).all()
    c.tx[0].copy_(kept[0]), c.tx[1].copy_(kept[1])
    assert all(torch.equal(a, b) for a, b in zip(grads, c.backward()))  # the same bits again
    assert torch.equal(dp1, grads[0]) and torch.equal(dp2, grads[1])


@pytest.mark.parametrize("layout", ["interleaved", "half"])
def test_nan_and_infinity_stay_in_their_row(layout):
    c = Case(9, 4, 2, 64, 64, layout, BF16)
    plain = c.forward()
    c.tx[0][4, 1, 7] = float("nan")
    c.tx[1][5, 0, 3] = float("inf")
    q, k = c.forward()
    assert torch.isnan(q[4, 1]).all() and torch.isnan(k[5, 0]).any()
    q[4, 1], k[5, 0] = plain[0][4, 1], plain[1][5, 0]
    assert torch.equal(q, plain[0]) and torch.equal(k, plain[1])


def test_zero_rows():
    """A row of zeros is zeros, its gradient that of eps alone."""
    c = Case(5, 2, 2, 64, 64, "half", F32, eps=1e-6)
    for t in c.tx:
        t.zero_()
    c.x = [np.zeros_like(x) for x in c.x]
    assert all((t == 0).all() for t in c.forward())
    c.check_grad(c.backward())


def test_many_tokens_and_heads():
    """Past the CTAs that keep partial sums, and rows of many heads."""
    c = Case(9001, 2, 1, 16, 16, "interleaved", BF16, seed=2)
    c.check(c.forward())
    c.check_grad(c.backward())
    c = Case(3, 301, 77, 40, 20, "half", F32, seed=3)
    c.check(c.forward())
    c.check_grad(c.backward())


def test_stream_and_capture():
    c = Case(300, 8, 4, 64, 64, "half", BF16)
    want, grads = c.forward(), c.backward()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got, back = c.forward(stream=s), c.backward(stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert all(torch.equal(a, b) for a, b in zip(want + grads, got + back))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got, back = c.forward(), c.backward()
    for t in c.tx + c.tdy:
        t.neg_()
    g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(-a, b) for a, b in zip(want + grads[:2], got + back[:2]))
    assert all(torch.equal(a, b) for a, b in zip(grads[2:], back[2:]))


def test_autograd():
    c = Case(12, 4, 2, 64, 32, "half", F32)
    p1, p2, w1, w2 = (t.detach().clone().requires_grad_() for t in (*c.tx, *c.tw))
    q, k = binding.NormRopeFunction.apply(p1, p2, w1, w2, c.rotary, c.positions)
    (q * c.tdy[0]).sum().add((k * c.tdy[1]).sum()).backward()
    c.check_grad([p1.grad, p2.grad, w1.grad, w2.grad])
    # a layout of its own for the gradient, no keys, no weights
    p1 = c.tx[0].detach().clone().requires_grad_()
    q, k = binding.NormRopeFunction.apply(p1, None, None, None, c.rotary, c.positions)
    assert k is None
    q.transpose(0, 1).backward(c.tdy[0].transpose(0, 1))
    want = binding.norm_rope_grad(c.tdy[0], None, c.tx[0], None, c.rotary, c.positions, weights=False)
    assert torch.equal(p1.grad, want[0])


def test_gradient_against_differences_of_the_kernel():
    """Along a random direction: central differences of the fp32 kernel with steps of 2^-10.  Its 15360 outputs
    of about 1 carry roundings of 2^-24, so the slope is off by sqrt(15360) 2^-24 2^9 = 0.004; its terms add up
    to a size of tens."""
    c = Case(40, 4, 2, 64, 64, "half", F32, seed=8)
    g = torch.Generator(device=DEV).manual_seed(0)
    dirs = [torch.randn(t.shape, generator=g, device=DEV) for t in (*c.tx, *c.tw)]
    f = lambda s: sum((o.double() * d.double()).sum() for o, d in zip(binding.norm_rope(  # noqa: E731
        *(t + s * v for t, v in zip(c.tx, dirs)), c.rotary, c.positions,
        *(t + s * v for t, v in zip(c.tw, dirs[2:])), eps=c.eps), c.tdy))
    slope = float(f(2.0 ** -10) - f(-2.0 ** -10)) * 2.0 ** 9
    terms = [(g.double() * v.double()).sum() for g, v in zip(c.backward(), dirs)]
    size = float(sum((g.double() * v.double()).square().sum() for g, v in zip(c.backward(), dirs)).sqrt())
    assert abs(slope - float(sum(terms))) < 0.01 * size


def test_binding_refuses():
    c = Case(4, 2, 2, 64, 64, "half", F32)
    with pytest.raises(ValueError):
        binding.norm_rope(c.tx[0], c.tx[1].bfloat16(), c.rotary)
    with pytest.raises(ValueError):
        binding.norm_rope(c.tx[0], c.tx[1][:3], c.rotary)
    with pytest.raises(ValueError):
        binding.norm_rope(c.tx[0], None, binding.Rotary(c.rotary.freqs.float()))
    with pytest.raises(ValueError):
        binding.norm_rope(c.tx[0], None, c.rotary._replace(layout="other"))
    with pytest.raises(ValueError):
        binding.norm_rope(c.tx[0], None, c.rotary, c.positions.long())
    with pytest.raises(ValueError):
        binding.norm_rope(c.tx[0], None, c.rotary, w1=c.tw[0].double())
    with pytest.raises(ValueError):
        binding.norm_rope(c.tx[0].transpose(1, 2), None, c.rotary)
    with pytest.raises(ValueError):
        binding.norm_rope_grad(c.tdy[0], None, *c.tx, c.rotary)
    with pytest.raises(binding.RelationError):
        binding.norm_rope(c.tx[0][:, :, :32].contiguous(), None, c.rotary)  # wider than the head
    with pytest.raises(TypeError):
        binding.norm_rope(c.tx[0].half(), None, c.rotary)
