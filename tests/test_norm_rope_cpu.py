"""Norm with rotation without a GPU: bad arguments are refused with nothing launched; the frequency
tables; the plain 64-bit form that the GPU tests compare with, against differences and by hand."""
import math

import numpy as np
import pytest
import torch

from paper_2608_20172_gb300 import binding
from paper_2608_20172_gb300 import build as libbuild
from tests import norm_rope_util as nu

P = [0x10000 * (i + 1) for i in range(16)]  # aligned, never dereferenced here
INVALID, UNSUPPORTED, ALIGNMENT, WORKSPACE = (binding.ERR_INVALID_ARG, binding.ERR_UNSUPPORTED,
                                              binding.ERR_ALIGNMENT, binding.ERR_WORKSPACE)


@pytest.fixture(scope="module")
def lib():
    libbuild.build()
    return binding.load()


def shape(B=1, T=4, H=2, d=64, sB=512, sT=128, sH=64):
    return binding.Shape(B, T, H, d, sB, sT, sH)


def rot(freqs=P[8], d_rot=64, layout=0, scale=1.0):
    return binding.RotaryArgs(freqs, d_rot, layout, scale)


def fwd(lib, p=None, norm=1, eps=1e-6, r=None, sq=None, sk=None, dt=binding.BF16):
    q = list(P[:7]) if p is None else p  # p1, p2, w1, w2, positions, q, k
    return lib.relation_norm_rope(q[0], q[1], q[2], q[3], norm, eps, rot() if r is None else r, q[4], q[5],
                                  q[6], shape() if sq is None else sq, shape() if sk is None else sk, dt,
                                  None)


def grad(lib, p=None, norm=1, eps=1e-6, r=None, sq=None, sk=None, dt=binding.BF16, ws=1 << 30):
    q = list(P[:12]) if p is None else p  # dq, dk, p1, p2, w1, w2, positions, dp1, dp2, dw1, dw2, ws
    return lib.relation_norm_rope_grad(q[0], q[1], q[2], q[3], q[4], q[5], norm, eps,
                                       rot(P[12]) if r is None else r, q[6], q[7], q[8], q[9], q[10],
                                       shape() if sq is None else sq, shape() if sk is None else sk, dt,
                                       q[11], ws, None)


BAD = [(dict(norm=2), INVALID), (dict(norm=-1), INVALID), (dict(eps=-1e-6), INVALID),
       (dict(eps=float("nan")), INVALID), (dict(r=rot(d_rot=66)), INVALID), (dict(r=rot(d_rot=7)), INVALID),
       (dict(r=rot(d_rot=-2)), INVALID), (dict(r=rot(layout=2)), INVALID),
       (dict(r=rot(scale=float("inf"))), INVALID), (dict(r=rot(freqs=None)), INVALID),
       (dict(r=rot(freqs=P[8] + 4)), ALIGNMENT), (dict(dt=2), INVALID), (dict(sq=shape(B=0)), INVALID),
       (dict(sq=shape(T=0)), INVALID), (dict(sq=shape(H=0)), INVALID), (dict(sq=shape(d=0)), INVALID),
       (dict(sq=shape(sT=0)), INVALID), (dict(sk=shape(sH=0)), INVALID), (dict(sk=shape(T=5)), INVALID),
       (dict(sk=shape(d=32)), INVALID), (dict(sk=shape(H=0)), INVALID),
       (dict(sq=shape(d=257), sk=shape(d=257)), UNSUPPORTED),
       (dict(sq=shape(B=1 << 16, T=1 << 15), sk=shape(B=1 << 16, T=1 << 15)), UNSUPPORTED),
       (dict(sq=shape(H=1 << 25)), UNSUPPORTED)]


@pytest.mark.parametrize("call", [fwd, grad])
@pytest.mark.parametrize("kw,expect", BAD)
def test_refuses(lib, call, kw, expect):
    assert call(lib, **kw) == expect


def test_refuses_pointers(lib):
    for i, low, none in ((0, 1, INVALID), (1, 1, INVALID), (2, 2, None), (3, 2, None), (4, 2, None),
                         (5, 1, INVALID), (6, 1, INVALID)):
        p = list(P[:7])
        p[i] += low
        assert fwd(lib, p) == ALIGNMENT, i
        if none is not None:
            p[i] = None
            assert fwd(lib, p) == none, i
    for i, low, none in ((0, 1, INVALID), (1, 1, INVALID), (2, 1, INVALID), (3, 1, INVALID), (4, 2, None),
                         (6, 2, None), (7, 1, INVALID), (8, 1, INVALID), (9, 2, None), (10, 2, None),
                         (11, 8, WORKSPACE)):
        p = list(P[:12])
        p[i] += low
        assert grad(lib, p) == ALIGNMENT, i
        if none is not None:
            p[i] = None
            assert grad(lib, p) == none, i
    p = list(P[:12])
    p[1] = p[3] = p[8] = None  # no keys, but their weights' gradient
    assert grad(lib, p) == INVALID
    assert grad(lib, ws=64) == WORKSPACE


def test_workspace_size(lib):
    size = lib.relation_norm_rope_grad_workspace_size
    base = size(shape(T=1), binding.BF16)  # (of the head's width alone)
    assert 0 < base == size(shape(B=8, T=1 << 20), binding.F32) < 1 << 20
    assert size(shape(d=128), binding.BF16) == 2 * base
    for bad in (shape(B=0), shape(T=0), shape(d=257)):
        assert size(bad, binding.BF16) == 0


def test_binding_refuses():
    x = torch.zeros(4, 2, 64)
    with pytest.raises(ValueError):  # not on a GPU
        binding.norm_rope(x, None, None)
    for kw in (dict(d_rot=7), dict(d_rot=0), dict(d_rot=64, base=0.0), dict(d_rot=64, factor=0.5),
               dict(d_rot=64, layout="other"), dict(d_rot=64, scaling="other"),
               dict(d_rot=64, scaling="yarn", factor=4.0), dict(d_rot=2, scaling="ntk", factor=2.0)):
        with pytest.raises(ValueError):
            binding.rotary(device="cpu", **kw)


def test_frequencies():
    plain = binding.rotary(64, 1e4, device="cpu")
    assert plain.scale == 1.0 and plain.layout == "interleaved" and plain.freqs.dtype == torch.float64
    want = 1e4 ** (-np.arange(32) / 32.0)
    assert np.allclose(plain.freqs.numpy(), want, rtol=1e-14)
    assert np.allclose(binding.rotary(64, scaling="linear", factor=4.0, device="cpu").freqs.numpy(), want / 4)
    ntk = binding.rotary(64, scaling="ntk", factor=4.0, device="cpu").freqs.numpy()
    assert ntk[0] == 1.0 and math.isclose(ntk[-1], want[-1] / 4, rel_tol=1e-12)
    yarn = binding.rotary(64, scaling="yarn", factor=4.0, context=2048, layout="half", device="cpu")
    turns = 2048 * want / (2 * math.pi)
    f = yarn.freqs.numpy()
    assert np.allclose(f[turns > 32], want[turns > 32]) and np.allclose(f[turns < 1], want[turns < 1] / 4)
    between = (turns > 1) & (turns < 32)
    assert between.any() and (f[between] < want[between]).all() and (f[between] > want[between] / 4).all()
    assert math.isclose(yarn.scale, 1 + 0.1 * math.log(4)) and yarn.layout == "half"


def test_plain_form_by_hand():
    x = np.array([[[3.0, 4.0, 0.0, 5.0]]])  # mean square 12.5
    w = np.array([1.0, 2.0, 1.0, 1.0])
    quarter = np.array([math.pi / 2])
    y, _ = nu.norm_rope(x, w, np.array([1]), quarter, False, 2.0, True, 0.0)
    r = 1 / math.sqrt(12.5)
    assert np.allclose(y[0, 0], [-16 * r, 6 * r, 0, 5 * r])
    two = np.array([math.pi / 2, 0.0])
    y, _ = nu.norm_rope(x, np.ones(4), np.array([1]), two, True, 1.0, False, 0.0)
    assert np.allclose(y[0, 0], [0, 4, 3, 5])  # (0, 2) a quarter turn, (1, 3) as they are


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("norm", [False, True])
def test_plain_gradient_against_differences(half, norm):
    rng = np.random.default_rng(3)
    x, dy = rng.standard_normal((2, 3, 2, 10))
    w = rng.standard_normal(10)
    pos, freqs = np.array([0, 5, -1]), np.array([1.0, 0.3, 0.01])
    f = lambda x, w: (nu.norm_rope(x, w, pos, freqs, half, 1.2, norm, 1e-6)[0] * dy).sum()  # noqa: E731
    dx, dw, *_ = nu.norm_rope_grad(dy, x, w, pos, freqs, half, 1.2, norm, 1e-6)
    for got, at in ((dx, x), (dw, w)):
        for i in np.ndindex(at.shape):
            e = np.zeros_like(at)
            e[i] = 1e-6
            num = (f(x + e, w) - f(x - e, w) if at is x else f(x, w + e) - f(x, w - e)) / 2e-6
            assert abs(num - got[i]) < 1e-7, i
