"""Log probabilities without a GPU: bad arguments are refused with nothing launched; the plain 64-bit form
that the GPU tests compare with, against differences and by hand."""
import math

import numpy as np
import pytest
import torch

from paper_2608_20172_gb300 import binding
from paper_2608_20172_gb300 import build as libbuild
from tests import logprobs_util as lu

P = [0x10000 * (i + 1) for i in range(16)]  # aligned, never dereferenced here
INVALID, UNSUPPORTED, ALIGNMENT = (binding.ERR_INVALID_ARG, binding.ERR_UNSUPPORTED,
                                   binding.ERR_ALIGNMENT)


@pytest.fixture(scope="module")
def lib():
    libbuild.build()
    return binding.load()


def fwd(lib, p=None, R=4, V=100, stride=100, dt=binding.F32, top=4, status=None):
    q = list(P[:8]) if p is None else p  # logits, targets, temperature, logprob, entropy, logz, tokens, logps
    return lib.relation_logprobs(q[0], R, V, stride, dt, q[1], q[2], q[3], q[4], q[5], top, q[6], q[7],
                                 status, None)


def grad(lib, p=None, R=4, V=100, stride=100, dt=binding.F32, out_stride=100):
    q = list(P[:9]) if p is None else p
    # logits, targets, temperature, logz, entropy, dlogprob, dentropy, dlogz, dlogits
    return lib.relation_logprobs_grad(q[0], R, V, stride, dt, q[1], q[2], q[3], q[4], q[5], q[6], q[7], q[8],
                                      out_stride, None)


@pytest.mark.parametrize("kw,expect", [
    (dict(R=0), INVALID), (dict(V=0), INVALID), (dict(stride=99), INVALID), (dict(dt=2), INVALID),
    (dict(top=-1), INVALID), (dict(top=33), UNSUPPORTED), (dict(status=2), ALIGNMENT),
    (dict(V=(1 << 30) + 1, stride=1 << 31), UNSUPPORTED), (dict(R=1 << 28), UNSUPPORTED)])
def test_forward_refuses(lib, kw, expect):
    assert fwd(lib, **kw) == expect


@pytest.mark.parametrize("kw,expect", [
    (dict(R=0), INVALID), (dict(V=0), INVALID), (dict(stride=99), INVALID), (dict(dt=2), INVALID),
    (dict(out_stride=99), INVALID), (dict(V=(1 << 30) + 1, stride=1 << 31, out_stride=1 << 31), UNSUPPORTED),
    (dict(R=1 << 30), UNSUPPORTED)])
def test_gradient_refuses(lib, kw, expect):
    assert grad(lib, **kw) == expect


def test_refuses_pointers(lib):
    for i in range(8):
        p = list(P[:8])
        p[i] += 2
        assert fwd(lib, p) == ALIGNMENT, i
        if i != 2:
            p[i] = None
            assert fwd(lib, p) == INVALID, i
    for i in range(9):
        p = list(P[:9])
        p[i] += 2
        assert grad(lib, p) == ALIGNMENT, i
        if i not in (2, 5, 6, 7):
            p[i] = None
            assert grad(lib, p) == INVALID, i
    p = list(P[:9])
    p[8] = p[0]  # in place, but with rows elsewhere
    assert grad(lib, p, out_stride=104) == INVALID


def test_binding_refuses():
    x, t = torch.zeros(4, 10), torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError):  # not on a GPU
        binding.logprobs(x, t)
    with pytest.raises(ValueError):
        binding.logprobs_grad(x, t, x[:, 0], x[:, 0])
    with pytest.raises(TypeError):
        binding.logprobs(x.double(), t)


def test_plain_form_by_hand():
    x = np.log(np.array([0.1, 0.4, 0.2, 0.3]))
    lp, h, lz, tok, top = lu.row(x, 2, 1.0, 5)
    assert math.isclose(lp, math.log(0.2)) and abs(lz) < 1e-15 and tok == [1, 3, 2, 0, -1]
    assert math.isclose(h, -sum(p * math.log(p) for p in (0.1, 0.4, 0.2, 0.3)))
    assert np.allclose(top[:4], np.log([0.4, 0.3, 0.2, 0.1])) and top[4] == -math.inf
    assert math.isclose(lu.row(x, 1, 0.5)[0], math.log(0.16 / 0.30))
    inf = math.inf
    assert lu.row(np.array([-inf, -inf]), 0, 1.0, 1)[:4] == (-inf, 0.0, -inf, [-1])
    lp, h, lz, tok, _ = lu.row(np.array([inf, 1.0, inf]), 2, 1.0, 3)
    assert math.isclose(lp, -math.log(2)) and math.isclose(h, math.log(2)) and lz == inf and tok == [0, 2, 1]
    assert lu.row(np.array([0.0, 0.0, -inf]), -1, 1.0, 3)[3] == [0, 1, -1]


@pytest.mark.parametrize("target", [-1, 3])
def test_plain_gradient_against_differences(target):
    rng = np.random.default_rng(1)
    x = rng.standard_normal(9) * 2
    x[5] = -math.inf
    g, h, k, T = 0.7, -0.4, 0.2, 1.3
    f = lambda x: sum(c * v for c, v in zip((g, h, k), lu.row(x, target, T)[:3]))  # noqa: E731
    got, _ = lu.grad_row(x, target, T, g, h, k)
    for i in range(9):
        e = np.zeros(9)
        e[i] = 1e-6
        assert abs((f(x + e) - f(x - e)) / 2e-6 - got[i]) < 1e-8, i
