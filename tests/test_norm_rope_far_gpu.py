"""Norm with rotation at the last positions: a turn is as exact there as at the first ones."""
from fractions import Fraction

import numpy as np
import pytest
import torch

from paper_2608_20172_gb300 import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
TWO_PI = 2 * Fraction("3.14159265358979323846264338327950288419716939937510582097494459230781640628620899862803")


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    binding.load()


def angle(position, freq):
    """position * freq modulo 2 pi, in whole numbers."""
    a = Fraction(int(position)) * Fraction(float(freq))
    return float(a - TWO_PI * round(a / TWO_PI))


@pytest.mark.parametrize("layout", ["interleaved", "half"])
@pytest.mark.parametrize("d_rot", [16, 256])
def test_last_positions(d_rot, layout):
    """A turn's angle, a part of a turn rounded to fp32, is off by pi u at most, its sine and cosine by 2 ulp of
    theirs, the factor, two products and their sum by one each: 11 u of |a| + |b|."""
    rng = np.random.default_rng(0)
    freqs = np.exp(rng.uniform(np.log(1e-9), np.log(1e5), d_rot // 2))
    freqs[:5] = 1.0, 0.5, 2.0 ** 0.5, 6.2831853, 99999.7
    freqs[5] = -3.3
    pos = np.array([0, 1, 2 ** 16 + 1, 2 ** 24 - 1, 2 ** 30 + 12345, 2 ** 31 - 1, 2 ** 31 - 7919], np.int32)
    x = rng.standard_normal((len(pos), 2, 256)).astype(np.float32)
    rot = binding.Rotary(torch.from_numpy(freqs).to(DEV), layout, 1.0)
    got, _ = binding.norm_rope(torch.from_numpy(x).to(DEV), None, rot, torch.from_numpy(pos).to(DEV), norm=False)
    got = got.double().cpu().numpy()
    p = np.arange(d_rot // 2)
    a, b = (p, p + d_rot // 2) if layout == "half" else (2 * p, 2 * p + 1)
    ang = np.array([[angle(m, f) for f in freqs] for m in pos])[:, None, :]
    xa, xb = x[..., a].astype(np.float64), x[..., b].astype(np.float64)
    tol = 12 * U * (np.abs(xa) + np.abs(xb))
    for channel, want in ((a, xa * np.cos(ang) - xb * np.sin(ang)), (b, xa * np.sin(ang) + xb * np.cos(ang))):
        err = np.abs(got[..., channel] - want)
        assert (err <= tol).all(), float((err / tol).max())
    assert np.array_equal(got[..., d_rot:], x[..., d_rot:].astype(np.float64))
