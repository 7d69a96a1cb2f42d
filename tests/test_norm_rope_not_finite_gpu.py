"""Norm with rotation where a value is infinite or NaN: it reaches what its formula has it in, and nothing else."""
import math

import numpy as np
import pytest
import torch

from paper_2608_20172_gb300 import binding
from tests.test_norm_rope_gpu import BF16, Case, F32

pytestmark = pytest.mark.gpu
INF, NAN = math.inf, math.nan


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    binding.load()


def same(a, b):
    """The same bits, NaN like NaN."""
    return torch.equal(torch.nan_to_num(a, nan=77.0, posinf=88.0, neginf=99.0),
                       torch.nan_to_num(b, nan=77.0, posinf=88.0, neginf=99.0))


def cases(**kw):
    """Rows in 16-byte groups and element by element, either layout of the pairs, a part of a head turned
    (12: a group of bf16 in part) or none, and the first and the last channel that are not."""
    for layout in ("interleaved", "half"):
        for dtype in (BF16, F32):
            for d_rot, pad, channel in ((32, 0, 32), (32, 0, 63), (12, 0, 13), (12, 0, 61), (0, 0, 1), (32, 1, 32),
                                        (32, 1, 63), (0, 1, 62)):
                yield Case(7, 3, 2, 64, d_rot, layout, dtype, seed=3, pad=pad, scale=1.0, **kw), channel


@pytest.mark.parametrize("value", [INF, -INF, NAN])
def test_channels_that_are_not_turned_stay_by_themselves(value):
    """Without the norm only the channel's own result, with it and an infinity a row of zeros (1 / inf) but for
    the channel itself (inf / inf)."""
    for c, at in cases(norm=False):
        plain = c.forward()
        for t in c.tx:
            t[4, 1, at] = value
        for got, want, w in zip(c.forward(), plain, c.tw):
            want = want.clone()
            want[4, 1, at] = value * w[at]
            assert same(got, want), (c.rotary, at)
    for c, at in cases(norm=True):
        plain = c.forward()
        for t in c.tx:
            t[4, 1, at] = value
        for got, want in zip(c.forward(), plain):
            want = want.clone()
            want[4, 1] = NAN if math.isnan(value) else 0.0
            want[4, 1, at] = NAN
            assert same(got, want), (c.rotary, at)


@pytest.mark.parametrize("head", [0, 1])
@pytest.mark.parametrize("value", [INF, -INF, NAN])
def test_gradients_of_channels_that_are_not_turned_stay_by_themselves(value, head):
    """dy of such a channel goes to its own dw, and without the norm to its own dx."""
    for norm in (False, True):
        for c, at in cases(norm=norm):
            plain = c.backward()
            for t in c.tdy:
                t[4, head, at] = value
            got = c.backward()
            for i in range(2):
                want = plain[2 + i].clone()
                want[at] = value * c.tx[i][4, head, at]
                assert same(got[2 + i], want), (norm, c.rotary, at)
                want = plain[i].clone()
                if norm:  # (the mean reaches every channel of the row)
                    want[4, head], got[i][4, head] = 0.0, 0.0
                else:
                    want[4, head, at] = value * c.tw[i][at]
                assert same(got[i], want), (norm, c.rotary, at)


@pytest.mark.parametrize("value", [INF, -INF, NAN])
def test_without_the_norm_dx_does_not_depend_on_x(value):
    """dx = w u; x goes to its channel's dw alone."""
    for c, at in cases(norm=False):
        plain = c.backward()
        for t in c.tx:
            t[4, 1, at] = value
        got = c.backward()
        for i in range(2):
            assert torch.equal(got[i], plain[i]), (c.rotary, at)
            want = plain[2 + i].clone()
            want[at] = value * c.tdy[i][4, 1, at]
            assert same(got[2 + i], want), (c.rotary, at)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("H,d,pad", [(1, 64, 0), (3, 64, 0), (9, 64, 0), (5, 32, 0), (3, 33, 0), (3, 64, 1)])
def test_last_head_counts_once(H, d, pad, dtype):
    """Numbers of heads that do not fill a warp's passes: an infinity in the last one's x or dy makes its
    column of dw infinite."""
    for which, norm in (("x", False), ("dy", False), ("dy", True)):
        c = Case(6, H, H, d, 0, "half", dtype, seed=4, pad=pad, norm=norm)
        plain = c.backward()
        for i in range(2):
            (c.tx if which == "x" else c.tdy)[i][3, H - 1, 5] = INF
        got = c.backward()
        for i in range(2):
            other = (c.tdy if which == "x" else c.tx)[i][3, H - 1, 5]
            want = plain[2 + i].clone()
            want[5] = INF * float(torch.sign(other))
            assert float(other) != 0 and same(got[2 + i], want), (which, norm)
