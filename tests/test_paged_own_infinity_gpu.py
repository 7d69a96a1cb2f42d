"""relation_paged_decode where the token's own value is infinite: Y = (1 - g) v_self + g sum p v with
0 < g < 1 is that infinity, NaN where the history's is the opposite one."""
import numpy as np
import pytest
import torch

from tests.test_paged_infinity_gpu import FORMS, INF, _lib, run  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [1, 2, 40, 66, 1200])
@pytest.mark.parametrize("dtype,H,Hk,d,pad", FORMS)
def test_own_value(dtype, H, Hk, d, pad, n):
    plain, y = run(n, H, Hk, d, dtype, [(n - 1, Hk - 1, 3, INF), (n - 1, Hk - 1, d - 1, -INF)], pad)
    mine = np.arange(H) // (H // Hk) == Hk - 1
    assert (y[mine, 3] == INF).all() and (y[mine, d - 1] == -INF).all()
    other = np.ones((H, d), bool)
    other[np.ix_(mine, [3, d - 1])] = False
    assert np.array_equal(y[other], plain[other])


@pytest.mark.parametrize("own,want", [(INF, INF), (-INF, float("nan"))])
@pytest.mark.parametrize("n", [40, 1200])
@pytest.mark.parametrize("dtype,H,Hk,d,pad", FORMS)
def test_own_value_and_the_history(dtype, H, Hk, d, pad, n, own, want):
    _, y = run(n, H, Hk, d, dtype, [(n - 1, 0, 1, own), (7, 0, 1, INF)], pad)
    mine = np.arange(H) // (H // Hk) == 0
    np.testing.assert_array_equal(y[mine, 1], np.full(mine.sum(), want, np.float32))



@pytest.mark.parametrize("n", [40, 1200])
@pytest.mark.parametrize("dtype,H,Hk,d,pad", FORMS)
def test_own_nan(dtype, H, Hk, d, pad, n):
    """NaN among the token's own values stays in its channel, beside an infinity in another."""
    plain, y = run(n, H, Hk, d, dtype, [(n - 1, 0, 1, float("nan")), (n - 1, 0, 2, INF)], pad)
    mine = np.arange(H) // (H // Hk) == 0
    assert np.isnan(y[mine, 1]).all() and (y[mine, 2] == INF).all()
    other = np.ones((H, d), bool)
    other[np.ix_(mine, [1, 2])] = False
    assert np.array_equal(y[other], plain[other])
