"""relation_paged_chunk without a GPU: bad arguments are refused with nothing launched; the size query; the
plain 64-bit rows that the GPU tests compare with, against the oracle."""
import numpy as np
import pytest
import torch

import oracle
from paper_2608_20172_gb300 import binding
from paper_2608_20172_gb300 import build as libbuild
from tests import chunk_util as cu

P = [0x10000 * (i + 1) for i in range(16)]  # aligned, never dereferenced here
INVALID, UNSUPPORTED, ALIGNMENT, WORKSPACE = (binding.ERR_INVALID_ARG, binding.ERR_UNSUPPORTED,
                                              binding.ERR_ALIGNMENT, binding.ERR_WORKSPACE)


@pytest.fixture(scope="module")
def lib():
    libbuild.build()
    return binding.load()


def pages(n=10, page=16, H=2, d=64, sP=None, sR=None, sH=None):
    sH = d if sH is None else sH
    sR = H * d if sR is None else sR
    return binding.Pages(n, page, H, d, page * H * d if sP is None else sP, sR, sH)


def chunk(lib, p=None, N=8, B=2, H=2, cols=8, stride=8, c=None, dt=binding.BF16, lam=0.5, tau=2.0, ws=1 << 32,
          sT=128, sH=64, status=None):
    q = list(P[:9]) if p is None else p  # q, k, v, table, starts, positions, o, logz, workspace
    return lib.relation_paged_chunk(q[0], q[1], q[2], q[3], cols, stride, q[4], q[5], q[6], q[7], lam, tau, N, B,
                                    H, pages() if c is None else c, sT, sH, dt, q[8], ws, status, None)


@pytest.mark.parametrize("kw,expect", [
    (dict(N=0), INVALID), (dict(B=0), INVALID), (dict(H=3), INVALID), (dict(H=0), INVALID),
    (dict(cols=0), INVALID), (dict(stride=7), INVALID), (dict(dt=2), INVALID), (dict(sT=0), INVALID),
    (dict(sH=-1), INVALID), (dict(lam=float("inf")), INVALID), (dict(tau=0.0), INVALID),
    (dict(tau=float("nan")), INVALID), (dict(c=pages(n=0)), INVALID), (dict(c=pages(page=0)), INVALID),
    (dict(c=pages(sR=0)), INVALID), (dict(c=pages(d=129)), UNSUPPORTED),
    (dict(c=pages(page=1 << 28), cols=8), UNSUPPORTED), (dict(N=1 << 30, H=4), UNSUPPORTED),
    (dict(B=1 << 30, H=4), UNSUPPORTED), (dict(ws=64), WORKSPACE), (dict(status=2), ALIGNMENT)])
def test_refuses(lib, kw, expect):
    assert chunk(lib, **kw) == expect


def test_refuses_pointers(lib):
    for i, low in ((0, 1), (1, 1), (2, 1), (3, 2), (4, 2), (5, 2), (6, 1), (7, 2), (8, 8)):
        p = list(P[:9])
        p[i] += low
        assert chunk(lib, p) == ALIGNMENT, i
        p[i] = None
        assert chunk(lib, p) == (WORKSPACE if i == 8 else INVALID), i


def test_workspace_size(lib):
    size = lib.relation_paged_chunk_workspace_size
    small = size(1, 1, 2, 8, pages(), binding.BF16)
    assert 0 < small < 1 << 16  # 128 rows of a table: one piece
    long = size(1, 1, 2, 10000, pages(), binding.BF16)
    assert small < long < 1 << 20  # rows of one token
    prompt = size(1 << 15, 64, 32, 10000, pages(H=32), binding.BF16)
    # partial results of at most 608 pieces of 128 rows, and the plan
    assert prompt < 608 * 128 * 68 * 4 + (1 << 22)
    assert size(1 << 15, 64, 32, 20000, pages(H=32), binding.BF16) == prompt
    for bad in ((0, 1, 2, 8, pages()), (1, 0, 2, 8, pages()), (1, 1, 3, 8, pages()), (1, 1, 2, 0, pages()),
                (1, 1, 2, 8, pages(d=129))):
        assert size(*bad, binding.BF16) == 0


def test_binding_refuses():
    x = torch.zeros(1, 16, 2, 64)
    i = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError):  # not on a GPU
        binding.paged_chunk(torch.zeros(1, 2, 64), x, x, i[None], i, i[:1], 0.5)


def test_plain_rows_against_the_oracle():
    rng = np.random.default_rng(0)
    T, H, d = 23, 2, 8
    q, k, v = rng.standard_normal((3, T, H, d))
    Y, Z, W, big = cu.rows(q, np.arange(T), k, v, 0.7)
    for h in range(H):
        want = oracle.fwd(*(np.ascontiguousarray(x[:, h]) for x in (q, k, v)), 0.7, 2.0)
        assert np.allclose(Y[:, h], want[0], atol=1e-12) and np.allclose(Z[:, h], want[1], atol=1e-12)
    # a key head that two query heads share; padding
    Y2, Z2, *_ = cu.rows(q, np.array([5, -1] + [0] * (T - 2)), k[:, :1], v[:, :1], 0.7)
    assert (Y2[1] == 0).all() and (Z2[1] == -np.inf).all()
    assert np.allclose(Y2[2], v[0, :1])
    one = cu.rows(q[:1, 1:], np.array([5]), k[:, :1], v[:, :1], 0.7)
    assert np.allclose(one[0][0, 0], Y2[0, 1])


def test_tokens_of_a_step():
    starts, pos = cu.tokens([2, 0, 3], [7, 5, 3], 6)
    assert starts.tolist() == [0, 2, 2, 5] and pos.tolist() == [5, 6, 0, 1, 2, -1]
