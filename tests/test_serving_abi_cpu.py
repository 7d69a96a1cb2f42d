"""The serving entry points without a GPU: bad arguments are refused synchronously, nothing launched;
the size query; the plain 64-bit plan that the GPU tests compare with."""
import ctypes

import numpy as np
import pytest

from paper_2608_20172_gb300 import binding
from paper_2608_20172_gb300 import build as libbuild
from tests import serving_util as su

P = [0x10000 * (i + 1) for i in range(16)]  # aligned, never dereferenced here
INVALID, UNSUPPORTED, ALIGNMENT = (binding.ERR_INVALID_ARG, binding.ERR_UNSUPPORTED,
                                   binding.ERR_ALIGNMENT)


@pytest.fixture(scope="module")
def lib():
    libbuild.build()
    return binding.load()


def pages(n=10, page=16, H=2, d=64, sP=None, sR=None, sH=None):
    sH = d if sH is None else sH
    sR = H * d if sR is None else sR
    return binding.Pages(n, page, H, d, page * H * d if sP is None else sP, sR, sH)


def plan(lib, ptrs=None, B=4, page=16, cols=8, stride=8, n_pages=32, n_tokens=8, status=None):
    q = list(P[:9]) if ptrs is None else ptrs
    return lib.relation_page_plan(q[0], q[1], B, page, q[2], cols, stride, q[3], n_pages, q[4], q[5],
                                  q[6], q[7], q[8], P[9], n_tokens, status, None)


@pytest.mark.parametrize("kw,expect", [
    (dict(B=0), INVALID), (dict(page=0), INVALID), (dict(cols=0), INVALID), (dict(stride=7), INVALID),
    (dict(n_pages=0), INVALID), (dict(n_tokens=0), INVALID),
    (dict(page=1 << 30, cols=8), UNSUPPORTED), (dict(B=1 << 28, cols=16, stride=16), UNSUPPORTED),
    (dict(status=2), ALIGNMENT)])
def test_page_plan_refuses(lib, kw, expect):
    assert plan(lib, **kw) == expect


def test_page_plan_refuses_pointers(lib):
    for i in range(9):
        q = list(P[:9])
        q[i] = None
        assert plan(lib, q) == INVALID
        q[i] = P[i] + (4 if i == 8 else 2)
        assert plan(lib, q) == ALIGNMENT
    q = list(P[:9])
    q[6] = q[0]  # lengths_out on top of lengths
    assert plan(lib, q) == INVALID
    q = list(P[:9])
    q[5] = q[4]  # free_state_out on top of free_state
    assert plan(lib, q) == INVALID


def append(lib, N=4, c=None, dt=binding.BF16, pairing=0, base=1e4, p=None, sT=128, sH=64, status=None):
    q = list(P[:9]) if p is None else p
    # p1, p2, info, theta, positions, slots, q, k, v
    return lib.relation_cache_append(q[0], q[1], q[2], q[3], pairing, base, q[4], q[5], q[6], N, sT, sH,
                                     q[7], q[8], pages() if c is None else c, dt, status, None)


@pytest.mark.parametrize("kw,expect", [
    (dict(N=0), INVALID), (dict(dt=2), INVALID), (dict(pairing=2), INVALID), (dict(base=-1.0), INVALID),
    (dict(base=float("nan")), INVALID), (dict(base=float("inf")), INVALID), (dict(sT=0), INVALID),
    (dict(sH=-64), INVALID), (dict(c=pages(n=0)), INVALID), (dict(c=pages(page=0)), INVALID),
    (dict(c=pages(H=0)), INVALID), (dict(c=pages(d=0)), INVALID), (dict(c=pages(sP=0)), INVALID),
    (dict(c=pages(d=258)), UNSUPPORTED), (dict(c=pages(d=63)), UNSUPPORTED),
    (dict(c=pages(H=3)), UNSUPPORTED), (dict(N=1 << 30), UNSUPPORTED), (dict(status=1), ALIGNMENT)])
def test_cache_append_refuses(lib, kw, expect):
    assert append(lib, **kw) == expect


def test_cache_append_refuses_pointers(lib):
    for i, low, none in ((1, 1, INVALID), (2, 1, INVALID), (5, 4, INVALID), (7, 1, INVALID),
                         (8, 1, INVALID), (4, 2, INVALID), (3, 2, None), (0, 1, INVALID),
                         (6, 1, INVALID)):
        q = list(P[:9])
        q[i] = P[i] + low
        assert append(lib, p=q) == ALIGNMENT, i
        if none is not None:
            q[i] = None
            assert append(lib, p=q) == none, i


def decode(lib, B=2, H=2, cols=8, stride=8, c=None, dt=binding.BF16, lam=0.5, tau=2.0, p=None,
           ws=1 << 30, sB=128, sH=64, status=None):
    q = list(P[:8]) if p is None else p
    # q, k, v, table, lengths, o, logz, workspace
    return lib.relation_paged_decode(q[0], q[1], q[2], q[3], cols, stride, q[4], q[5], q[6], lam, tau, B,
                                     H, pages() if c is None else c, sB, sH, dt, q[7], ws, status, None)


@pytest.mark.parametrize("kw,expect", [
    (dict(B=0), INVALID), (dict(H=3), INVALID), (dict(H=0), INVALID), (dict(cols=0), INVALID),
    (dict(stride=4), INVALID), (dict(dt=7), INVALID), (dict(lam=float("nan")), INVALID),
    (dict(tau=0.0), INVALID), (dict(sB=0), INVALID), (dict(sH=0), INVALID),
    (dict(c=pages(d=129)), UNSUPPORTED), (dict(c=pages(page=1 << 28), cols=8), UNSUPPORTED),
    (dict(ws=100), binding.ERR_WORKSPACE), (dict(status=2), ALIGNMENT)])
def test_paged_decode_refuses(lib, kw, expect):
    assert decode(lib, **kw) == expect


def test_paged_decode_refuses_pointers(lib):
    for i, low in ((0, 1), (1, 1), (2, 1), (3, 2), (4, 2), (5, 1), (6, 2), (7, 8)):
        q = list(P[:8])
        q[i] = P[i] + low
        assert decode(lib, p=q) == ALIGNMENT, i
        q[i] = None
        assert decode(lib, p=q) == (binding.ERR_WORKSPACE if i == 7 else INVALID), i


def test_paged_decode_workspace(lib):
    size = lib.relation_paged_decode_workspace_size
    base = size(2, pages(), binding.BF16)
    assert base > 0 and base == size(2, pages(n=100000, page=64), binding.F32)
    assert 4 * base < size(16, pages(), binding.BF16) <= 8 * base  # eight query heads at once
    for H, c in ((3, pages()), (0, pages()), (2, pages(d=129)), (2, pages(n=0))):
        assert size(H, c, binding.BF16) == 0


def sample(lib, R=4, V=100, stride=100, dt=binding.F32, p=None, status=None):
    q = list(P[:9]) if p is None else p
    # logits, u, temperature, top_k, top_p, min_p, token, logprob, logz
    return lib.relation_sample(q[0], R, V, stride, dt, q[1], q[2], q[3], q[4], q[5], q[6], q[7], q[8],
                               status, None)


@pytest.mark.parametrize("kw,expect", [
    (dict(R=0), INVALID), (dict(V=0), INVALID), (dict(stride=99), INVALID), (dict(dt=2), INVALID),
    (dict(V=262145, stride=262145), UNSUPPORTED), (dict(R=1 << 28), UNSUPPORTED),
    (dict(status=2), ALIGNMENT)])
def test_sample_refuses(lib, kw, expect):
    assert sample(lib, **kw) == expect


def test_sample_refuses_pointers(lib):
    for i in range(9):
        q = list(P[:9])
        q[i] = P[i] + 2
        assert sample(lib, p=q) == ALIGNMENT, i
        if i not in (2, 3, 4, 5):
            q[i] = None
            assert sample(lib, p=q) == INVALID, i


def test_status_of_a_full_pool(lib):
    assert binding.status_string(binding.ERR_CAPACITY) == "RELATION_ERR_CAPACITY"
    assert ctypes.sizeof(binding.Pages) == 40


def test_plain_plan_by_hand():
    """Three requests of pages of 4: one grows past its page, one ends, one is new."""
    table = np.array([[5, 6, -1], [7, -1, -1], [-1, -1, -1]], np.int32)
    free = np.array([9, 0, 1, 2, 3, 8], np.int32)  # head 1: 0 1 2 3 free
    got = su.plan(np.array([8, 3, 0], np.int32), np.array([2, -1, 5], np.int32), table, free,
                  np.array([1, 4], np.int32), 4, 9)
    slots, positions, starts, lengths, state, new, ring = got
    assert slots.tolist() == [0, 1, 4, 5, 6, 7, 8, -1, -1]
    assert positions.tolist() == [8, 9, 0, 1, 2, 3, 4, -1, -1]
    assert starts.tolist() == [0, 2, 2, 7] and lengths.tolist() == [10, 0, 5]
    assert new.tolist() == [[5, 6, 0], [7, -1, -1], [1, 2, -1]]
    assert ring.tolist() == [9, 0, 1, 2, 3, 7] and state.tolist() == [4, 2]


def test_plain_cuts_by_hand():
    x = np.log(np.array([0.1, 0.4, 0.2, 0.3]))
    kept = lambda **kw: su.kept_tokens(x, **kw)[0].tolist()  # noqa: E731
    assert kept() == [0, 1, 2, 3]
    assert kept(top_k=2) == [1, 3] and kept(top_p=0.5) == [1, 3] and kept(top_p=0.39) == [1]
    assert kept(min_p=0.45) == [1, 2, 3] and kept(temperature=0.0) == [1]
    assert kept(top_k=3, top_p=0.7) == [1, 3]  # of 0.9: 0.63 is reached by the second
    w = su.kept_tokens(x, temperature=0.5)[1]
    assert np.allclose(w, (np.exp(x) / 0.4) ** 2)
