"""relation_paged_decode over hundreds of ragged requests, so that a run holds whole heads, several heads
and parts of two: head groups that share keys in both types, every form's head sizes, unaligned rows.
All requests are compared with the row in fp64; the bounds are those of test_paged_decode_gpu.py."""
import numpy as np
import pytest
import torch

from tests.test_paged_decode_gpu import _lib, check  # noqa: F401

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def lengths(B, most, seed):
    n = np.random.default_rng(seed).integers(0, most, B)
    n[:3] = (0, 1, 2)
    return n.tolist()


@pytest.mark.parametrize("d", [32, 64, 80, 96, 128])
@pytest.mark.parametrize("H,Hk", [(4, 2), (8, 2), (16, 2), (24, 2)])
def test_shared_keys(H, Hk, d):
    """(24, 2): twelve query heads to a key head, in groups of eight and four."""
    check(lengths(300, 400, d + H), H, Hk, d, 16, BF16, seed=d + H)


@pytest.mark.parametrize("H,Hk,d", [(2, 2, 128), (4, 4, 80), (4, 2, 64), (8, 2, 32), (16, 2, 128), (12, 1, 80)])
def test_fp32(H, Hk, d):
    check(lengths(300, 400, d + H), H, Hk, d, 16, F32, seed=d + H)


@pytest.mark.parametrize("H,Hk,d", [(2, 2, 128), (4, 4, 96), (3, 3, 32)])
def test_one_query_head(H, Hk, d):
    check(lengths(400, 400, d + H), H, Hk, d, 16, BF16, seed=d + H)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("H,Hk,d", [(2, 2, 128), (4, 4, 33), (4, 2, 80), (8, 2, 64), (16, 2, 127), (12, 1, 64)])
def test_unaligned_rows(dtype, H, Hk, d):
    check(lengths(300, 300, d + H), H, Hk, d, 24, dtype, pad=1, seed=d + H)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("H,Hk,d", [(2, 2, 128), (8, 2, 80), (8, 1, 64)])
def test_short_and_long_requests_together(dtype, H, Hk, d):
    """Hundreds of requests of a tile or less beside a few that many runs share."""
    n = lengths(600, 66, d + H)
    n[::97] = (3000, 0, 5000, 1, 2500, 64, 65)
    check(n, H, Hk, d, 16, dtype, seed=d + H)
