"""Numbers that the native calls cannot hold are left to the binding, which takes or refuses them."""
import pytest
import torch

from paper_2608_20172_gb300 import binding
from tests.test_native_calls_gpu import decode_args, native, plan_args, token_args  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("big", [2 ** 63, 2 ** 64, -(2 ** 63) - 1, 10 ** 30])
def test_integers_past_64_bits(native, big):  # noqa: F811
    d = decode_args()[:-1]
    want = binding.paged_decode(*d, float(big))
    got = binding.paged_decode(*d, big)
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    assert native.paged_decode(*d, big, 2.0, None) is None
    a = plan_args()
    for i in (5, 6):
        b = list(a)
        b[i] = big
        assert native.page_plan(*b, None) is None
    t = token_args()
    assert native.cache_append(*t, big, 1e4, None) is None
    assert native.cache_append(*t, 0, big, None) is None


def test_minus_one_is_a_number(native):  # noqa: F811
    d = decode_args()[:-1]
    want = binding.paged_decode(*d, -1.0)
    got = native.paged_decode(*d, -1, 2, None)
    for a, b in zip(got, want):
        assert torch.equal(a, b)
