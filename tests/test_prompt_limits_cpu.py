"""The sizes that the calls around a prompt refuse are those that their declarations state: the first size past each
limit, and where the call has something else to refuse afterwards the last one before it.  Nothing is launched."""
import os
import re

import pytest

from paper_2608_20172_gb300 import binding
from paper_2608_20172_gb300 import build as libbuild
from tests import test_logprobs_cpu as logprobs
from tests import test_norm_rope_cpu as norm_rope
from tests import test_paged_chunk_cpu as chunk

UNSUPPORTED, WORKSPACE = binding.ERR_UNSUPPORTED, binding.ERR_WORKSPACE
HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "relation.h")


@pytest.fixture(scope="module")
def lib():
    libbuild.build()
    return binding.load()


def states(text):
    with open(HEADER) as f:
        return text in re.sub(r"\s+", " ", re.sub(r"\n \*", " ", f.read()))


def test_chunk(lib):
    """(N + B) H: the same sum whichever of the two is large."""
    assert states("(N + B) H at most 2^31 - 65536")
    most = (1 << 31) - 65536
    for H in (2, 64):
        c = chunk.pages(H=2)
        for N, B in ((most // H - 1, 1), (most // H - 4096, 4096), (1, most // H - 1)):
            assert chunk.chunk(lib, N=N, B=B, H=H, c=c, ws=0) == WORKSPACE
            assert chunk.chunk(lib, N=N + 1, B=B, H=H, c=c, ws=0) == UNSUPPORTED
            assert chunk.chunk(lib, N=N, B=B + 1, H=H, c=c, ws=0) == UNSUPPORTED
            size = lambda N, B: lib.relation_paged_chunk_workspace_size(N, B, H, 8, c, binding.BF16)  # noqa: E731
            assert size(N, B) > 0 and size(N + 1, B) == size(N, B + 1) == 0
    assert states("cols * page_size is at most 2^31 - 8192")
    rows = (1 << 31) - 8192
    assert chunk.chunk(lib, c=chunk.pages(page=8192), cols=rows // 8192, stride=rows, ws=0) == WORKSPACE
    assert chunk.chunk(lib, c=chunk.pages(page=8192), cols=rows // 8192 + 1, stride=rows, ws=0) == UNSUPPORTED


def test_logprobs(lib):
    assert states("V <= 2^30, R <= 2^27 (else RELATION_ERR_UNSUPPORTED)")
    assert logprobs.fwd(lib, R=(1 << 27) + 1) == UNSUPPORTED
    assert logprobs.fwd(lib, V=(1 << 30) + 1, stride=1 << 31) == UNSUPPORTED
    assert states("R (V / 4096 + 2) < 2^31, the quotient rounded down")
    for V in (1, 4095, 4096, 50257, 1 << 30):
        R = ((1 << 31) - 1) // (V // 4096 + 2)
        assert logprobs.grad(lib, R=R + 1, V=V, stride=V, out_stride=V) == UNSUPPORTED, V


def test_norm_rope(lib):
    assert states("heads of queries and keys together up to 2^24 (else RELATION_ERR_UNSUPPORTED)")
    for call in (norm_rope.fwd, norm_rope.grad):
        H = 1 << 23
        assert call(lib, sq=norm_rope.shape(H=H), sk=norm_rope.shape(H=H + 1)) == UNSUPPORTED
        assert call(lib, sq=norm_rope.shape(H=H + 1), sk=norm_rope.shape(H=H)) == UNSUPPORTED
    assert states("B T up to 2^30")
    big = norm_rope.shape(B=1 << 15, T=(1 << 15) + 1)
    assert norm_rope.fwd(lib, sq=big, sk=big) == UNSUPPORTED
    # (the gradient's last refusal is its workspace's)
    two = norm_rope.shape(H=1 << 23)
    assert norm_rope.grad(lib, sq=two, sk=two, ws=0) == WORKSPACE
