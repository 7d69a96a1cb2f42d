"""relation_paged_decode with infinities among the values: Y of a channel is a sum of values with positive
weights, so that one infinity makes it that infinity, two of opposite signs NaN, and no other channel
feels it.  The scores are small here: no weight underflows."""
import numpy as np
import pytest
import torch

from paper_2608_20172_gb300 import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
INF = float("inf")


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    binding.load()


def run(n, H, Hk, d, dtype, places, pad=0, page=16):
    """Y [H, d] of one request of n rows, its values replaced at places (row, key head, channel, value),
    and the same without them."""
    rng = np.random.default_rng(n + d)
    pages = -(-n // page)
    k, v = (torch.zeros((pages, page, Hk, d + pad), dtype=dtype)[..., :d] for _ in range(2))
    k.copy_(torch.from_numpy(rng.standard_normal(k.shape)))
    v.copy_(torch.from_numpy(rng.standard_normal(v.shape)))
    q = torch.from_numpy(rng.standard_normal((1, H, d))).to(dtype).to(DEV)
    put = lambda x: torch.empty_strided(x.size(), x.stride(), dtype=dtype, device=DEV).copy_(x)  # noqa: E731
    table = torch.arange(pages, dtype=torch.int32, device=DEV)[None]
    lengths = torch.tensor([n], dtype=torch.int32, device=DEV)
    kd, out = put(k), []
    for places in ([], places):
        for r, h, c, x in places:
            v[r // page, r % page, h, c] = x
        out.append(binding.paged_decode(q, kd, put(v), table, lengths, 0.5)[0][0].float().cpu().numpy())
    return out


FORMS = [(torch.bfloat16, 1, 1, 64, 0), (torch.bfloat16, 1, 1, 128, 0), (torch.bfloat16, 1, 1, 64, 3),
         (torch.float32, 1, 1, 64, 0), (torch.float32, 4, 1, 80, 0), (torch.float32, 8, 1, 32, 1),
         (torch.bfloat16, 2, 1, 32, 0), (torch.bfloat16, 8, 1, 64, 0), (torch.bfloat16, 4, 1, 80, 0),
         (torch.bfloat16, 8, 2, 128, 0), (torch.bfloat16, 9, 1, 64, 0), (torch.bfloat16, 5, 1, 64, 1)]


# the first row; one inside a tile; the last row of the history (in a tile's end that is cut off); many runs
@pytest.mark.parametrize("n,row", [(2, 0), (40, 17), (40, 38), (66, 64), (1200, 700), (1200, 1198)])
@pytest.mark.parametrize("dtype,H,Hk,d,pad", FORMS)
def test_infinity_in_the_history(dtype, H, Hk, d, pad, n, row):
    last = Hk - 1
    plain, y = run(n, H, Hk, d, dtype, [(row, last, 3, INF), (row, last, d - 1, -INF)], pad)
    mine = np.arange(H) // (H // Hk) == last
    assert (y[mine, 3] == INF).all() and (y[mine, d - 1] == -INF).all()
    other = np.ones((H, d), bool)
    other[np.ix_(mine, [3, d - 1])] = False
    assert np.array_equal(y[other], plain[other])


@pytest.mark.parametrize("dtype,H,Hk,d,pad", FORMS)
def test_opposite_infinities(dtype, H, Hk, d, pad):
    plain, y = run(300, H, Hk, d, dtype, [(5, 0, 2, INF), (250, 0, 2, -INF)], pad)
    mine = np.arange(H) // (H // Hk) == 0
    assert np.isnan(y[mine, 2]).all()
    other = np.ones((H, d), bool)
    other[mine, 2] = False
    assert np.array_equal(y[other], plain[other])
