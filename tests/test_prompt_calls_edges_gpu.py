"""The calls around a prompt where offsets pass 32 bits, pages are shared by requests or of odd sizes, the plan
is as large as its small form allows or larger by one, and two calls run at once."""
import numpy as np
import pytest
import torch

from paper_2608_20172_gb300 import binding
from tests import logprobs_util as lu
from tests.test_logprobs_gpu import check as check_logprobs, rows as logit_rows
from tests.test_paged_chunk_gpu import Step

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    binding.load()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("page", [1, 8, 40, 56, 72])
def test_pages_of_odd_sizes(page, dtype):
    Step([5, 130, 1], [300, 450, 65], 4, 2, 80, dtype, page, seed=21).check()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("B", [31, 32, 33, 512, 513])
def test_around_the_small_plans_limits(B, dtype):
    """Requests and tiles (one each) around 32 and the requests that the plan orders around 512."""
    Step([1] * B, [1 + (7 * i) % 90 for i in range(B)], 2, 1, 64, dtype, 16, seed=22).check()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("tiles", [32, 33])
def test_tiles_of_one_request_around_the_limit(tiles, dtype):
    rows = 128 if dtype is BF16 else 64
    Step([tiles * rows], [tiles * rows], 1, 1, 32, dtype, 64, seed=23).check()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_requests_share_pages(dtype):
    """A common beginning in the same pages, and a request twice: the same tokens give the same bits."""
    s = Step([6, 6, 20], [200, 200, 90], 4, 2, 64, dtype, 16, seed=24)
    c = s.cache
    c.table[1] = c.table[0]
    c.table[2, :5] = c.table[0, :5]
    c.block_table = torch.from_numpy(c.table).to(DEV)
    s.q[6:12] = s.q[:6]
    s.check()
    y, z = s.run()
    assert torch.equal(y[:6], y[6:12]) and torch.equal(z[:6], z[6:12])


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_pages_past_32_bits(dtype):
    """Pages at the end of a cache of more than 2^31 elements give what the same pages give at its beginning."""
    s = Step([3, 70], [150, 260], 2, 2, 64, dtype, 16, seed=25)
    want = s.run()
    c = s.cache
    n, (P, p, Hk, d) = c.k.shape[0], c.k.shape
    total = (2 ** 31 + 2 ** 20) // (p * Hk * d)
    for name in ("k", "v"):
        big = torch.empty((total, p, Hk, d), dtype=dtype, device=DEV)
        big[total - n:] = getattr(c, name)
        setattr(c, name, big)
    c.block_table = torch.where(c.block_table < 0, c.block_table, c.block_table + (total - n)).to(torch.int32)
    got = s.run()
    assert all(torch.equal(a, b) for a, b in zip(want, got))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rows_past_32_bits(dtype):
    """Tokens 2^30 elements apart: queries, logits and normed rows."""
    far = 2 ** 30
    store = torch.empty(2 * far + 4096, dtype=dtype, device=DEV)
    s = Step([3], [50], 2, 2, 64, dtype, 16, seed=26)
    want = s.run()
    q = store.as_strided((3, 2, 64), (far, 64, 1)).copy_(s.q)
    out = torch.empty(2 * far + 4096, dtype=dtype, device=DEV).as_strided((3, 2, 64), (far, 64, 1))
    c = s.cache
    binding.paged_chunk(q, c.k, c.v, c.block_table, s.t_starts, s.t_pos, s.lam, out=out)
    assert torch.equal(out, want[0])
    rot = binding.rotary(64, device=DEV)
    pos = torch.arange(3, dtype=torch.int32, device=DEV)
    a, _ = binding.norm_rope(s.q, None, rot, pos)
    b, _ = binding.norm_rope(q, None, rot, pos, out=(out, None))
    assert torch.equal(a, b)
    x = logit_rows(3, 1000, dtype, seed=27)
    t = torch.tensor([0, 999, 5], dtype=torch.int32, device=DEV)
    r = binding.logprobs(x, t, top=3)
    y = store.as_strided((3, 1000), (far, 1)).copy_(x)
    for u, v in zip(r, binding.logprobs(y, t, top=3)):
        assert torch.equal(u, v)
    g = torch.ones(3, device=DEV)
    want = binding.logprobs_grad(x, t, r.logz, r.entropy, g)
    assert torch.equal(want, binding.logprobs_grad(y, t, r.logz, r.entropy, g, out=y))


def test_two_calls_at_once():
    """Calls of two streams, each with a workspace of its own."""
    a = Step([40, 1, 7], [900, 3000, 700], 4, 2, 64, BF16, 16, seed=28)
    b = Step([3, 200], [2500, 400], 4, 2, 64, BF16, 16, seed=29)
    steps, want = (a, b), (a.run(), b.run())
    space = [torch.empty(binding.paged_chunk_workspace_size(s.q, s.cache.k, s.cache.block_table),
                         dtype=torch.uint8, device=DEV) for s in steps]
    streams = [torch.cuda.Stream() for _ in steps]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(20):
        for i, s in enumerate(steps):
            with torch.cuda.stream(streams[i]):
                got[i].append(s.run(workspace=space[i]))
    torch.cuda.synchronize()
    for w, runs in zip(want, got):
        assert all(torch.equal(x, y) for r in runs for x, y in zip(w, r))


def test_temperatures_at_the_ends_of_the_type():
    """Small ones whose reciprocal fits are served, others refused; the largest make every token as likely."""
    x = logit_rows(3, 500, F32, seed=30)
    temperature = [3e38, 2.0 ** -126, 1.0]
    check_logprobs(x[::2], [1, 3], temperature=temperature[::2], top=2)
    # At 2^-126 the logarithms are 2^126 times differences of several units: those above 4 are past fp32's
    # largest (2^128), and what the type holds of them is an infinity.
    t = torch.tensor([1, 2, 3], dtype=torch.int32, device=DEV)
    r = binding.logprobs(x, t, temperature=torch.tensor(temperature, device=DEV), top=2)
    want = lu.row(x[1].double().cpu().numpy(), 2, temperature[1], 2)
    with np.errstate(over="ignore"):
        for got, w in zip((r.logprob[1], r.entropy[1], r.logz[1], r.top_logprobs[1]), (*want[:3], want[4])):
            # (a difference, a product and the logarithm's sum: 4 roundings)
            np.testing.assert_allclose(got.cpu().numpy(), np.float32(w), rtol=4 * lu.U, atol=4 * lu.U)
    assert r.top_tokens[1].tolist() == want[3]
    check_logprobs(x[:1], [1], temperature=[1e30], top=2)
    t = torch.zeros(1, dtype=torch.int32, device=DEV)
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    r = binding.logprobs(x[:1], t, temperature=torch.tensor([1e-40], device=DEV), dev_status=st)
    assert int(st) == binding.ERR_INVALID_ARG and all(v.isnan().all() for v in r[:3])
