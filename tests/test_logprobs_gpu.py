"""relation_logprobs and its gradient against 64 bits: types, odd lengths, strides, masks, ties, infinities,
NaN, temperatures, clusters of CTAs, in place, streams, capture, autograd."""
import math

import numpy as np
import pytest
import torch

from paper_2608_20172_gb300 import binding
from tests import logprobs_util as lu

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32
INF, NAN = math.inf, math.nan


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    binding.load()


def rows(R, V, dtype, seed=0, pad=0, offset=0):
    """Logits [R, V] with a few likely tokens, rows `pad` elements apart, the first `offset` from a 16-byte
    boundary."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((R, V)) * 2
    x[np.arange(R)[:, None], rng.integers(0, V, (R, 4))] += 6
    wide = torch.full((R * (V + pad) + offset,), 55.0, dtype=dtype, device=DEV)
    t = wide[offset:].view(R, V + pad)[:, :V]
    return t.copy_(torch.from_numpy(x))


def check(logits, targets, temperature=None, top=0, status=None, **kw):
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    T = None if temperature is None else torch.tensor(temperature, dtype=F32, device=DEV)
    t = torch.tensor(targets, dtype=torch.int32, device=DEV)
    r = binding.logprobs(logits, t, temperature=T, top=top, dev_status=st, **kw)
    got = [x.double().cpu().numpy() for x in r if x is not None]
    for i, x in enumerate(logits.double().cpu().numpy()):
        Ti = 1.0 if T is None else float(T[i])
        want = lu.row(x, targets[i], Ti, top)
        l_err, h_err, m = lu.bounds(x, Ti if Ti > 0 and math.isfinite(Ti) else 1.0)
        tol = lambda v, e: e + lu.U * (4 * abs(v) if math.isfinite(v) else 0)  # noqa: E731
        for j, e in ((0, l_err), (1, h_err), (2, l_err + 2 * lu.U * m)):
            np.testing.assert_allclose(got[j][i], want[j], rtol=0, atol=tol(want[j], e), err_msg=f"{i} {j}")
        if top:
            assert got[3][i].astype(int).tolist() == want[3], i
            for a, b in zip(got[4][i], want[4]):
                np.testing.assert_allclose(a, b, rtol=0, atol=tol(b, l_err))
    assert int(st) == (binding.OK if status is None else status)
    return r


SHAPES = [(1, 1), (3, 2), (2, 7), (5, 33), (4, 255), (3, 1000), (7, 4097), (2, 20011), (1, 32000), (1, 131072),
          (9, 50257), (200, 3001)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("R,V", SHAPES)
def test_forward(R, V, dtype):
    targets = [(7 * i + 3) % V if i % 3 != 1 else -1 for i in range(R)]
    for top in (0, 1, min(20, V), 32):
        check(rows(R, V, dtype), targets, top=top)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("pad,offset", [(0, 1), (1, 0), (3, 5), (8, 8)])
def test_strides_and_alignments(pad, offset, dtype):
    x = rows(5, 1003, dtype, pad=pad, offset=offset)
    check(x, [0, 1002, 500, -1, 7], temperature=[0.5, 1.0, 2.0, 1.0, 0.9], top=7)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("V", [300, 40000])
def test_masks(V, dtype):
    """-inf and the type's lowest; one token left; none left; with and without a given token."""
    x = rows(8, V, dtype, seed=2)
    low = torch.finfo(dtype).min
    x[0, 5:] = -INF
    x[1, :] = -INF
    x[2, :] = -INF
    x[3, :] = -INF
    x[3, V - 1] = 2.0
    x[4, 10:] = low
    x[5, :] = low
    x[6, 1::2] = -INF
    check(x, [3, 5, -1, V - 1, 4, 17, 2, -1], top=8)
    check(x, [3, 5, -1, V - 1, 4, 17, 2, -1], temperature=[1.5] * 8, top=32)


@pytest.mark.parametrize("V", [300, 40000])
def test_infinities_and_nan(V):
    x = rows(6, V, F32, seed=3)
    x[0, 7] = INF
    x[1, [3, V - 2]] = INF
    x[2, 9] = NAN
    x[3, :] = NAN
    x[4, :] = -INF
    x[4, 1] = NAN
    x[5, 2], x[5, 3] = INF, NAN
    check(x, [7, 4, 0, 0, 2, 2], top=4)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("V", [100, 5000, 60000])
def test_ties(V, dtype):
    """Equal logits go by their index: all of them, two values, -0 beside 0, ascending and descending rows."""
    x = torch.zeros((5, V), dtype=dtype, device=DEV)
    x[1, 1::2] = 1.0
    x[2, ::3] = -0.0
    x[3] = torch.arange(V, device=DEV).float().mul_(1 / 64).to(dtype)
    x[4] = x[3].flip(0)
    check(x, [0, 1, 2, V - 1, 0], top=32)
    check(x, [0, 1, 2, V - 1, 0], top=3)


def test_the_largest_all_in_one_thread():
    """The 32 largest among one thread's elements, and spread over every warp's first lane."""
    x = rows(2, 60000, F32, seed=4)
    x[0, 4 * 512 * torch.arange(29)] = 30 + torch.arange(29, device=DEV).float()
    x[1, 128 * torch.arange(32)] = 40.0
    check(x, [0, 0], top=32)


def test_bad_temperatures_and_tokens():
    x = rows(6, 500, F32, seed=5)
    st = binding.ERR_INVALID_ARG
    check(x, [1] * 6, temperature=[1.0, 0.0, -1.0, NAN, INF, 2.0], top=2, status=st)
    check(x, [500, 1, 2, 2 ** 31 - 1, 499, -7], top=2, status=st)


def test_one_row_is_every_batch_row():
    """A row has the same bits alone in its cluster size's batch, and again."""
    x = rows(300, 9000, BF16, seed=6)
    t = torch.arange(300, dtype=torch.int32, device=DEV)
    a, b = binding.logprobs(x, t, top=5), binding.logprobs(x, t, top=5)
    c = binding.logprobs(x[37:], t[37:], top=5)
    for u, v, w in zip(a, b, c):
        assert torch.equal(u, v) and torch.equal(u[37:], w)


def test_agrees_with_sample():
    x = rows(16, 32000, F32, seed=7)
    T = torch.full((16,), 0.8, device=DEV)
    token, logprob, logz = binding.sample(x, torch.rand(16, device=DEV), temperature=T)
    r = binding.logprobs(x, token, temperature=T)
    # (the sampler's weights are whole numbers of 2^-40: 32000 of them are off by less than 2^-25 together)
    assert torch.allclose(r.logprob, logprob, atol=1e-5) and torch.allclose(r.logz, logz, atol=1e-5)


def check_grad(logits, targets, temperature, g, h, k, **kw):
    R, V = logits.shape
    f = lambda v: None if v is None else torch.tensor(v, dtype=F32, device=DEV)  # noqa: E731
    t, T = torch.tensor(targets, dtype=torch.int32, device=DEV), f(temperature)
    r = binding.logprobs(logits, t, temperature=T)
    x = logits.double().cpu().numpy()  # (before a gradient in its place)
    got = binding.logprobs_grad(logits, t, r.logz, r.entropy, f(g), f(h), f(k), temperature=T, **kw)
    step = torch.finfo(logits.dtype).eps / 2
    out = got.double().cpu().numpy()
    at = lambda v, i: 0.0 if v is None else float(np.float32(v[i]))  # noqa: E731
    for i in range(R):
        Ti = 1.0 if temperature is None else float(np.float32(temperature[i]))
        want, tol = lu.grad_row(x[i], targets[i], Ti, at(g, i), at(h, i), at(k, i))
        l_err, h_err, _ = lu.bounds(x[i], Ti)
        # the forward's logz and entropy are off by these
        p = np.abs(want) + np.abs(tol) / lu.U / 8
        tol = tol + (l_err + h_err) * p
        np.testing.assert_array_equal(np.isnan(out[i]), np.isnan(want))
        ok = ~np.isnan(want)
        assert (np.abs(out[i] - want)[ok] <= (step * 1.01 * np.abs(want) + tol + 1e-37)[ok]).all(), i
    return got


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("R,V", [(1, 1), (3, 2), (4, 255), (3, 1000), (2, 8193), (1, 32000), (9, 50257)])
def test_gradient(R, V, dtype):
    rng = np.random.default_rng(R + V)
    targets = [(7 * i + 3) % V if i % 3 != 1 else -1 for i in range(R)]
    g, h, k = (rng.standard_normal(R).tolist() for _ in range(3))
    T = (0.5 + rng.random(R)).tolist()
    check_grad(rows(R, V, dtype), targets, None, g, None, None)
    check_grad(rows(R, V, dtype), targets, T, g, h, k)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_gradient_of_masked_rows(dtype):
    x = rows(9, 700, dtype, seed=9)
    low = torch.finfo(dtype).min
    x[0, 5:] = -INF
    x[1, :] = -INF
    x[2, :] = -INF
    x[3, 1:] = low
    x[4, [3, 9]] = INF
    x[5, 6] = NAN
    x[6, :] = low
    check_grad(x, [4, 5, -1, 0, 3, 2, 8, 700, -1], [1.0, 1.0, 1.0, 0.7, 1.3, 1.0, 1.0, 1.0, 2.0], [0.5] * 9,
               [0.2] * 9, [-0.3] * 9)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("pad,offset", [(0, 1), (1, 0), (3, 5), (8, 8)])
def test_gradient_strides_and_in_place(pad, offset, dtype):
    args = [0, 1002, 500, -1, 7], [0.5, 1.0, 2.0, 1.0, 0.9], [1.0, -1.0, 2.0, 3.0, 0.1], [0.1] * 5, [0.2] * 5
    x = rows(5, 1003, dtype, pad=pad, offset=offset)
    a = check_grad(x, *args)
    b = check_grad(x, *args, out=rows(5, 1003, dtype, pad=2, offset=3))
    c = check_grad(x, *args, out=x)
    assert c is x and torch.equal(a, b) and torch.equal(a, c)
    if pad:  # nothing is written between the rows
        beside = x.as_strided((5, pad), x.stride(), x.storage_offset() + 1003)
        assert (beside[:4] == 55).all()


def test_stream_and_capture():
    x = rows(40, 5001, BF16)
    t = torch.arange(40, dtype=torch.int32, device=DEV)
    g = torch.randn(40, device=DEV)

    def both(**kw):
        r = binding.logprobs(x, t, top=3, **kw)
        return (*r, binding.logprobs_grad(x, t, r.logz, r.entropy, g, g, **kw))

    want = both()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = both(stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both()
    x.copy_(x.flip(0).contiguous())
    want = both()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_autograd():
    x = rows(6, 1500, F32, seed=11)
    t = torch.tensor([1, 5, -1, 1499, 0, 3], dtype=torch.int32, device=DEV)
    T = torch.full((6,), 0.9, device=DEV)
    leaf = x.clone().requires_grad_()
    lp, h, lz = binding.LogprobsFunction.apply(leaf, t, T)
    (-lp.sum() + 0.1 * h.sum() + 0.01 * lz.square().sum()).backward()
    ref = x.double().requires_grad_()
    logp = torch.log_softmax(ref / 0.9, 1)
    live = t >= 0
    loss = -(logp[live, t[live].long()]).sum() - 0.1 * (logp.exp() * logp).sum()
    (loss + 0.01 * torch.logsumexp(ref / 0.9, 1).square().sum()).backward()
    # entries of at most 2, off by roundings of log p of about 10: 2 * 40 * 2^-24
    assert torch.allclose(leaf.grad.double(), ref.grad, atol=5e-6, rtol=0)
    leaf.grad = None
    binding.LogprobsFunction.apply(leaf, t)[0].sum().backward()  # one of the three alone
    assert torch.isfinite(leaf.grad).all()


def test_binding_refuses():
    x = rows(4, 100, F32)
    t = torch.zeros(4, dtype=torch.int32, device=DEV)
    z = torch.zeros(4, device=DEV)
    for call in (lambda: binding.logprobs(x, t.long()), lambda: binding.logprobs(x, t[:3]),
                 lambda: binding.logprobs(x.t(), t), lambda: binding.logprobs(x, t, temperature=z.double()),
                 lambda: binding.logprobs_grad(x, t, z[:3], z), lambda: binding.logprobs_grad(x, t, z, z, z.cpu()),
                 lambda: binding.logprobs_grad(x, t, z, z, out=x.bfloat16())):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: binding.logprobs(x, t, top=33), lambda: binding.logprobs(x, t, top=-1),
                 lambda: binding.logprobs(x[:1].expand(4, -1), t)):
        with pytest.raises(binding.RelationError):
            call()
    with pytest.raises(TypeError):
        binding.logprobs(x.half(), t)
