"""The logits' gradient where the rows' log-normaliser is large: low temperatures, logits with a large common
part, a normaliser past the type.  Its rounding is no excuse there: the formula only has differences of
logits."""
import math

import numpy as np
import pytest
import torch

from paper_2608_20172_gb300 import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32
U = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    binding.load()


def grad_row(x, target, T, g, h, k):
    """(gradient, bound) of a row of finite logits from t = (x - max) / T.  The kernel's t is off by 4 u of
    itself (the difference, 1 / T, log2 e and the product), 2^t by 4 u, the sum by V / 128 + 24 roundings, log l
    and the difference t - log l by 4 u of theirs; the given entropy by as much (as the forward's bound).  Rows whose logarithm is
    small take x / T and logz from each other: |logz| <= 64 there, 4 roundings of at most that and log V.
    A weight 2^t below the smallest normal number, 2^-126, counts as 0: as l >= 1, p is off by less than 2^-126."""
    if target < 0:
        g = 0.0  # (no token that it could belong to)
    t = (x - x.max()) / T
    l = np.exp(t).sum()
    logp = t - math.log(l)
    p = np.exp(logp)
    H = -(p[p > 0] * logp[p > 0]).sum()
    mean, mean2 = (p * -t).sum(), (p * t * t).sum()
    sums = U * (len(x) / 128 + 24 + 4 * mean + 4 * abs(math.log(l)))
    lp = U * 4 * np.abs(t) + sums + 4 * U * (64 + math.log(len(x)))
    h_err = sums * (1 + mean) + U * (4 * mean2 + (24 + len(x) / 128) * mean)
    d = p * (k - g - h * (logp + H))
    size = abs(k) + abs(g) + abs(h) * (np.abs(logp) + H)
    err = p * ((lp + 8 * U) * size + abs(h) * (lp + h_err))
    err += np.where(np.exp(t) < 2.0 ** -125, 2.0 ** -126 * size, 0.0)
    if target >= 0:
        d[target] += g
        err[target] += 2 * U * abs(g)
    return d / T, (err + 4 * U * np.abs(d)) / T


def check(x, targets, T, *, inplace=False):
    R, V = x.shape
    t = torch.tensor(targets, dtype=torch.int32, device=DEV)
    temp = torch.tensor(T, dtype=F32, device=DEV)
    rng = np.random.default_rng(1)
    g, h, k = (torch.tensor(rng.standard_normal(R), dtype=F32, device=DEV) for _ in range(3))
    r = binding.logprobs(x, t, temperature=temp)
    rows = x.double().cpu().numpy()
    got = binding.logprobs_grad(x, t, r.logz, r.entropy, g, h, k, temperature=temp, out=x if inplace else None)
    got = got.double().cpu().numpy()
    step = torch.finfo(x.dtype).eps / 2
    for i in range(R):
        with np.errstate(all="ignore"):
            want, tol = grad_row(rows[i], targets[i], float(temp[i]), *(float(v[i]) for v in (g, h, k)))
        err = np.abs(got[i] - want)
        assert (err <= 1.01 * step * np.abs(want) + tol + 1e-37).all(), (i, float(temp[i]), err.max())


def logits(R, V, dtype, shift=0.0, seed=0):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((R, V)) * 2
    x[np.arange(R)[:, None], rng.integers(0, V, (R, 4))] += 6
    return torch.from_numpy(x + shift).to(dtype).to(DEV)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("V", [5, 1003, 9000, 50257])
@pytest.mark.parametrize("inplace", [False, True])
def test_low_temperatures(V, dtype, inplace):
    T = [1.0, 0.1, 1e-2, 1e-3, 1e-4, 1e-6, 1e-8, 1e-20]
    check(logits(8, V, dtype), [0, 1, V - 1, 3, -1, 2, 4, 0], T, inplace=inplace)


@pytest.mark.parametrize("shift", [100.0, -300.0, 3e4, -1e6])
def test_large_common_part(shift):
    check(logits(4, 20011, F32, shift), [0, 20010, -1, 7], [1.0, 0.5, 2.0, 1.0])


def test_equal_and_nearly_equal_largest():
    """Differences of a step of fp32 decide at temperatures of that size, at 1e-38 every one."""
    x = torch.full((3, 3000), -1.0, dtype=F32, device=DEV)
    x[:, [5, 900]] = 1.0
    x[:, 2999] = 1.0 - 2.0 ** -24
    check(x, [5, 2999, 7], [2.0 ** -24, 1e-30, 1e-30])


@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_normaliser_past_the_type(sign):
    """logz is +inf or -inf, the logits finite: neither masked nor infinite ones."""
    x = torch.zeros(2, 700, dtype=F32, device=DEV) - 9.0
    x[:, :3] = 5.0 * sign
    x[0, 600] = 5.0 * sign
    if sign < 0:
        x[:, 3:600], x[:, 601:] = -9.0, -9.0
    t = torch.tensor([0, 1], dtype=torch.int32, device=DEV)
    T = torch.full((2,), 1e-38, dtype=F32, device=DEV)
    r = binding.logprobs(x, t, temperature=T)
    assert torch.isinf(r.logz).all() and (r.logz * sign > 0).all()
    one = torch.full((2,), 1e-3, dtype=F32, device=DEV)
    got = binding.logprobs_grad(x, t, r.logz, r.entropy, one, temperature=T).double().cpu().numpy()
    for i, n in ((0, 4), (1, 3)):
        want = np.where(x[i].cpu().numpy() == 5.0 * sign, -1.0 / n, 0.0)
        want[i] += 1.0
        # 1e-3 / T is off by 4 u, 1 / n by the sum and logarithm of n, their exponents and 2^x: 32 u
        want *= float(one[i]) / float(T[i])
        assert np.abs(got[i] - want).max() <= 40 * U * np.abs(want).max()


def test_replayed_on_another_temperature():
    x = logits(6, 9000, F32)
    t = torch.arange(6, dtype=torch.int32, device=DEV)
    T = torch.ones(6, dtype=F32, device=DEV)
    g = torch.ones(6, dtype=F32, device=DEV)
    step = lambda: (lambda r: binding.logprobs_grad(x, t, r.logz, r.entropy, g, temperature=T))(  # noqa: E731
        binding.logprobs(x, t, temperature=T))
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    T.copy_(torch.tensor([1.0, 1e-3, 1e-7, 0.5, 1e-5, 2.0], device=DEV))
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(got, step())
