"""The gradient of a token that is almost certain, 1 - p, where the rows' log-normaliser is some tens: a
difference of two numbers of that size, which is to be as exact as the normaliser that it is given."""
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


def rows(R, V, low, high, temperature, gap, dtype, seed):
    """Logits whose largest, at a random place, is low to high temperatures above 0 and about `gap` of them
    above all others."""
    rng = np.random.default_rng(seed)
    top = rng.uniform(low, high, R)
    x = (top[:, None] - gap + rng.standard_normal((R, V))) * temperature
    at = rng.integers(0, V, R)
    x[np.arange(R), at] = top * temperature
    return torch.from_numpy(x).to(dtype).to(DEV), at


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("T", [1.0, 0.7, 0.3, 3.3])
def test_almost_certain_tokens(T, sign, dtype):
    """1 - p of the given token.  Its logarithm is x / T - logz.  logz is a number between 32 and 64 in size,
    rounded once: off by 2^-19 = 32 u, and by the error of log l; l is a sum of 1 and small weights, a thread
    adds up at most V / 128 of them and 24 additions join the threads, each with a rounding of a number of about
    1; log l adds 2 of itself, at most 0.1.  The difference is taken to a few u of itself, 2^x has 2 ulp (4 u);
    g / T, its product and the sum add 4 u of g p / T.  Weights far below 1 carry errors of theirs: 30 u each."""
    R, V = 256, 300
    x, at = rows(R, V, *((34.0, 62.0) if sign > 0 else (-62.0, -34.0)), T, 14.0, dtype, seed=int(10 * T))
    rng = np.random.default_rng(1)
    g = torch.tensor(rng.choice([-1.0, 1.0], R) * rng.uniform(0.5, 2.0, R), dtype=F32, device=DEV)
    temperature = torch.full((R,), T, dtype=F32, device=DEV)
    targets = torch.from_numpy(at.astype(np.int32)).to(DEV)
    r = binding.logprobs(x, targets, temperature=temperature)
    assert float(r.logz.abs().min()) > 32 and float(r.logz.abs().max()) < 64
    got = binding.logprobs_grad(x, targets, r.logz, r.entropy, g, temperature=temperature)
    got = got.double().cpu().numpy()[np.arange(R), at]
    v = x.double().cpu().numpy()
    T = float(temperature[0])
    t = (v - v[np.arange(R), at][:, None]) / T
    w = np.exp(t)
    w[np.arange(R), at] = 0.0
    rest = w.sum(1)
    want = g.double().cpu().numpy() / T * (rest / (1 + rest))
    assert rest.max() < 0.1
    tol = np.abs(g.double().cpu().numpy()) / T * U * (32 + V / 128 + 24 + 1 + 4 + 4 + 30 * rest)
    tol += (torch.finfo(dtype).eps / 2 * 1.01 + 4 * U) * np.abs(want)
    err = np.abs(got - want)
    assert (err <= tol).all(), (float((err / tol).max()), float((err * T / U).max()))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("mask", [-math.inf, "lowest"])
@pytest.mark.parametrize("V", [7, 300, 1001])
def test_masked_tokens_at_any_temperature(V, mask, dtype):
    """Masked tokens get exactly 0, the others what they get without them: zeros for any of many temperatures,
    whose parts of log2 e / T have either sign."""
    R = 64
    rng = np.random.default_rng(V)
    T = rng.uniform(0.5, 3.0, R).astype(np.float32)
    x = torch.from_numpy(rng.standard_normal((R, V)) + 8).to(dtype).to(DEV)
    x[:, 1::3] = torch.finfo(dtype).min if mask == "lowest" else mask
    targets = torch.zeros(R, dtype=torch.int32, device=DEV)
    targets[1] = 1  # (a masked one: g / T alone)
    temperature = torch.from_numpy(T).to(DEV)
    g, h, k = (torch.tensor(rng.standard_normal(R), dtype=F32, device=DEV) for _ in range(3))
    r = binding.logprobs(x, targets, temperature=temperature)
    assert float(r.logz.abs().max()) < 64
    got = binding.logprobs_grad(x, targets, r.logz, r.entropy, g, h, k, temperature=temperature)
    assert torch.isfinite(got).all()
    masked = got[:, 1::3].clone()
    assert abs(float(masked[1, 0]) - float(g[1]) / float(T[1])) <= 2.0 ** -7 * abs(float(g[1]) / float(T[1]))
    masked[1, 0] = 0
    assert (masked == 0).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("V", [8, 301])
def test_masked_tokens_of_large_coefficients(V, dtype):
    """A gradient of the entropy near the type's end: masked tokens get 0, whatever 0 would be multiplied by."""
    rng = np.random.default_rng(V)
    x = torch.from_numpy(rng.standard_normal((4, V))).to(dtype).to(DEV)
    x[:, 2::3] = -math.inf
    targets = torch.full((4,), -1, dtype=torch.int32, device=DEV)
    h = torch.tensor([3e36, -3e36, 1e35, 2e37], dtype=F32, device=DEV)
    r = binding.logprobs(x, targets)
    got = binding.logprobs_grad(x, targets, r.logz, r.entropy, None, h).double().cpu().numpy()
    assert (got[:, 2::3] == 0).all()
    v, hh = x.double().cpu().numpy(), h.double().cpu().numpy()[:, None]
    logp = v - np.log(np.exp(v).sum(1, keepdims=True))
    p = np.exp(logp)
    with np.errstate(invalid="ignore"):
        plogp = np.where(p > 0, p * logp, 0.0)
    H = -plogp.sum(1, keepdims=True)
    want = -hh * (plogp + p * H)
    # log p and H are off by 60 u of 1 and of themselves (at most 64 additions of each, and logz's rounding)
    tol = 60 * U * np.abs(hh) * p * (2 + np.abs(np.where(p > 0, logp, 0)) + 2 * H) + 1.01 * torch.finfo(dtype).eps / 2 * np.abs(want)
    assert (np.abs(got - want) <= tol).all()
