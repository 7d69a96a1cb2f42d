"""relation_sample on the GPU against the distribution in fp64, and against its own definition in
whole numbers written out with elementary torch operations.

Bounds: a weight exp((x - max) / T) is off by the rounding of its argument (|x - max| / T <= 28 where
it counts: 1.7e-6) and 1 ulp, so masses and their logarithms agree to 4e-6 relative; a token is
compared where the uniform number lies further than that from both ends of its interval, and a row
where its top-p and min-p cuts do."""
import math

import numpy as np
import pytest
import torch

from paper_2608_20172_gb300 import binding
from tests import serving_util as su

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = 4e-6


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    binding.load()


def call(x, u, **kw):
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    t = {n: torch.tensor(v, dtype=torch.int32 if n == "top_k" else torch.float32, device=DEV)
         for n, v in kw.items()}
    out = binding.sample(x, torch.as_tensor(u, dtype=torch.float32, device=DEV), **t,
                         dev_status=status)
    torch.cuda.synchronize()
    return [o.cpu().numpy() for o in out], int(status.item())


def defined(x, u, temperature=None, top_k=None, top_p=None, min_p=None):
    """The token and the kept mass of one fp32 row by the definition in whole numbers."""
    t = 1.0 if temperature is None else float(np.float32(temperature))
    top = x.max()
    if t == 0:
        w, k = (x == top).float(), 1
    else:
        s = 1.0 / torch.tensor(t, dtype=torch.float32, device=x.device)
        w, k = torch.exp((x - top) * s), 0 if top_k is None else top_k
        w = torch.where(x == top, torch.ones_like(w), w)
    q = (w * 2.0 ** 40).long()
    ws, order = torch.sort(w, dim=0, descending=True, stable=True)
    qs = q[order]
    keep = torch.ones_like(ws, dtype=torch.bool)
    if k > 0:
        keep[k:] = False
    qs = torch.where(keep, qs, torch.zeros_like(qs))
    if top_p is not None and top_p < 1:
        want = math.floor(float(np.float32(top_p)) * float(int(qs.sum())))
        before = qs.cumsum(0) - qs
        keep &= before < max(want, 1)
    if min_p is not None:
        keep &= ws >= min(float(np.float32(min_p)), 1.0)
    kept = torch.zeros_like(keep)
    kept[order] = keep
    q = torch.where(kept, q, torch.zeros_like(q))
    total = int(q.sum())
    target = min(math.floor(float(np.float32(u)) * float(total)), total - 1)
    return int((q.cumsum(0) <= target).sum()), total


def logits(rng, R, V, dtype=torch.float32, std=2.5, ties=False):
    x = rng.standard_normal((R, V)) * std
    x[:, :: max(1, V // 40)] += rng.uniform(0, 8, x[:, :: max(1, V // 40)].shape)
    if ties:
        x = np.round(x * 2) / 2
    return torch.from_numpy(x).to(dtype).to(DEV)


def compare(x, rng, share=0.5, **kw):
    """Every row against the definition, and against fp64 where its cuts are clear (at least `share`
    of the rows); returns the tokens."""
    R, V = x.shape
    u = rng.random(R).astype(np.float32)
    (token, logprob, logz), status = call(x, u, **{n: np.broadcast_to(v, (R,)).copy()
                                                   for n, v in kw.items()})
    assert status == 0
    sure = 0
    for r in range(R):
        one = {n: (int if n == "top_k" else float)(np.broadcast_to(v, (R,))[r]) for n, v in kw.items()}
        row = x[r].float()
        assert token[r] == defined(row, u[r], **one)[0], (r, one)
        f = {n: float(np.float32(v)) if n != "top_k" else v for n, v in one.items()}
        full = row.double().cpu().numpy()
        kept, w = su.kept_tokens(full, **f)
        # cuts that 32-bit weights may place elsewhere
        if "top_p" in f:
            lo, hi = (len(su.kept_tokens(full, **{**f, "top_p": f["top_p"] * (1 + s * EPS)})[0])
                      for s in (-1, 1))
            if lo != hi:
                continue
        if "min_p" in f:
            lo, hi = (len(su.kept_tokens(full, **{**f, "min_p": f["min_p"] * (1 + s * EPS)})[0])
                      for s in (-1, 1))
            if lo != hi:
                continue
        t = 1.0 if f.get("temperature", 1.0) == 0 else f.get("temperature", 1.0)
        want = full.max() / t + math.log(w.sum())
        assert abs(logz[r] - want) <= EPS * max(1.0, abs(want)) + 2e-6, (r, logz[r], want)
        c = np.cumsum(w)
        at = float(u[r]) * c[-1]
        i = int(np.searchsorted(kept, token[r]))
        assert i < len(kept) and kept[i] == token[r], (r, token[r])
        assert c[i] - w[i] - EPS * c[-1] <= at <= c[i] + EPS * c[-1]
        assert abs(logprob[r] - math.log(w[i] / c[-1])) <= 4 * EPS
        sure += 1
    assert sure >= share * R
    return token


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [1, 2, 31, 33, 1000, 4096, 4097, 20011, 50257, 131072])
def test_plain_sampling(dtype, V):
    rng = np.random.default_rng(V)
    compare(logits(rng, 5, V, dtype), rng)
    compare(logits(rng, 3, V, dtype), rng, temperature=[0.3, 1.0, 2.5])


@pytest.mark.parametrize("V", [131071, 131073, 150001, 262144])
def test_long_slices(V):
    """Vocabularies on both sides of the longest slice that shares an SM, up to the longest served."""
    rng = np.random.default_rng(V)
    x = logits(rng, 3, V)
    compare(x, rng, top_k=[0, 40, 3000], top_p=[0.9, 0.95, 1.0], share=0)
    compare(logits(rng, 3, V, torch.bfloat16), rng, top_p=0.8, share=0)
    compare(torch.zeros((2, V), device=DEV), rng, top_k=[V - 7, 5], share=0)


@pytest.mark.parametrize("R", [38, 43, 50, 60, 76, 101, 152, 153, 320])
def test_clusters_of_any_size(R):
    """A row's CTAs by the number of rows: 8 down to 1."""
    rng = np.random.default_rng(R)
    x = logits(rng, R, 20011, torch.bfloat16)
    u = rng.random(R).astype(np.float32)
    kw = dict(temperature=rng.choice([0.0, 0.7, 1.0], R), top_k=rng.choice([0, 5, 300], R),
              top_p=rng.choice([1.0, 0.9], R), min_p=rng.choice([0.0, 0.05], R))
    whole, _ = call(x, u, **kw)
    for r in range(R):
        one = {n: (int if n == "top_k" else float)(v[r]) for n, v in kw.items()}
        assert whole[0][r] == defined(x[r].float(), u[r], **one)[0]


@pytest.mark.parametrize("ties", [False, True])
@pytest.mark.parametrize("V", [2, 50, 4000, 32000, 100003])
def test_top_k(V, ties):
    rng = np.random.default_rng(V)
    x = logits(rng, 8, V, ties=ties)
    compare(x, rng, top_k=[1, 2, 5, 40, 1000, 20000, V, 0])
    compare(x, rng, top_k=[1, 3, 7, 50, 100, 2000, -1, V + 5], temperature=0.7)


@pytest.mark.parametrize("ties", [False, True])
@pytest.mark.parametrize("V", [2, 50, 4000, 32000, 100003])
def test_top_p(V, ties):
    rng = np.random.default_rng(V + 1)
    x = logits(rng, 8, V, ties=ties)
    # (of equal weights a share may end exactly between two tokens)
    share = 0.25 if ties else 0.5
    compare(x, rng, share, top_p=[1e-6, 0.1, 0.5, 0.8, 0.9, 0.95, 0.999, 1.0])
    compare(x, rng, share, top_p=0.9, top_k=[1, 2, 10, 50, 200, 1000, 0, 0],
            temperature=[0.5, 0.7, 1.0, 1.0, 1.3, 2.0, 4.0, 0.0])


@pytest.mark.parametrize("V", [50, 32000])
def test_min_p(V):
    rng = np.random.default_rng(V + 2)
    x = logits(rng, 8, V)
    compare(x, rng, min_p=[0.0, 1e-4, 0.01, 0.05, 0.1, 0.5, 1.0, 2.0])
    compare(x, rng, min_p=0.02, top_p=0.9, top_k=[5, 0, 100, 0, 50, 0, 1000, 20])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_flat_rows(dtype):
    """Equal logits everywhere: the ties go by index through every cut."""
    rng = np.random.default_rng(3)
    for V in (7, 5000, 70001):
        x = torch.full((6, V), 1.25, dtype=dtype, device=DEV)
        compare(x, rng, top_k=[0, 1, 3, V // 2, V - 1, V])
        compare(x, rng, 0, top_p=[0.9999, 0.5, 0.25, 0.1, 1e-9, 0.75])


def test_greedy_takes_the_largest_logit_lowest_index():
    rng = np.random.default_rng(4)
    x = logits(rng, 6, 40000, torch.bfloat16, ties=True)
    # logits that differ by less than a weight's rounding
    y = torch.zeros((1, 9000), device=DEV)
    y[0, 5000], y[0, 7000] = 1e-9, 1e-9
    for t in (x, y):
        (token, logprob, logz), _ = call(t, np.full(t.shape[0], 0.99), temperature=np.zeros(t.shape[0]))
        want = [int((r == r.max()).nonzero()[0]) for r in t.float()]
        assert token.tolist() == want
        assert (logprob == 0).all() and np.array_equal(logz, t.float().amax(1).cpu().numpy())


@pytest.mark.parametrize("V", [100, 40000])
def test_masked_rows(V):
    rng = np.random.default_rng(5)
    for dtype in (torch.float32, torch.bfloat16):
        x = logits(rng, 6, V, dtype)
        x[0, torch.rand(V, device=DEV) > 0.05] = -math.inf
        x[1, 1:] = -math.inf                     # a single token
        x[2] = -math.inf                         # none
        x[3, ::2] = torch.finfo(dtype).min       # the type's lowest
        x[4] = torch.finfo(dtype).min            # everywhere: all alike
        x[5, V // 2] = math.inf
        for kw in ({}, dict(top_k=np.full(6, 20)), dict(top_p=np.full(6, 0.9)),
                   dict(min_p=np.full(6, 0.05)), dict(temperature=np.full(6, 0.0))):
            u = rng.random(6)
            (token, logprob, logz), status = call(x, u, **kw)
            assert status == 0
            assert token[2] == -1 and logprob[2] == -np.inf and logz[2] == -np.inf
            assert token[1] == 0 and logprob[1] == 0
            assert x[0, token[0]] > -math.inf and token[3] % 2 == 1
            assert 0 <= token[4] < V and token[5] == V // 2
            if not kw:
                assert token[4] == int(np.float32(u[4]) * V)
                assert abs(logprob[4] + math.log(V)) < 1e-5


def test_nan_and_bad_parameters():
    rng = np.random.default_rng(6)
    x = logits(rng, 8, 30000)
    x[1, 29999] = math.nan
    good = np.ones(8)
    (token, logprob, logz), status = call(x, good * 0.5)
    assert status == 0 and token[1] == -1 and np.isnan(logprob[1]) and np.isnan(logz[1])
    assert (np.delete(token, 1) >= 0).all()
    for kw, row in ((dict(temperature=-1.0), 3), (dict(temperature=math.nan), 3),
                    (dict(temperature=math.inf), 3)):
        v = good.copy()
        v[row] = kw["temperature"]
        (token, _, logz), status = call(x, good * 0.5, temperature=v)
        assert status == binding.ERR_INVALID_ARG and token[row] == -1 and np.isnan(logz[row])
        assert (np.delete(token, [1, row]) >= 0).all()
    for bad in (-0.1, 1.5, math.nan):
        u = good * 0.5
        u[4] = bad
        (token, _, _), status = call(x, u)
        assert status == binding.ERR_INVALID_ARG and token[4] == -1
    (token, _, _), status = call(x, good * 0.5, top_p=good * math.nan, min_p=good * math.nan)
    assert status == 0 and (np.delete(token, 1) >= 0).all()  # a NaN cut keeps every token


def test_ends_of_the_unit_interval():
    rng = np.random.default_rng(7)
    x = logits(rng, 2, 20000)
    x[:, 0] = -math.inf
    x[:, 19999] = -math.inf
    (token, _, _), _ = call(x, [0.0, 1.0])
    assert token.tolist() == [1, 19998]


def test_rows_do_not_depend_on_the_batch():
    rng = np.random.default_rng(8)
    x = logits(rng, 300, 9001, torch.bfloat16)
    u = rng.random(300).astype(np.float32)
    kw = dict(temperature=rng.choice([0.0, 0.7, 1.0], 300), top_k=rng.choice([0, 5, 300], 300),
              top_p=rng.choice([1.0, 0.9], 300), min_p=rng.choice([0.0, 0.05], 300))
    whole, _ = call(x, u, **kw)
    for r in range(0, 300, 23):
        alone, _ = call(x[r:r + 1], u[r:r + 1], **{n: v[r:r + 1] for n, v in kw.items()})
        for a, b in zip(alone, whole):
            assert a[0] == b[r]


def test_strided_rows_and_given_outputs():
    rng = np.random.default_rng(9)
    wide = logits(rng, 4, 10007, torch.bfloat16)
    x = wide[:, 3:10001]
    u = torch.rand(4, device=DEV)
    want = binding.sample(x.contiguous(), u)
    out = (torch.empty(4, dtype=torch.int32, device=DEV), torch.empty(4, device=DEV),
           torch.empty(4, device=DEV))
    got = binding.sample(x, u, out=out)
    assert got is out
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_frequencies():
    """65536 draws of one small row follow its probabilities (chi-square at 5 sigma)."""
    rng = np.random.default_rng(10)
    row = logits(rng, 1, 40, std=1.0)
    u = torch.from_numpy(rng.random(65536)).float().to(DEV)
    token, _, _ = binding.sample(row.expand(65536, 40).contiguous(), u)
    p = torch.softmax(row[0].double(), 0).cpu().numpy()
    seen = np.bincount(token.cpu().numpy(), minlength=40)
    chi = ((seen - 65536 * p) ** 2 / (65536 * p)).sum()
    assert chi < 39 + 5 * math.sqrt(2 * 39)


def test_refusals():
    x, u = torch.zeros((3, 50), device=DEV), torch.zeros(3, device=DEV)
    binding.sample(x, u)
    for args, kw in (((x[0], u), {}), ((x, u[:2]), {}), ((x, u.double()), {}),
                     ((x.T, u), {}), ((x.double(), u), {}), ((x, u), dict(top_k=u)),
                     ((x, u), dict(temperature=u[:1])), ((x, u), dict(top_p=u.cpu()))):
        with pytest.raises((ValueError, TypeError)):
            binding.sample(*args, **kw)
    big = torch.zeros((1, 400000), device=DEV)
    with pytest.raises(binding.RelationError):
        binding.sample(big, u[:1])
