"""relation_paged_decode on the GPU against the row in fp64: every head of ragged requests over shuffled
pages, query heads that share keys, page sizes that do not divide anything, both layouts and types.

Bounds: a score is a dot product of d <= 128 normals in fp32, off by about sqrt(d) 2^-24 of sums of
|q_c k_c| / sqrt(d), below 1e-5; the weights' relative error is twice that, and so is Y's against the
largest |v|: 1e-4 max|v| leaves a factor of five; bf16 adds half an ulp of Y, 2^-8 |Y| (8 significant bits).  logZ: 1e-4."""
import numpy as np
import pytest
import torch

from paper_2608_20172_gb300 import binding
from tests import serving_util as su

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    binding.load()


def cache(rng, lengths, page, Hk, d, dtype, layout="pthd", pad=0, cols=None, std=1.0):
    """Rows of every request, and the same in shuffled pages: (rows, k_pages, v_pages, table)."""
    used = [-(-n // page) for n in lengths]
    n_pages = sum(used) + 2
    perm = rng.permutation(n_pages)
    cols = cols or max(max(used), 1)
    table = np.full((len(lengths), cols), -1, np.int32)
    a, b = (page, Hk) if layout == "pthd" else (Hk, page)
    kp, vp = (torch.full((n_pages, a, b, d + pad), float("nan"), dtype=dtype)[..., :d]
              for _ in range(2))
    if layout != "pthd":
        kp, vp = kp.transpose(1, 2), vp.transpose(1, 2)
    rows, at = [], 0
    for i, n in enumerate(lengths):
        k, v = (torch.from_numpy(rng.standard_normal((n, Hk, d)) * s).to(dtype) for s in (std, 1.0))
        for j in range(used[i]):
            table[i, j] = perm[at + j]
            m = min(page, n - j * page)
            kp[table[i, j], :m], vp[table[i, j], :m] = k[j * page:j * page + m], v[j * page:j * page + m]
        at += used[i]
        rows.append((k.double().numpy(), v.double().numpy()))
    put = lambda x: torch.empty_strided(x.size(), x.stride(), dtype=dtype, device=DEV).copy_(x)  # noqa: E731
    return rows, put(kp), put(vp), torch.from_numpy(table).to(DEV)


def check(lengths, H, Hk, d, page, dtype=torch.bfloat16, lam=0.5, layout="pthd", pad=0, cols=None,
          seed=0, std=1.0, heads=None, requests=None):
    rng = np.random.default_rng(seed)
    rows, kp, vp, table = cache(rng, lengths, page, Hk, d, dtype, layout, pad, cols, std)
    B = len(lengths)
    q = torch.from_numpy(rng.standard_normal((B, H, d)) * std).to(dtype)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    y, lz = binding.paged_decode(q.to(DEV), kp, vp, table,
                                 torch.tensor(lengths, dtype=torch.int32, device=DEV), lam,
                                 dev_status=status)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    y, lz = y.double().cpu().numpy(), lz.double().cpu().numpy()
    half = 2.0 ** -8 if dtype == torch.bfloat16 else 0.0
    for b in (range(B) if requests is None else requests):
        if lengths[b] == 0:
            assert (y[b] == 0).all() and (lz[b] == -np.inf).all()
            continue
        wy, wz = su.decode_row(q[b].double().numpy(), *rows[b], lam)
        tol = half * np.abs(wy) + 1e-4 * np.abs(rows[b][1]).max()
        assert (np.abs(y[b] - wy) <= tol).all(), (b, lengths[b], np.abs(y[b] - wy).max())
        assert np.abs(lz[b] - wz).max() <= 1e-4, (b, lengths[b], np.abs(lz[b] - wz).max())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [8, 32, 64, 80, 128])
def test_ragged_lengths(dtype, d):
    check([1, 2, 3, 0, 64, 65, 66, 300, 513, 1200], 2, 2, d, 16, dtype, seed=d)


@pytest.mark.parametrize("H,Hk", [(2, 1), (6, 2), (8, 2), (16, 2), (5, 1), (7, 1), (24, 2), (9, 1)])
def test_shared_keys(H, Hk):
    check([1, 700, 33, 0, 129], H, Hk, 64, 16, seed=H)
    check([1, 90, 33], H, Hk, 128, 16, torch.float32, seed=H)


@pytest.mark.parametrize("page", [1, 3, 7, 8, 24, 64, 100, 1000])
def test_page_sizes(page):
    check([1, 5, 64, 200, 777, 0], 4, 2, 64, page, seed=page)
    check([65, 400], 2, 2, 80, page, torch.float32, seed=page)


@pytest.mark.parametrize("layout", ["pthd", "phtd"])
@pytest.mark.parametrize("pad", [0, 8, 3, 1])
def test_layouts_and_unaligned_rows(layout, pad):
    check([3, 250, 90], 4, 2, 64, 16, layout=layout, pad=pad, seed=pad)
    check([3, 250, 90], 2, 2, 64, 16, torch.float32, layout=layout, pad=pad, seed=pad)


@pytest.mark.parametrize("d", [1, 7, 33, 100, 127])
def test_odd_head_sizes(d):
    check([2, 130, 300], 3, 3, d, 16, seed=d)
    check([2, 130], 8, 2, d, 16, torch.float32, seed=d)


@pytest.mark.parametrize("lam", [0.0, -1.0, 3.0])
def test_lambda(lam):
    check([7, 640, 2], 2, 2, 64, 16, lam=lam, seed=3)


@pytest.mark.parametrize("B", [1, 200, 700])
def test_many_and_few_requests(B):
    """Runs of several requests, requests of several runs, and fewer units than runs."""
    rng = np.random.default_rng(B)
    lengths = rng.integers(0, 400 if B > 1 else 9000, B)
    lengths[0] = 6000
    check(lengths.tolist(), 4, 4, 64, 16, seed=B, requests=sorted({0, 1 % B, B // 2, B - 1}))


def test_sharp_rows_raise_the_scale_late():
    """Scores that grow along the history: the running maximum is raised in many tiles."""
    rng = np.random.default_rng(1)
    rows, kp, vp, table = cache(rng, [3000], 16, 2, 64, torch.float32)
    k, v = rows[0]
    grow = np.linspace(0.05, 12.0, 3000)[:, None, None]
    k = (k * 0.05 + grow / 8.0).astype(np.float32)
    flat = torch.from_numpy(k).to(DEV)
    for j in range(-(-3000 // 16)):
        m = min(16, 3000 - 16 * j)
        kp[int(table[0, j]), :m] = flat[16 * j:16 * j + m]
    q = np.ones((1, 2, 64), np.float32)
    y, lz = binding.paged_decode(torch.from_numpy(q).to(DEV), kp, vp, table,
                                 torch.tensor([3000], dtype=torch.int32, device=DEV), 0.5)
    wy, wz = su.decode_row(q[0].astype(np.float64), k.astype(np.float64), v, 0.5)
    # scores reach 96, each off by up to 64 2^-24 of itself, 4e-4 at the top
    assert np.abs(y[0].double().cpu().numpy() - wy).max() <= 1e-3 * np.abs(v).max()
    assert np.abs(lz[0].double().cpu().numpy() - wz).max() <= 1e-3


def test_nan_reaches_its_rows_and_no_others():
    rng = np.random.default_rng(2)
    rows, kp, vp, table = cache(rng, [500, 500], 16, 2, 64, torch.bfloat16)
    kp[int(table[0, 20]), 3, 1, 5] = float("nan")
    vp[int(table[1, 2]), 1, 0, 9] = float("nan")
    q = torch.from_numpy(rng.standard_normal((2, 4, 64))).to(torch.bfloat16).to(DEV)
    y, lz = binding.paged_decode(q, kp, vp, table,
                                 torch.tensor([500, 500], dtype=torch.int32, device=DEV), 0.5)
    bad = torch.isnan(y).cpu()
    assert bad[0, 2:].all() and not bad[0, :2].any()
    assert bad[1, :2, 9].all() and int(bad[1].sum()) == 2
    assert torch.isnan(lz[0, 2:]).all() and not torch.isnan(lz[1]).any()


def test_equals_contiguous_decode():
    """The same rows in a contiguous cache through relation_decode: equal up to bf16 rounding."""
    rng = np.random.default_rng(6)
    B, T, H, d, page = 3, 640, 4, 64, 16
    lengths = torch.tensor([640, 1, 333], dtype=torch.int32, device=DEV)
    k, v = (torch.from_numpy(rng.standard_normal((B, T, H, d))).to(torch.bfloat16).to(DEV)
            for _ in range(2))
    q = torch.from_numpy(rng.standard_normal((B, H, d))).to(torch.bfloat16).to(DEV)
    table = torch.arange(B * T // page, dtype=torch.int32, device=DEV).view(B, T // page)
    y0, z0 = binding.decode(q, k, v, lengths, 0.5)
    y1, z1 = binding.paged_decode(q, k.view(-1, page, H, d), v.view(-1, page, H, d), table, lengths,
                                  0.5)
    assert (y0.float() - y1.float()).abs().max() <= 2.0 ** -8 * y0.float().abs().max()
    assert (z0 - z1).abs().max() <= 1e-5


def test_strided_table_given_buffers_and_stream():
    rng = np.random.default_rng(8)
    rows, kp, vp, table = cache(rng, [90, 200], 16, 2, 64, torch.bfloat16)
    wide = torch.full((2, table.shape[1] + 5), 10 ** 6, dtype=torch.int32, device=DEV)
    wide[:, :table.shape[1]] = table
    lengths = torch.tensor([90, 200], dtype=torch.int32, device=DEV)
    q = torch.from_numpy(rng.standard_normal((2, 2, 64))).to(torch.bfloat16).to(DEV)
    y0, z0 = binding.paged_decode(q, kp, vp, table, lengths, 0.5)
    ws = torch.empty(binding.paged_decode_workspace_size(q, kp), dtype=torch.uint8, device=DEV)
    out, logz = torch.empty_like(q), torch.empty((2, 2), device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y1, z1 = binding.paged_decode(q, kp, vp, wide[:, :table.shape[1]], lengths, 0.5, out=out,
                                  logz=logz, workspace=ws, stream=side)
    side.synchronize()
    assert y1 is out and torch.equal(y0, y1) and torch.equal(z0, z1)


def test_bad_lengths_and_pages_are_reported():
    rng = np.random.default_rng(8)
    rows, kp, vp, table = cache(rng, [90, 200, 64], 16, 2, 64, torch.bfloat16)
    q = torch.from_numpy(rng.standard_normal((3, 2, 64))).to(torch.bfloat16).to(DEV)
    cap = table.shape[1] * 16
    for lengths in ([90, cap + 1, 64], [90, -1, 64]):
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        y, lz = binding.paged_decode(q, kp, vp, table,
                                     torch.tensor(lengths, dtype=torch.int32, device=DEV), 0.5,
                                     dev_status=status)
        assert int(status.item()) == binding.ERR_INVALID_ARG
        assert (y[1] == 0).all() and (lz[1] == -float("inf")).all()
        assert torch.isfinite(lz[0]).all() and torch.isfinite(lz[2]).all()
    for bad in (-1, kp.shape[0], 1 << 30):
        broken = table.clone()
        broken[1, 3] = bad
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        binding.paged_decode(q, kp, vp, broken,
                             torch.tensor([90, 200, 64], dtype=torch.int32, device=DEV), 0.5,
                             dev_status=status)
        assert int(status.item()) == binding.ERR_INVALID_ARG


def test_refusals():
    rng = np.random.default_rng(8)
    rows, kp, vp, table = cache(rng, [90, 200], 16, 2, 64, torch.bfloat16)
    q = torch.zeros((2, 4, 64), dtype=torch.bfloat16, device=DEV)
    lengths = torch.tensor([90, 200], dtype=torch.int32, device=DEV)
    good = [q, kp, vp, table, lengths]
    binding.paged_decode(*good, 0.5)
    for at, bad in ((0, q.float()), (0, q[:, :, :32]), (2, vp[:1]), (3, table.long()),
                    (3, table[:1]), (4, lengths.long()), (4, lengths[:1])):
        args = list(good)
        args[at] = bad
        with pytest.raises((ValueError, TypeError)):
            binding.paged_decode(*args, 0.5)
    small = torch.empty(64, dtype=torch.uint8, device=DEV)
    for args, kw in ((good, dict(workspace=small)), (good, dict(tau_s=0.0)),
                     ([q[:, :3]] + good[1:], {})):
        with pytest.raises((binding.RelationError, RuntimeError)):
            binding.paged_decode(*args, 0.5, **kw)
