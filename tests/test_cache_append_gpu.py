"""relation_cache_append on the GPU: rotated queries, keys and mixed values in their slots of the
pages against fp64, in both element types, aligned and not, token- and head-major pages.

Bound per element: the angle is rounded to fp32 once (|r| <= pi: 1.2e-7), its sine and cosine are
within 2 ulp (2.4e-7) and the two products and their sum rounded (1.8e-7), together below 1e-6 of the
pair's |x0| + |x1|; bf16 adds half an ulp of the result, 2^-8 of it (8 significant bits)."""
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


def tokens(g, N, H, d, dtype, layout="nhd", pad=0):
    """[N, H, d] with d contiguous; `pad` elements between rows, head-major if "hnd"."""
    a, b = (N, H) if layout == "nhd" else (H, N)
    x = torch.randn((a, b, d + pad), generator=g).to(dtype).to(DEV)[..., :d]
    return x if layout == "nhd" else x.transpose(0, 1)


def pages(n, page, H, d, dtype, layout="pthd", pad=0):
    a, b = (page, H) if layout == "pthd" else (H, page)
    x = torch.full((n, a, b, d + pad), 7.0, dtype=dtype, device=DEV)[..., :d]
    return x if layout == "pthd" else x.transpose(1, 2)


def check(N, H, d, page, dtype, *, layout="nhd", p_layout="pthd", pad=0, base=1e4, pairing=0,
          mix=True, positions=None, queries=True, seed=0):
    g = torch.Generator().manual_seed(seed)
    rng = np.random.default_rng(seed)
    p1, p2, info = (tokens(g, N, H, d, dtype, layout, pad) for _ in range(3))
    theta = torch.randn(H // 2, generator=g).to(DEV) if mix else None
    n_pages = N // page + 3
    slots = rng.permutation(n_pages * page)[:N].astype(np.int64)
    slots[rng.random(N) < 0.1] = -1
    pos = rng.integers(0, 40000, N) if positions is None else np.resize(positions, N)
    kp, vp = (pages(n_pages, page, H, d, dtype, p_layout, pad) for _ in range(2))
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    q = binding.cache_append(p1 if queries else None, p2, info, theta,
                             torch.from_numpy(pos.astype(np.int32)).to(DEV),
                             torch.from_numpy(slots).to(DEV), kp, vp, pairing, base,
                             dev_status=status)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    f8 = lambda t: t.double().cpu().numpy()  # noqa: E731
    # (the base is an fp32 argument)
    turn = lambda x: su.rope(x, pos, float(np.float32(base))) if base else x  # noqa: E731
    live = slots >= 0
    x1, x2, xi = f8(p1), f8(p2), f8(info)
    want_v = su.givens(xi, theta.double().cpu().numpy(), pairing) if mix else xi
    half = 2.0 ** -8 if dtype == torch.bfloat16 else 0.0
    size = lambda x: np.abs(x).max(-1, keepdims=True) * 2 + np.zeros_like(x)  # noqa: E731

    def near(name, got, want, scale):
        tol = half * np.abs(want) + 1e-6 * scale
        bad = np.abs(got - want) > tol
        assert not bad.any(), (name, np.argwhere(bad)[:4], np.abs(got - want).max())

    def pair(x):  # |x0| + |x1| of the pair of every element
        return np.repeat(np.abs(x[..., 0::2]) + np.abs(x[..., 1::2]), 2, -1) if base else np.abs(x)

    if queries:
        near("q", f8(q), turn(x1) * live[:, None, None], pair(x1))
    else:
        assert q is None
    rows = lambda t: f8(t).reshape(n_pages * page, H, d)  # noqa: E731
    k, v = rows(kp.contiguous()), rows(vp.contiguous())
    near("k", k[slots[live]], turn(x2)[live], pair(x2)[live])
    near("v", v[slots[live]], want_v[live], 2 * np.abs(xi).max(1, keepdims=True)[live])
    rest = np.setdiff1d(np.arange(n_pages * page), slots[live])
    assert (k[rest] == 7).all() and (v[rest] == 7).all()
    if pad:  # the bytes between rows are not touched
        whole = kp.as_strided((kp.untyped_storage().nbytes() // kp.element_size(),), (1,))
        assert int((whole == 7).sum()) >= n_pages * page * H * pad


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N,H,d,page", [(1, 2, 64, 16), (3, 12, 64, 16), (64, 16, 128, 64),
                                        (301, 8, 80, 24), (1300, 4, 48, 1), (1217, 6, 256, 7),
                                        (5, 2, 8, 3)])
def test_append(dtype, N, H, d, page):
    check(N, H, d, page, dtype, seed=N)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("how", [dict(layout="hnd"), dict(p_layout="phtd"), dict(pad=8),
                                 dict(pad=3), dict(pairing=1), dict(mix=False), dict(base=0.0),
                                 dict(queries=False), dict(base=0.7), dict(base=5e5),
                                 dict(pad=3, pairing=1, layout="hnd", p_layout="phtd")])
def test_layouts_and_options(dtype, how):
    check(77, 6, 64, 16, dtype, seed=7, **how)
    check(1300, 6, 64, 16, dtype, seed=8, **how)


@pytest.mark.parametrize("d,mix,base", [(62, True, 1e4), (2, True, 1e4), (63, True, 0.0),
                                        (33, False, 0.0), (1, True, 0.0)])
def test_odd_head_sizes(d, mix, base):
    check(90, 4, d, 16, torch.bfloat16, mix=mix, base=base)
    check(90, 4, d, 16, torch.float32, mix=mix, base=base)


def test_odd_heads_without_mixing():
    check(20, 3, 64, 16, torch.bfloat16, mix=False)


@pytest.mark.parametrize("positions", [[0], [1], [32767, 32768, 32769], [1 << 20, (1 << 24) - 1],
                                       [0, 100000]])
def test_positions(positions):
    check(65, 2, 64, 16, torch.float32, positions=np.array(positions))


def test_query_in_place():
    g = torch.Generator().manual_seed(1)
    p1, p2, info = (tokens(g, 40, 4, 64, torch.bfloat16) for _ in range(3))
    theta = torch.randn(2, generator=g).to(DEV)
    pos = torch.arange(40, dtype=torch.int32, device=DEV)
    slots = torch.arange(40, device=DEV)
    kp, vp = (pages(3, 16, 4, 64, torch.bfloat16) for _ in range(2))
    q = binding.cache_append(p1, p2, info, theta, pos, slots, kp, vp)
    same = p1.clone()
    assert binding.cache_append(same, p2, info, theta, pos, slots, kp, vp, out=same) is same
    assert torch.equal(q, same)


def test_slot_past_the_pages_is_reported():
    g = torch.Generator().manual_seed(1)
    p1, p2, info = (tokens(g, 3, 2, 64, torch.bfloat16) for _ in range(3))
    slots = torch.tensor([5, 32, 1 << 40], device=DEV)
    pos = torch.zeros(3, dtype=torch.int32, device=DEV)
    kp, vp = (pages(2, 16, 2, 64, torch.bfloat16) for _ in range(2))
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    q = binding.cache_append(p1, p2, info, None, pos, slots, kp, vp, dev_status=status)
    torch.cuda.synchronize()
    assert int(status.item()) == binding.ERR_INVALID_ARG
    assert (q[1:] == 0).all() and torch.equal(vp[0, 5], info[0])
    assert int((vp != 7).any(-1).any(-1).sum()) == 1


def test_refusals():
    g = torch.Generator().manual_seed(1)
    x = tokens(g, 3, 2, 64, torch.bfloat16)
    pos, slots = torch.zeros(3, dtype=torch.int32, device=DEV), torch.arange(3, device=DEV)
    kp, vp = (pages(2, 16, 2, 64, torch.bfloat16) for _ in range(2))
    theta = torch.zeros(1, device=DEV)
    good = [x, x, x, theta, pos, slots, kp, vp]
    binding.cache_append(*good)
    for at, bad in ((0, x[:2]), (1, x.float()), (3, torch.zeros(2, device=DEV)), (4, pos[:2]),
                    (5, slots.int()), (7, vp[:1]), (6, kp.float())):
        args = list(good)
        args[at] = bad
        with pytest.raises((ValueError, TypeError)):
            binding.cache_append(*args)
    for kw in (dict(pairing=2), dict(rope_base=-1.0), dict(rope_base=float("nan"))):
        with pytest.raises(binding.RelationError):
            binding.cache_append(*good, **kw)
    with pytest.raises(binding.RelationError):  # no positions to rotate by
        binding.cache_append(x, x, x, theta, None, slots, kp, vp)
