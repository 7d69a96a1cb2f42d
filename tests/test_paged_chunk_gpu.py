"""relation_paged_chunk against the rows in fp64: types, shared key heads, ragged requests, pages, strides,
odd widths, padding, infinities and NaN, bad positions and pages, many pieces, streams, capture."""
import numpy as np
import pytest
import torch

from paper_2608_20172_gb300 import binding
from tests import chunk_util as cu

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    binding.load()


def queries(N, H, d, dtype, seed=0, pad=0, scale=1.0):
    rng = np.random.default_rng(seed + 100)
    x = torch.full((N, H, d + pad), 7.0, dtype=dtype, device=DEV)[..., :d]
    return x.copy_(torch.from_numpy(rng.standard_normal((N, H, d)) * scale))


class Step:
    """One call's inputs and the rows in fp64."""

    def __init__(self, counts, lengths, H, Hk, d, dtype, page, *, lam=0.5, extra=0, seed=0, pad=0, scale=1.0,
                 **kw):
        self.N, self.lam, self.H = sum(counts) + extra, lam, H
        self.cache = cu.Cache(lengths, Hk, d, dtype, page, seed=seed, pad=pad, **kw)
        self.q = queries(self.N, H, d, dtype, seed, pad, scale)
        self.starts, self.pos = cu.tokens(counts, lengths, self.N)
        self.up()

    def up(self):
        self.t_starts, self.t_pos = (torch.from_numpy(x).to(DEV) for x in (self.starts, self.pos))

    def run(self, **kw):
        c = self.cache
        return binding.paged_chunk(self.q, c.k, c.v, c.block_table, self.t_starts, self.t_pos, self.lam, **kw)

    def want(self):
        q = self.q.double().cpu().numpy()
        out = [np.zeros(q.shape), np.full(q.shape[:2], -INF), np.zeros(q.shape), np.zeros(q.shape[:2] + (2,))]
        for b in range(len(self.starts) - 1):
            s = slice(self.starts[b], min(self.starts[b + 1], self.N))
            if s.stop > s.start:
                K, V = self.cache.request(b)
                for o, x in zip(out, cu.rows(q[s], self.pos[s], K, V, self.lam)):
                    o[s] = x
        return out

    def check(self, status=binding.OK, rows=slice(None), **kw):
        st = torch.zeros(1, dtype=torch.int32, device=DEV)
        y, logz = self.run(dev_status=st, **kw)
        assert int(st) == status
        Y, Z, W, big = (x[rows] for x in self.want())
        y, logz = y.double().cpu().numpy()[rows], logz.double().cpu().numpy()[rows]
        ytol, ztol = cu.bounds(Y, Z, W, big, self.q.shape[2], self.cache.dtype, self.lam, max(self.pos.max(), 1))
        none = np.isinf(Z)
        assert np.array_equal(np.isinf(logz), none) and (y[none] == 0).all()
        err = np.where(none, 0, np.abs(np.where(none, 0, logz) - np.where(none, 0, Z)))
        assert (err <= ztol).all(), f"logz off by {err.max()}, {(err / ztol).max()} of its bound"
        err = np.abs(y - Y)
        assert (err <= ytol + 1e-37).all(), f"Y off by {err.max()}, {(err / (ytol + 1e-37)).max()} of its bound"
        return y, logz


FORMS = [  # counts, lengths, H, Hk, d, page
    ([1], [1], 1, 1, 64, 16), ([2], [2], 2, 1, 64, 16), ([1], [300], 4, 4, 64, 16), ([5], [200], 12, 12, 64, 16),
    ([64, 1, 0, 130], [64, 77, 50, 400], 4, 4, 64, 16), ([129], [129], 2, 2, 128, 64),
    ([3, 200, 1], [3, 256, 1000], 8, 2, 128, 24), ([70, 9], [500, 9], 6, 2, 80, 7), ([33], [66], 5, 1, 96, 1),
    ([40, 1], [700, 900], 16, 2, 32, 1000), ([17, 4], [60, 100], 3, 3, 8, 32), ([128], [640], 1, 1, 128, 128),
    ([100, 28, 1, 1], [1500, 28, 2000, 64], 8, 8, 48, 20)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("counts,lengths,H,Hk,d,page", FORMS)
def test_rows(counts, lengths, H, Hk, d, page, dtype):
    Step(counts, lengths, H, Hk, d, dtype, page, extra=2).check()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [1, 2, 20, 33, 65, 127])
def test_odd_widths(d, dtype):
    Step([30, 2], [140, 90], 4, 2, d, dtype, 10, extra=1).check()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("kw", [dict(pad=8), dict(pad=1), dict(layout="phtd"), dict(layout="phtd", pad=3),
                                dict(lam=0.0), dict(lam=-1.0), dict(lam=3.0)])
def test_layouts_and_lambda(kw, dtype):
    Step([60, 5], [200, 133], 4, 2, 64, dtype, 24, extra=1, seed=1, **kw).check()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_table_rows_are_strided(dtype):
    s = Step([6, 7], [90, 50], 2, 2, 64, dtype, 16, seed=2)
    wide = torch.full((2, 40), -5, dtype=torch.int32, device=DEV)
    wide[:, :s.cache.table.shape[1]] = s.cache.block_table
    s.cache.block_table = wide[:, :s.cache.table.shape[1]]
    s.check()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_large_scores(dtype, d):
    """Scores up to hundreds, growing along the request: the scale is raised late and often."""
    s = Step([90], [400], 2, 1, d, dtype, 16, seed=3, scale=3.0)
    grow = torch.linspace(0.1, 4.0, 400)
    for r in range(400):
        page, row = s.cache.place(0, r)
        s.cache.store[0][page, row] *= grow[r]
    s.cache.upload()
    s.check()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("H,Hk,d", [(4, 4, 64), (8, 1, 64), (2, 2, 128), (2, 1, 72)])
def test_many_pieces(H, Hk, d, dtype):
    """Few rows over thousands of keys: every tile in many pieces, some requests in one."""
    Step([4, 1, 2], [9000, 5000, 30], H, Hk, d, dtype, 64, seed=4).check()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_many_requests(dtype):
    rng = np.random.default_rng(7)
    lengths = rng.integers(1, 60, 1500)
    counts = np.minimum(lengths, rng.integers(0, 4, 1500))
    Step(counts.tolist(), lengths.tolist(), 2, 1, 32, dtype, 16, seed=5, extra=3).check()


def test_more_tiles_than_the_plan_has_threads():
    """1100 tiles of a request each, and a head for every one of many."""
    Step([1] * 1100, [3 + i % 70 for i in range(1100)], 1, 1, 64, BF16, 16, seed=6).check()
    Step([200], [300], 70, 70, 64, BF16, 16, seed=6).check()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_padding_inside_and_outside(dtype):
    """Requests that were not served (positions -1), a buffer that ends before the last request, tokens before
    the first request and behind the last."""
    s = Step([10, 150, 20], [40, 300, 33], 4, 2, 64, dtype, 16, seed=8, extra=30)
    s.pos[10:160] = -1
    s.up()
    s.check()
    s = Step([10, 20], [40, 33], 4, 2, 64, dtype, 16, seed=8)
    s.N = 25  # the last request does not fit the buffer: a step's plan leaves it out
    s.q, s.pos = s.q[:25], s.pos[:25].copy()
    s.pos[10:] = -1
    s.up()
    s.check()
    s = Step([10, 20], [40, 33], 4, 2, 64, dtype, 16, seed=8, extra=9)
    s.pos = np.roll(s.pos, 4)
    s.starts += 4
    s.up()
    s.check()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_every_token_is_padding(dtype):
    s = Step([6, 130], [40, 200], 2, 2, 64, dtype, 16)
    s.pos[:] = -1
    s.up()
    s.check()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_positions_in_any_order(dtype):
    """Tokens of a request need not follow each other."""
    s = Step([150, 3], [400, 3000], 4, 2, 64, dtype, 16, seed=9)
    rng = np.random.default_rng(0)
    s.pos[:150] = rng.permutation(400)[:150]
    s.pos[20] = -1
    s.pos[150:] = [2999, 0, 1500]
    s.up()
    s.check()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("many", [False, True])
def test_bad_positions_and_pages_are_reported(dtype, many):
    n = 4000 if many else 100
    s = Step([8, 9], [n, 60], 2, 2, 64, dtype, 16, seed=10)
    plain, plain_z = s.run()
    s.pos[3] = s.cache.table.shape[1] * 16
    s.pos[5] = 2 ** 31 - 1
    s.up()
    y, z = s.check(status=binding.ERR_INVALID_ARG, rows=[0, 1, 2, 4, 6, 7, *range(8, 17)])
    got, gz = s.run()
    assert (got[[3, 5]] == 0).all() and (gz[[3, 5]] == -INF).all()
    s = Step([8, 9], [n, 60], 2, 2, 64, dtype, 16, seed=10)
    for bad in (-1, s.cache.k.shape[0], 2 ** 31 - 1):
        s.cache.block_table[0, 2] = bad
        st = torch.zeros(1, dtype=torch.int32, device=DEV)
        y, z = s.run(dev_status=st)
        assert int(st) == binding.ERR_INVALID_ARG
        assert torch.equal(y[8:], plain[8:]) and torch.equal(z[8:], plain_z[8:])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d,pad", [(64, 0), (128, 0), (80, 3)])
@pytest.mark.parametrize("n", [150, 3000])
def test_infinities_among_the_values(n, d, pad, dtype):
    """An infinite or NaN value reaches the rows that see it, in its channel, and no others."""
    count = 140
    s = Step([count, 5], [n, 20], 2, 2, d, dtype, 16, seed=11, pad=pad)
    first = n - count
    plain, plain_z = s.run()
    bad = [(first + 3, 0, 1, INF), (first + 70, 0, 5, -INF), (n - 1, 1, 2, NAN), (first + 100, 1, d - 1, INF),
           (first + 130, 1, d - 1, -INF)]
    if first > 0:
        bad.append((first - 1, 0, 7, INF))
    if first > 200:
        bad.append((5, 1, 9, -INF))
    want = plain.clone()
    for row, h, c, x in bad:
        page, r = s.cache.place(0, row)
        s.cache.store[1][page, r, h, c] = x
        at = want[max(0, row - first):count, h, c]
        at += x  # (finite + infinity, opposite ones NaN)
    s.cache.upload()
    y, z = s.run()
    assert torch.equal(z, plain_z)
    assert torch.equal(y.isnan(), want.isnan())
    assert torch.equal(y.nan_to_num(nan=0.0), want.nan_to_num(nan=0.0))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [150, 3000])
def test_nan_among_the_keys_and_queries(n, d, dtype):
    """NaN in a key reaches the rows that see it; in a query its row; behind a row and behind a request's end
    nothing does."""
    count = 140
    s = Step([count, 5], [n, 23], 2, 2, d, dtype, 16, seed=12)
    first = n - count
    plain, plain_z = s.run()
    page, r = s.cache.place(0, first + 60)
    s.cache.store[0][page, r, 1, 3] = NAN
    for b, end in ((0, n), (1, 23)):
        for row in range(end, -(-end // 16) * 16):  # the last page's rows past the request
            page, r = int(s.cache.table[b, row // 16]), row % 16
            s.cache.store[0][page, r] = NAN
            s.cache.store[1][page, r] = INF
    s.cache.upload()
    s.q[7, 0, 5] = NAN
    y, z = s.run()
    seen = torch.zeros((count + 5, 2), dtype=torch.bool, device=DEV)
    seen[60:count, 1] = True
    seen[7, 0] = True
    assert torch.equal(y.isnan().all(-1), seen) and torch.equal(z.isnan(), seen)
    assert torch.equal(y[~seen], plain[~seen]) and torch.equal(z[~seen], plain_z[~seen])


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_agrees_with_decode_and_forward(dtype):
    """A chunk of one token is the decode step's row; a whole sequence's chunk is the forward."""
    d, H, n = 64, 4, 260
    s = Step([n], [n], H, H, d, dtype, 16, seed=13)
    y, z = s.run()
    K, V = (torch.from_numpy(x).to(dtype).to(DEV)[None] for x in s.cache.request(0))
    fy, fz = binding.fwd(s.q[None].contiguous(), K, V, s.lam)
    # each is within its bound of the rows in 64 bits, so that two are within twice of it of each other
    ytol, ztol = (torch.from_numpy(2 * x).to(DEV) for x in
                  cu.bounds(*s.want(), d, dtype, s.lam, n))
    assert ((y.double() - fy[0].double()).abs() <= ytol).all()
    assert ((z.double() - fz[0].t().double()).abs() <= ztol).all()
    dy, dz = binding.paged_decode(s.q[-1:].contiguous(), s.cache.k, s.cache.v, s.cache.block_table,
                                  torch.tensor([n], dtype=torch.int32, device=DEV), s.lam)
    one = Step([1], [n], H, H, d, dtype, 16, seed=13)
    one.q = s.q[-1:].contiguous()
    oy, oz = one.run()
    assert ((oy.double() - dy.double()).abs() <= ytol[-1:]).all()
    assert ((oz.double() - dz.double()).abs() <= ztol[-1:]).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_again_in_place_and_neighbours(dtype):
    """The same bits again, with the output in the queries' place, and nothing beside the rows written."""
    s = Step([70, 3], [500, 2500], 4, 2, 64, dtype, 16, seed=14, pad=8, extra=2)
    a, az = s.run()
    b, bz = s.run()
    assert torch.equal(a, b) and torch.equal(az, bz)
    wide = s.q.as_strided((s.N, 4, 72), s.q.stride())
    c, cz = s.run(out=s.q)
    assert torch.equal(a, c) and torch.equal(az, cz) and (wide[..., 64:] == 7).all()


def test_stream_and_capture():
    s = Step([40, 1, 7], [900, 3000, 7], 4, 2, 64, BF16, 16, seed=15, extra=4)
    want = s.run()
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    got = s.run(stream=st)
    torch.cuda.current_stream().wait_stream(st)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = s.run()
    # other counts and positions on replay: the host knows none of them
    counts, lengths = [1, 44, 3], [850, 2990, 5]
    starts, pos = cu.tokens(counts, lengths, s.N)
    s.t_starts.copy_(torch.from_numpy(starts))
    s.t_pos.copy_(torch.from_numpy(pos))
    want = s.run()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_calls_after_one_another():
    """Calls whose tensors each overwrites for the next, without and with a synchronisation between them."""
    outs = []
    for sync in (False, True):
        s = Step([30, 2], [600, 4000], 4, 2, 64, BF16, 16, seed=16)
        ws = torch.empty(binding.paged_chunk_workspace_size(s.q, s.cache.k, s.cache.block_table),
                         dtype=torch.uint8, device=DEV)
        for i in range(6):
            y, z = s.run(workspace=ws)
            s.q.add_(y, alpha=0.1)
            s.t_pos[31] -= 100
            if sync:
                torch.cuda.synchronize()
        outs.append((s.q.clone(), z))
    assert all(torch.equal(a, b) for a, b in zip(*outs))


def test_binding_refuses():
    s = Step([4], [20], 4, 2, 64, BF16, 16)
    c = s.cache
    call = lambda **kw: binding.paged_chunk(**{**dict(  # noqa: E731
        q=s.q, k_pages=c.k, v_pages=c.v, block_table=c.block_table, starts=s.t_starts, positions=s.t_pos,
        lam=0.5), **kw})
    for kw in (dict(q=s.q.float()), dict(q=s.q[..., :32]), dict(starts=s.t_starts.long()),
               dict(positions=s.t_pos[:3]), dict(block_table=c.block_table.t()), dict(v_pages=c.v.float()),
               dict(out=s.q.float()), dict(logz=torch.zeros(3, device=DEV)), dict(starts=s.t_starts[:1])):
        with pytest.raises(ValueError):
            call(**kw)
    with pytest.raises(binding.RelationError):
        call(workspace=torch.empty(64, dtype=torch.uint8, device=DEV))
    with pytest.raises(binding.RelationError):
        call(q=s.q[:, :3].contiguous())
