"""relation_page_plan on the GPU: block tables, slots, positions and the ring of free pages, equal to
a plain request-by-request plan; what does not fit is refused and the rest served."""
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


def world(rng, B, page, cols, spare, longest, fill=1.0):
    """Requests with lengths up to a share of their table rows, distinct pages, a rotated ring."""
    lengths = rng.integers(0, max(1, int(fill * cols * page) - longest) + 1, B).astype(np.int32)
    counts = rng.integers(0, longest + 1, B).astype(np.int32)
    counts[rng.random(B) < 0.15] = -1
    used = -(-lengths // page)
    n_pages = int(used.sum()) + spare
    perm = rng.permutation(n_pages).astype(np.int32)
    table = np.full((B, cols), -7, np.int32)
    at = 0
    for b in range(B):
        table[b, :used[b]] = perm[at:at + used[b]]
        at += used[b]
    head = int(rng.integers(0, n_pages))
    free = np.full(n_pages, -9, np.int32)
    for i in range(spare):
        free[(head + i) % n_pages] = perm[at + i]
    return lengths, counts, table, free, np.array([head, spare], np.int32)


def run(args, page, n_tokens, out=None, stride=None):
    dev = [torch.from_numpy(a).to(DEV) for a in args]
    if stride:  # a table whose rows are strided
        wide = torch.full((args[2].shape[0], stride), -5, dtype=torch.int32, device=DEV)
        wide[:, :args[2].shape[1]] = dev[2]
        dev[2] = wide[:, :args[2].shape[1]]
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    p = binding.page_plan(dev[0], dev[1], dev[2], dev[3], dev[4], page, n_tokens, out=out,
                          dev_status=status)
    torch.cuda.synchronize()
    got = [x.cpu().numpy() for x in (p.slots, p.positions, p.starts, p.lengths, p.free_state,
                                     dev[2], dev[3])]
    return got, int(status.item()), dev


def same(got, want):
    for name, g, w in zip(("slots", "positions", "starts", "lengths", "state", "table", "free"),
                          got, want):
        assert np.array_equal(g, w), (name, np.flatnonzero((g != w).reshape(-1))[:5])


@pytest.mark.parametrize("B,page,longest", [(1, 16, 1), (1, 1, 5), (7, 24, 100), (64, 16, 1),
                                            (511, 8, 3), (512, 8, 3), (513, 7, 40), (1500, 32, 90),
                                            (3, 64, 20000)])
def test_plan_equals_the_request_by_request_plan(B, page, longest):
    rng = np.random.default_rng(B * 1000 + page)
    cols = max(4, (longest + 200) // page + 3)
    w = world(rng, B, page, cols, B * (longest // page + 2), longest)
    total = int(np.maximum(w[1], 0).sum())
    for n_tokens in (max(1, total), total + 37):
        got, status, dev = run(w, page, n_tokens)
        same(got, su.plan(*w, page, n_tokens))
        assert status == binding.OK
        # the same call again: nothing it reads has changed but the entries it wrote alike
        p = binding.page_plan(*dev, page, n_tokens)
        torch.cuda.synchronize()
        assert np.array_equal(p.slots.cpu().numpy(), got[0])
        assert np.array_equal(dev[3].cpu().numpy(), got[6])


def test_steps_follow_each_other():
    """Forty steps of a batch that admits, decodes and ends requests: no page is held twice, none
    is lost, and every token lies where its request's table says."""
    rng = np.random.default_rng(5)
    B, page, cols, n_pages, n_tokens = 40, 4, 16, 400, 300
    length = np.zeros(B, np.int32)
    table = np.full((B, cols), -1, np.int32)
    free, state = rng.permutation(n_pages).astype(np.int32), np.array([17, n_pages], np.int32)
    dev = [torch.from_numpy(x).to(DEV) for x in (length, length, table, free, state)]
    for step in range(40):
        counts = np.where(length == 0, rng.integers(0, 12, B), rng.integers(0, 3, B))
        counts[(rng.random(B) < 0.1) & (length > 0)] = -1
        counts = counts.astype(np.int32)
        dev[1] = torch.from_numpy(counts).to(DEV)
        want = su.plan(length, counts, table, free, state, page, n_tokens)
        p = binding.page_plan(*dev, page, n_tokens)
        got = [x.cpu().numpy() for x in (p.slots, p.positions, p.starts, p.lengths, p.free_state,
                                         dev[2], dev[3])]
        same(got, want)
        length, state, table, free = want[3], want[4], want[5], want[6]
        dev[0], dev[4] = p.lengths, p.free_state
        held = [table[b, j] for b in range(B) for j in range(-(-int(length[b]) // page))]
        idle = [free[(state[0] + i) % n_pages] for i in range(state[1])]
        assert sorted(held + idle) == list(range(n_pages))


def test_strided_table_and_given_outputs():
    rng = np.random.default_rng(9)
    w = world(rng, 33, 16, 20, 200, 40)
    n = int(np.maximum(w[1], 0).sum()) + 3
    i32 = lambda *s: torch.empty(s, dtype=torch.int32, device=DEV)  # noqa: E731
    out = binding.PagePlan(torch.empty(n, dtype=torch.int64, device=DEV), i32(n), i32(34), i32(33),
                           i32(2))
    got, status, dev = run(w, 16, n, out=out, stride=29)
    same(got, su.plan(*w, 16, n))
    assert status == binding.OK
    assert (dev[2].as_strided((33, 29), (29, 1))[:, 20:] == -5).all()


@pytest.mark.parametrize("why", ["pages", "tokens", "row"])
def test_requests_that_do_not_fit(why):
    rng = np.random.default_rng(3)
    w = world(rng, 700, 8, 12, 900, 30, fill=1.0)
    total = int(np.maximum(w[1], 0).sum())
    n_tokens = total + 5
    if why == "pages":
        w[4][1] = 100
    elif why == "tokens":
        n_tokens = total // 2
    else:
        w[0][::3] = np.where(w[1][::3] > 0, 12 * 8 - np.maximum(w[1][::3], 0) // 2, w[0][::3])
        w[1][::3] = np.where(w[1][::3] > 1, w[1][::3], 0)
    got, status, _ = run(w, 8, n_tokens)
    same(got, su.plan(*w, 8, n_tokens))
    assert status == binding.ERR_CAPACITY


def test_bad_lengths_and_states_are_reported():
    rng = np.random.default_rng(4)
    w = world(rng, 50, 8, 12, 300, 30)
    w[0][7], w[0][20] = -3, 12 * 8 + 1
    got, status, _ = run(w, 8, 2000)
    same(got, su.plan(*w, 8, 2000))
    assert status == binding.ERR_INVALID_ARG
    w = world(rng, 50, 8, 12, 300, 30)
    w[4][:] = (len(w[3]), 5)
    got, status, _ = run(w, 8, 2000)
    same(got, su.plan(*w, 8, 2000))
    assert status == binding.ERR_INVALID_ARG
    w = world(rng, 50, 8, 12, 300, 30)
    w[1][:] = -1  # every page back into a ring that says it is nearly full
    w[4][1] = len(w[3]) - 10
    got, status, _ = run(w, 8, 2000)
    same(got, su.plan(*w, 8, 2000))
    assert status == binding.ERR_INVALID_ARG


def test_refusals():
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device=DEV)  # noqa: E731
    ok = [i32(4), i32(4), i32(4, 8), i32(32), i32(2)]
    binding.page_plan(*ok, 16, 8)
    for at, bad in ((0, i32(4).long()), (1, i32(5)), (2, i32(3, 8)), (2, i32(8, 4).T),
                    (3, i32(32).float()), (4, i32(3))):
        args = list(ok)
        args[at] = bad
        with pytest.raises(ValueError):
            binding.page_plan(*args, 16, 8)
    for page, n in ((0, 8), (16, 0), (1 << 30, 8)):
        with pytest.raises((binding.RelationError, RuntimeError)):
            binding.page_plan(*ok, page, n)
    p = binding.page_plan(*ok, 16, 8)
    with pytest.raises(binding.RelationError):  # lengths_out on top of lengths
        binding.page_plan(*ok, 16, 8, out=p._replace(lengths=ok[0]))
