"""Performance cases of the serving operators: pages of the key/value cache planned from request
lengths, new tokens rotated, mixed and written into their pages, one new token per request read
against them, and the next token drawn from its logits.

``listed()`` names the fixed cases and ``draw(rng)`` gives one more of the same ranges;
``prepare`` makes what a program holds before the call, ``run`` is one pass (with ``own`` through
``paper_2608_20172_gb300.binding``, otherwise in elementary torch operations), ``work`` the bytes
and operations the pass cannot do without, and ``exact`` the results in 64 bits.

Kinds
  plan    block tables, slots and positions of the new tokens, and the ring of free pages, from
          request lengths and counts (count -1: the request has ended, its pages go back)
  append  RoPE of the new tokens' coordinates at their positions and Givens mixing of their
          information, keys and information written to the tokens' slots of the paged cache
  decode  the Relation row of one new token per request over its pages
  sample  a token per row from given uniform numbers: temperature, top-k, top-p, min-p
"""
from __future__ import annotations

import math

import torch

own = False

TAU_S = 2.0
ROPE_BASE = 1.0e4
FIXED = 2.0 ** 40  # a token's sampling weight is a whole number of 2^-40 of the largest


def listed():
    return [
        # One decoding step of a full batch: a token per request, a page now and then.
        dict(name="plan_step", kind="plan", B=64, page=16, cols=512, longest=1, n_tokens=64),
        # A step that decodes some requests and prefills chunks of others, some having ended.
        dict(name="plan_mixed", kind="plan", B=333, page=24, cols=400, longest=2048, n_tokens=20000),
        # Many requests admitted at once with their whole prompts: the largest plan.
        dict(name="plan_admit", kind="plan", B=2048, page=32, cols=256, longest=256,
             n_tokens=131072),
        # The layer's transforms and cache write of one decoding step.
        dict(name="append_step", kind="append", dtype="bf16", N=32, H=12, d=64, page=16,
             layout="pthd"),
        # A ragged chunk in full precision, 80-wide heads, pages that are no power of two.
        dict(name="append_ragged_fp32", kind="append", dtype="fp32", N=1001, H=8, d=80, page=24,
             layout="pthd"),
        # Prompts of 32k tokens together, head-major pages: the largest write.
        dict(name="append_prompt", kind="append", dtype="bf16", N=32768, H=16, d=128, page=64,
             layout="phtd"),
        # One user's step against a cache of moderate size: latency.
        dict(name="decode_single", kind="decode", dtype="bf16", B=1, H=12, G=1, T=2048, d=64,
             page=16, layout="pthd", lam=0.5),
        # Query heads that share keys, odd pages, ragged requests, one idle and one just begun.
        dict(name="decode_grouped", kind="decode", dtype="bf16", B=48, H=24, G=4, T=3000, d=80,
             page=24, layout="pthd", lam=0.3),
        # Serving: a full batch of long ragged requests: the largest case.
        dict(name="decode_batch", kind="decode", dtype="bf16", B=32, H=16, G=1, T=8192, d=128,
             page=64, layout="pthd", lam=0.5),
        # One user's next token: a small vocabulary, the usual top-k and top-p.
        dict(name="sample_one", kind="sample", dtype="fp32", R=1, V=32000, mode="topk_topp"),
        # A batch whose requests ask for different things, bf16 rows of odd length, some
        # masked by a grammar.
        dict(name="sample_mixed", kind="sample", dtype="bf16", R=64, V=50257, mode="mixed"),
        # A large batch over a large vocabulary with top-p alone: the longest candidate lists.
        dict(name="sample_topp", kind="sample", dtype="fp32", R=256, V=131072, mode="topp"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["plan", "append", "decode", "decode", "sample", "sample"])
    if kind == "plan":
        B, page = _log_int(rng, 1, 2048), rng.choice([8, 16, 24, 32, 64])
        longest = rng.choice([1, _log_int(rng, 2, 2048)])
        return dict(kind=kind, B=B, page=page, cols=max(8, 8192 // page), longest=longest,
                    n_tokens=min(131072, B * max(1, longest * 3 // 4) + 7))
    if kind == "append":
        H, d = rng.choice([2, 4, 6, 8, 12, 16]), rng.choice([32, 48, 64, 80, 96, 128])
        return dict(kind=kind, dtype=rng.choice(["bf16", "bf16", "fp32"]), H=H, d=d,
                    N=_log_int(rng, 1, 16384), page=rng.choice([8, 16, 24, 32, 64, 128]),
                    layout=rng.choice(["pthd", "phtd"]))
    if kind == "decode":
        G = rng.choice([1, 1, 1, 2, 4, 8])
        Hk = rng.choice([h for h in (1, 2, 4, 8, 12, 16) if h * G <= 32])
        return dict(kind=kind, dtype=rng.choice(["bf16", "bf16", "bf16", "fp32"]), G=G, H=Hk * G,
                    B=_log_int(rng, 1, 32), T=_log_int(rng, 40, 8192),
                    d=rng.choice([32, 64, 64, 80, 128, 128]), page=rng.choice([8, 16, 24, 64, 128]),
                    layout=rng.choice(["pthd", "pthd", "phtd"]), lam=round(rng.uniform(0.0, 1.0), 3))
    return dict(kind=kind, dtype=rng.choice(["bf16", "fp32"]), R=_log_int(rng, 1, 256),
                V=_log_int(rng, 2000, 131072),
                mode=rng.choice(["topk_topp", "topp", "minp", "full", "mixed", "mixed"]))


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------
def _dt(case):
    return torch.float32 if case["dtype"] == "fp32" else torch.bfloat16


def _gen(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    return gen


def _pages(case, gen, n, empty=False, mean=0.0):
    """n pages of a cache [n, page, H, d], stored token-major or head-major within a page; every
    channel has a mean of its own."""
    H, page, d = case["H"] // case.get("G", 1), case["page"], case["d"]
    shape = (n, page, H, d) if case["layout"] == "pthd" else (n, H, page, d)
    if empty:
        x = torch.zeros(shape, device="cuda", dtype=_dt(case))
    else:
        x = torch.randn(shape, generator=gen, device="cuda")
        x = x.add_(torch.randn(d, generator=gen, device="cuda") * mean).to(_dt(case))
    return x if case["layout"] == "pthd" else x.transpose(1, 2)


def _prepare_plan(case, gen):
    B, page, cols = case["B"], case["page"], case["cols"]
    i32, dev = torch.int32, "cuda"
    # requests anywhere between their first token and a row of their table short of its end
    room = cols * page - case["longest"]
    lengths = torch.randint(0, room + 1, (B,), generator=gen, device=dev)
    # counts up to `longest` as long as they fit the step's token buffer; one in sixteen has
    # ended, and where chunks are prefilled half of the requests decode one token
    counts = torch.randint(1, case["longest"] + 1, (B,), generator=gen, device=dev)
    what = torch.rand(B, generator=gen, device=dev)
    counts = torch.where(what < 0.5, torch.ones_like(counts), counts) if case["longest"] > 1 else counts
    counts = torch.where(what > 1 - 1 / 16, torch.full_like(counts, -1), counts)
    counts = torch.where(counts.clamp(min=0).cumsum(0) <= case["n_tokens"], counts,
                         torch.zeros_like(counts))
    used = (lengths + page - 1) // page
    n_pages = B * cols
    perm = torch.randperm(n_pages, generator=gen, device=dev).to(i32)
    # the pages in use first, then the ring of free ones behind a head that has moved on
    first = used.cumsum(0) - used
    col = torch.arange(cols, device=dev)
    held = col[None, :] < used[:, None]
    table = torch.where(held, perm[(first[:, None] + col[None, :]).clamp(max=n_pages - 1)],
                        torch.full((), -1, dtype=i32, device=dev))
    head = int(torch.randint(0, n_pages, (1,), generator=gen, device=dev))
    free = torch.roll(torch.roll(perm, -int(used.sum())), head)
    return {"lengths": lengths.to(i32), "counts": counts.to(i32), "table": table.contiguous(),
            "free": free.contiguous(), "page": page, "n_tokens": case["n_tokens"],
            "state": torch.tensor([head, n_pages - int(used.sum())], dtype=i32, device=dev)}


def _prepare_append(case, gen):
    N, H, d, page, dt = (case[k] for k in ("N", "H", "d", "page", "dtype"))
    dev = "cuda"
    s = {n: torch.randn((N, H, d), generator=gen, device=dev).to(_dt(case))
         for n in ("p1", "p2", "info")}
    s["theta"] = torch.randn(H // 2, generator=gen, device=dev) * 0.5
    # requests' chunks one after the other: positions run on from where each request stands
    owner = torch.sort(torch.randint(0, max(1, N // 300 + 1), (N,), generator=gen, device=dev))[0]
    begin = torch.randint(0, 16000, (int(owner.max()) + 1,), generator=gen, device=dev)
    at = torch.arange(N, device=dev)
    first = torch.searchsorted(owner, owner)
    s["positions"] = (begin[owner] + at - first).to(torch.int32)
    n_pages = (N + page - 1) // page + 3
    order = torch.randperm(n_pages, generator=gen, device=dev)
    s["slots"] = order[at // page] * page + at % page
    if N > 4:  # the step's buffer ends in padding
        s["slots"][-2:] = -1
        s["positions"][-2:] = -1
    s["k"], s["v"] = _pages(case, gen, n_pages, empty=True), _pages(case, gen, n_pages, empty=True)
    return s


def _prepare_decode(case, gen):
    B, H, T, d, page = (case[k] for k in ("B", "H", "T", "d", "page"))
    dev = "cuda"
    lengths = torch.randint(max(1, T // 4), T + 1, (B,), generator=gen, device=dev)
    if B >= 8:
        lengths[1], lengths[2] = 1, 0
    used = (lengths + page - 1) // page
    cols, total = (T + page - 1) // page, int(used.sum())
    perm = torch.randperm(total + 2, generator=gen, device=dev).to(torch.int32)
    col = torch.arange(cols, device=dev)
    first = used.cumsum(0) - used
    table = torch.where(col[None, :] < used[:, None],
                        perm[(first[:, None] + col[None, :]).clamp(max=total + 1)],
                        torch.full((), -1, dtype=torch.int32, device=dev))
    return {"k": _pages(case, gen, total + 2), "v": _pages(case, gen, total + 2, mean=0.5),
            "q": torch.randn((B, H, d), generator=gen, device=dev).to(_dt(case)),
            "table": table.contiguous(), "lengths": lengths.to(torch.int32), "lam": case["lam"]}


def _prepare_sample(case, gen):
    R, V, mode = case["R"], case["V"], case["mode"]
    dev = "cuda"
    # a broad body and a few likely tokens, sharper in some rows than in others
    x = torch.randn((R, V), generator=gen, device=dev) * 2.0
    few = torch.randint(0, V, (R, 64), generator=gen, device=dev)
    x.scatter_add_(1, few, 4.0 + 8.0 * torch.rand((R, 64), generator=gen, device=dev))
    x.mul_(0.7 + 0.8 * torch.rand((R, 1), generator=gen, device=dev))
    s = {"u": torch.rand(R, generator=gen, device=dev), "temperature": None, "top_k": None,
         "top_p": None, "min_p": None}
    pick = lambda values: torch.tensor(values, device=dev)[  # noqa: E731
        torch.randint(0, len(values), (R,), generator=gen, device=dev)]
    if mode != "full":
        s["temperature"] = pick([0.7, 0.8, 1.0, 1.0, 1.2])
    if mode == "topk_topp":
        s["top_k"], s["top_p"] = pick([20, 40, 50]).to(torch.int32), pick([0.9, 0.95])
    elif mode == "topp":
        s["top_p"] = pick([0.8, 0.9, 0.95])
    elif mode == "minp":
        s["min_p"] = pick([0.02, 0.05, 0.1])
    elif mode == "mixed":
        s["temperature"] = pick([0.0, 0.6, 0.8, 1.0, 1.3])
        s["top_k"] = pick([0, 0, 1, 20, 50, 1000]).to(torch.int32)
        s["top_p"], s["min_p"] = pick([1.0, 0.9, 0.95]), pick([0.0, 0.0, 0.05])
        # a grammar leaves one token in eight: -inf in some rows, the type's lowest in others
        mask = torch.rand((R, V), generator=gen, device=dev) > 1 / 8
        rows = torch.arange(R, device=dev)[:, None] % 4
        x.masked_fill_(mask & (rows == 1), -math.inf)
        x.masked_fill_(mask & (rows == 3), torch.finfo(_dt(case)).min)
    s["logits"] = x.to(_dt(case))
    return s


def prepare(case, seed):
    make = {"plan": _prepare_plan, "append": _prepare_append, "decode": _prepare_decode,
            "sample": _prepare_sample}[case["kind"]]
    s = make(case, _gen(seed))
    s["kind"] = case["kind"]
    return s


# ---------------------------------------------------------------------------
# One pass in elementary operations
# ---------------------------------------------------------------------------
def _plain_plan(s):
    page, n_tokens = s["page"], s["n_tokens"]
    length, count = s["lengths"].long(), s["counts"].long()
    B, cols = s["table"].shape
    n_pages = s["free"].numel()
    head, avail = s["state"][0].long(), s["state"][1].long()
    new = count.clamp(min=0)
    ends = new.cumsum(0)
    fits = (length + new <= cols * page) & (ends <= n_tokens)
    held, want = (length + page - 1) // page, (length + new + page - 1) // page
    need = torch.where(fits, want - held, torch.zeros_like(held))
    upto = need.cumsum(0)
    served = fits & ((upto <= avail) | (need == 0))
    taken = torch.where(upto <= avail, upto, torch.zeros_like(upto)).max()
    given = torch.where(count < 0, held, torch.zeros_like(held))
    given_before = given.cumsum(0) - given
    col = torch.arange(cols, device=length.device)[None, :]
    fresh = served[:, None] & (col >= held[:, None]) & (col < want[:, None])
    at = (head + (upto - need)[:, None] + col - held[:, None]).clamp(min=0) % n_pages
    s["table"].copy_(torch.where(fresh, s["free"][at], s["table"]))
    back = (count < 0)[:, None] & (col < held[:, None])
    to = torch.where(back, (head + avail + given_before[:, None] + col) % n_pages,
                     torch.full_like(col, n_pages))
    ring = torch.cat([s["free"], s["free"][:1]])
    ring[to.reshape(-1)] = s["table"].reshape(-1)
    s["free"].copy_(ring[:n_pages])
    t = torch.arange(n_tokens, device=length.device)
    b = torch.searchsorted(ends, t, right=True).clamp(max=B - 1)
    position = length[b] + t - (ends - new)[b]
    live = (t < ends[-1]) & served[b]
    entry = s["table"][b, (position // page).clamp(0, cols - 1)].long()
    none = torch.full_like(t, -1)
    return {"slots": torch.where(live, entry * page + position % page, none),
            "positions": torch.where(live, position, none).int(),
            "starts": torch.cat([torch.zeros_like(ends[:1]), ends]).int(),
            "lengths": torch.where(count < 0, torch.zeros_like(length),
                                   torch.where(served, length + new, length)).int(),
            "state": torch.stack([(head + taken) % n_pages, avail - taken + given.sum()]).int(),
            "table": s["table"], "free": s["free"]}


def _turned(x, cos, sin):
    even, odd = x[..., 0::2], x[..., 1::2]
    return torch.stack((even * cos - odd * sin, even * sin + odd * cos), -1).reshape(x.shape)


def _mixed(info, theta):
    cos, sin = torch.cos(theta)[:, None], torch.sin(theta)[:, None]
    a, b = info[:, 0::2], info[:, 1::2]
    return torch.stack((cos * a - sin * b, sin * a + cos * b), 2).reshape(info.shape)


def _angles(positions, d):
    """position * base^(-2c/d) modulo 2 pi; positions reach 16k, so the product is in 64 bits."""
    w = ROPE_BASE ** (-torch.arange(0, d, 2, dtype=torch.float64, device=positions.device) / d)
    return torch.remainder(positions.double()[:, None] * w, 2 * math.pi)[:, None, :]


def _write_pages(s, q, k, v):
    page = s["k"].shape[1]
    live = s["slots"] >= 0
    # padding writes the first token again, to the same place
    src = torch.where(live, torch.arange(live.numel(), device=live.device), 0)
    slot = s["slots"][src]
    s["k"][slot // page, slot % page] = k.to(s["k"].dtype)[src]
    s["v"][slot // page, slot % page] = v.to(s["v"].dtype)[src]
    return {"q": torch.where(live[:, None, None], q, torch.zeros_like(q)).to(s["p1"].dtype),
            "k": s["k"], "v": s["v"]}


def _plain_append(s):
    a = _angles(s["positions"], s["p1"].shape[2]).float()
    cos, sin = torch.cos(a), torch.sin(a)
    return _write_pages(s, _turned(s["p1"].float(), cos, sin), _turned(s["p2"].float(), cos, sin),
                        _mixed(s["info"].float(), s["theta"]))


def _relation_rows(q, k, v, lengths, lam):
    """Rows len_b - 1 of the Relation for q [B, H, d] over k, v [B, T, Hk, d], all of one type."""
    B, H, d = q.shape
    T, Hk = k.shape[1:3]
    n = lengths.long()
    q = q.view(B, Hk, H // Hk, d)
    k, v = k.permute(0, 2, 1, 3), v.permute(0, 2, 1, 3)  # [B, Hk, T, d]
    U = torch.matmul(q, k.transpose(2, 3)) * (1.0 / math.sqrt(d))
    own_row = (n - 1).clamp(min=0)
    S = torch.sigmoid(U.gather(3, own_row[:, None, None, None].expand(B, Hk, H // Hk, 1)) / TAU_S)
    E = U / (1.0 + torch.exp(-U))
    past = torch.arange(T, device=q.device)[None, None, None, :] >= (n - 1)[:, None, None, None]
    E = E.masked_fill(past, -math.inf)
    m = E.amax(3, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    P = torch.exp(E - m)
    l = P.sum(3, keepdim=True)
    z = torch.matmul(P, v)
    i = n.clamp(min=1).to(q.dtype)[:, None, None, None]
    A = m + torch.log(l) - lam * torch.log(i)
    g = torch.sigmoid(A - S)
    vi = v[torch.arange(B, device=q.device), :, own_row][:, :, None]
    y = vi + g * (torch.where(l > 0, z / l, vi) - vi)
    logz = torch.logaddexp(S, A)
    idle = (n < 1)[:, None, None, None]
    y = torch.where(idle, torch.zeros_like(y), y)
    logz = torch.where(idle, torch.full_like(logz, -math.inf), logz)
    return y.reshape(B, H, d), logz.reshape(B, H)


def _gathered(s):
    """The requests' rows of the pages, [B, T, Hk, d] (rows past a request's end: page 0's)."""
    page = s["k"].shape[1]
    t = torch.arange(s["table"].shape[1] * page, device=s["k"].device)
    entry = s["table"].long().clamp(min=0)[:, t // page]
    return s["k"][entry, t % page], s["v"][entry, t % page]


def _plain_decode(s):
    k, v = _gathered(s)
    y, logz = _relation_rows(s["q"].float(), k.float(), v.float(), s["lengths"], s["lam"])
    return {"y": y.to(s["q"].dtype), "logz": logz}


def _plain_sample(s):
    x, u = s["logits"].float(), s["u"]
    R, V = x.shape
    ones = torch.ones(R, device=x.device)
    temperature = ones if s["temperature"] is None else s["temperature"]
    greedy = temperature == 0
    scale = torch.where(greedy, ones, ones / temperature)[:, None]
    top = x.amax(1, keepdim=True)
    w = torch.exp((x - top) * scale)
    w = torch.where(x == top, torch.ones_like(w), torch.where(greedy[:, None], torch.zeros_like(w), w))
    weight = (w * FIXED).long()  # whole numbers: their sums are the same in any order
    w_sorted, order = torch.sort(w, dim=1, descending=True, stable=True)
    q_sorted = weight.gather(1, order)
    rank = torch.arange(V, device=x.device)[None, :]
    k = torch.zeros(R, dtype=torch.long, device=x.device) if s["top_k"] is None else s["top_k"].long()
    k = torch.where(greedy, torch.ones_like(k), k)
    k = torch.where(k <= 0, torch.full_like(k, V), k)[:, None]
    keep = rank < k
    q_sorted = torch.where(keep, q_sorted, torch.zeros_like(q_sorted))
    if s["top_p"] is not None:
        before = q_sorted.cumsum(1) - q_sorted
        p = s["top_p"][:, None]
        least = torch.floor(p.double() * q_sorted.sum(1, keepdim=True).double()).long()
        keep &= (before < least) | (p >= 1) | (rank == 0)
    if s["min_p"] is not None:
        keep &= w_sorted >= s["min_p"][:, None].clamp(max=1.0)
    kept = torch.zeros_like(keep).scatter_(1, order, keep)
    weight = torch.where(kept, weight, torch.zeros_like(weight))
    total = weight.sum(1)
    target = torch.minimum(torch.floor(u.double() * total.double()).long(), total - 1)
    token = torch.searchsorted(weight.cumsum(1), target[:, None], right=True)
    logsum = torch.log(total.float() / FIXED)
    logprob = torch.log(w.gather(1, token))[:, 0] - logsum
    return {"token": token[:, 0].int(), "logprob": logprob, "logz": top[:, 0] * scale[:, 0] + logsum}


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------
def run(s):
    kind = s["kind"]
    if not own:
        return {"plan": _plain_plan, "append": _plain_append, "decode": _plain_decode,
                "sample": _plain_sample}[kind](s)
    from paper_2608_20172_gb300 import binding
    if kind == "plan":
        p = binding.page_plan(s["lengths"], s["counts"], s["table"], s["free"], s["state"],
                              s["page"], s["n_tokens"])
        return {"slots": p.slots, "positions": p.positions, "starts": p.starts,
                "lengths": p.lengths, "state": p.free_state, "table": s["table"],
                "free": s["free"]}
    if kind == "append":
        q = binding.cache_append(s["p1"], s["p2"], s["info"], s["theta"], s["positions"],
                                 s["slots"], s["k"], s["v"], rope_base=ROPE_BASE)
        return {"q": q, "k": s["k"], "v": s["v"]}
    if kind == "decode":
        y, logz = binding.paged_decode(s["q"], s["k"], s["v"], s["table"], s["lengths"], s["lam"],
                                       TAU_S)
        return {"y": y, "logz": logz}
    token, logprob, logz = binding.sample(s["logits"], s["u"], temperature=s["temperature"],
                                          top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"])
    return {"token": token, "logprob": logprob, "logz": logz}


# ---------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    kind = case["kind"]
    if kind == "plan":
        # lengths and counts in; slots (8), positions (4), lengths and starts out; the new
        # pages' ids in and out, about one for `page` tokens, and the ended requests' pages
        B, n = case["B"], case["n_tokens"]
        ended = B // 16 * case["cols"] // 2
        return {"bytes": 16 * B + 12 * n + 8 * (n // case["page"] + ended), "flops": 8 * n}
    e = 4 if case.get("dtype") == "fp32" else 2
    if kind == "append":  # three inputs and three outputs, slots and positions
        n = case["N"] * case["H"] * case["d"]
        return {"bytes": 6 * n * e + 12 * case["N"], "flops": 9 * n}
    if kind == "decode":  # lengths are uniform over the upper three quarters
        B, H, d = case["B"], case["H"], case["d"]
        rows = B * (case["T"] * 5 // 8)
        return {"bytes": 2 * rows * (H // case["G"]) * d * e + 2 * B * H * d * e + 4 * B * H
                + 4 * rows // case["page"], "flops": 4 * rows * H * d}
    n = case["R"] * case["V"]
    return {"bytes": n * e + 32 * case["R"], "flops": 4 * n}


# ---------------------------------------------------------------------------
# The same in 64 bits
# ---------------------------------------------------------------------------
def _exact_plan(s):
    """Request by request and page by page, as a host program would do it."""
    page, n_tokens = s["page"], s["n_tokens"]
    lengths, counts = s["lengths"].tolist(), s["counts"].tolist()
    table, free = s["table"].tolist(), s["free"].tolist()
    head, avail = s["state"].tolist()
    n_pages, cols = len(free), len(table[0])
    ring, slots, positions = list(free), [-1] * n_tokens, [-1] * n_tokens
    starts, out, wanted, given, taken = [0], [], 0, 0, 0
    for b, (n, c) in enumerate(zip(lengths, counts)):
        held, first = -(-n // page), starts[-1]
        starts.append(first + max(c, 0))
        if c < 0:
            for j in range(held):
                ring[(head + avail + given + j) % n_pages] = table[b][j]
            given += held
            out.append(0)
            continue
        if n + c > cols * page or first + c > n_tokens:
            out.append(n)
            continue
        need = -(-(n + c) // page) - held
        wanted += need
        if need and wanted > avail:
            out.append(n)
            continue
        for j in range(need):
            table[b][held + j] = free[(head + taken + j) % n_pages]
        taken += need
        for j in range(c):
            slots[first + j] = table[b][(n + j) // page] * page + (n + j) % page
            positions[first + j] = n + j
        out.append(n + c)
    t = lambda x, dt=torch.int32: torch.tensor(x, dtype=dt, device="cuda")  # noqa: E731
    return {"slots": t(slots, torch.int64), "positions": t(positions), "starts": t(starts),
            "lengths": t(out), "state": t([(head + taken) % n_pages, avail - taken + given]),
            "table": t(table), "free": t(ring)}


def _exact_append(s):
    N, H, d = s["p1"].shape
    f8 = torch.float64
    page = s["k"].shape[1]
    w = torch.exp(torch.arange(d // 2, device="cuda", dtype=f8) * (-2.0 / d * math.log(ROPE_BASE)))
    turn = torch.polar(torch.ones((), dtype=f8, device="cuda"), s["positions"].to(f8)[:, None] * w)
    live = s["slots"] >= 0
    out = {}
    for name, src in (("q", "p1"), ("k", "p2")):
        x = torch.view_as_complex(s[src].to(f8).reshape(N, H, d // 2, 2).contiguous())
        out[name] = torch.view_as_real(x * turn[:, None]).reshape(N, H, d)
    th = torch.polar(torch.ones((), dtype=f8, device="cuda"), s["theta"].to(f8))
    x = s["info"].to(f8).reshape(N, H // 2, 2, d)
    x = torch.complex(x[:, :, 0], x[:, :, 1]) * th[None, :, None]
    v = torch.stack((x.real, x.imag), 2).reshape(N, H, d)
    cache = {}
    for name, new in (("k", out["k"]), ("v", v)):
        c = torch.zeros(s[name].shape, dtype=f8, device="cuda")
        c[s["slots"][live] // page, s["slots"][live] % page] = new[live]
        cache[name] = c
    return {"q": out["q"] * live[:, None, None], **cache}


def _exact_decode(s):
    """Request by request over its own rows, the row of R and F written out as defined."""
    B, H, d = s["q"].shape
    page, Hk, f8 = s["k"].shape[1], s["k"].shape[2], torch.float64
    y = torch.zeros((B, H, d), dtype=f8, device="cuda")
    logz = torch.full((B, H), -math.inf, dtype=f8, device="cuda")
    for b, n in enumerate(s["lengths"].tolist()):
        if n < 1:
            continue
        pages = s["table"][b, :-(-n // page)].long()
        K, V = (x[pages].reshape(-1, Hk, d)[:n].to(f8).repeat_interleave(H // Hk, 1)
                for x in (s["k"], s["v"]))
        U = (s["q"][b].to(f8)[None] * K).sum(2) / math.sqrt(d)
        R = U * torch.sigmoid(U) - s["lam"] * math.log(n)
        R[n - 1] = torch.sigmoid(U[n - 1] / TAU_S)
        logz[b] = torch.logsumexp(R, 0)
        y[b] = (torch.exp(R - logz[b])[:, :, None] * V).sum(0)
    return {"y": y, "logz": logz}


def _exact_sample(s):
    """The tokens in descending order of probability, cut off by each rule in turn.  A choice
    that falls within the last bits of 32-bit weights has no value in 64 bits: then token and
    logprob are None."""
    f8 = torch.float64
    R, V = s["logits"].shape
    token, logprob, logz, sure = [], [], [], True
    value = lambda name, r, none: none if s[name] is None else float(s[name][r])  # noqa: E731
    for r in range(R):
        x = s["logits"][r].to(f8)
        t, k = value("temperature", r, 1.0), int(value("top_k", r, 0))
        p, least = value("top_p", r, 1.0), value("min_p", r, 0.0)
        if t == 0:
            t, k = 1.0, 1
        xs, order = torch.sort(x / t, dim=0, descending=True, stable=True)
        w = torch.exp(xs - xs[0])
        n = min(k, V) if k > 0 else V
        if p < 1:
            c = w[:n].cumsum(0)
            n = max(1, int(((c - w[:n]) < p * c[-1]).sum()))
        n = max(1, min(n, int((w >= least).sum())))
        logz.append(xs[0] + torch.log(w[:n].sum()))
        kept, back = torch.sort(order[:n])
        c = w[:n][back].cumsum(0)
        at = float(s["u"][r]) * c[-1]
        j = min(n - 1, int(torch.searchsorted(c, at, right=True)))
        margin = 1e-6 * float(c[-1])
        sure &= j == n - 1 or float(c[j] - at) > margin
        sure &= j == 0 or float(at - c[j - 1]) > margin
        token.append(kept[j])
        logprob.append(torch.log(w[back[j]] / c[-1]))
    return {"token": torch.stack(token).int() if sure else None,
            "logprob": torch.stack(logprob) if sure else None, "logz": torch.stack(logz)}


def exact(case, seed):
    s = prepare(case, seed)
    return {"plan": _exact_plan, "append": _exact_append, "decode": _exact_decode,
            "sample": _exact_sample}[case["kind"]](s)
