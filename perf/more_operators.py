"""Performance cases of the operators around a prompt that is served, scored or trained on in chunks:
queries and keys normed per head and rotated, a chunk of new tokens read against the paged cache, and
the log probabilities of given tokens, with the gradients of the first and the last.

``listed()`` names the fixed cases and ``draw(rng)`` gives one more of the same ranges;
``prepare`` makes what a program holds before the call, ``run`` is one pass (with ``own`` through
``paper_2608_20172_gb300.binding``, otherwise in elementary torch operations), ``work`` the bytes
and operations the pass cannot do without, and ``exact`` the results in 64 bits.

Kinds
  rotate       RMS norm of every query and key head with its weights, and the rotation of the first
               d_rot channels by the token's position, in either layout of the pairs
  rotate_grad  its gradient: coordinates and weights
  chunk        the Relation rows of several new tokens per request over the request's pages
  score        log probability of a given token per row, the row's entropy and its top alternatives
  score_grad   the logits' gradient from those of the log probabilities and entropies
"""
from __future__ import annotations

import math

import torch

own = False

TAU_S = 2.0
EPS = 1.0e-6


def listed():
    return [
        # One decoding step's queries and keys: latency.
        dict(name="rotate_step", kind="rotate", dtype="bf16", N=32, H=12, G=1, d=64, d_rot=64,
             layout="interleaved", reach=4096),
        # Prompts of 32k tokens, shared key heads, a long context's frequencies: the largest.
        dict(name="rotate_prompt", kind="rotate", dtype="bf16", N=32768, H=32, G=4, d=128,
             d_rot=128, layout="half", reach=131072),
        # Training in full precision: an odd number of tokens, a part of an 80-wide head.
        dict(name="rotate_grad_fp32", kind="rotate_grad", dtype="fp32", N=1001, H=8, G=4, d=80,
             d_rot=40, layout="half", reach=2048),
        # A training batch of 16k tokens, half of every head rotated.
        dict(name="rotate_grad_batch", kind="rotate_grad", dtype="bf16", N=16384, H=16, G=1, d=128,
             d_rot=64, layout="interleaved", reach=2048),
        # A few drafted tokens of one user's request checked at once: latency.
        dict(name="chunk_draft", kind="chunk", dtype="bf16", B=1, C=5, N=5, H=12, G=1, T=2048, d=64,
             page=16, layout="pthd", lam=0.5),
        # A serving step: half of the requests decode, the others bring pieces of their prompts.
        dict(name="chunk_mixed", kind="chunk", dtype="bf16", B=48, C=512, N=8192, H=32, G=4, T=3000,
             d=80, page=24, layout="pthd", lam=0.3),
        # Full precision, ragged, a head width and pages that are no power of two, head-major.
        dict(name="chunk_ragged_fp32", kind="chunk", dtype="fp32", B=3, C=150, N=451, H=8, G=2,
             T=1000, d=72, page=20, layout="phtd", lam=0.7),
        # Pieces of long prompts: the largest case.
        dict(name="chunk_prompt", kind="chunk", dtype="bf16", B=4, C=2048, N=8192, H=16, G=1,
             T=16384, d=128, page=64, layout="pthd", lam=0.5),
        # The token that one user's request has just drawn, with five alternatives: latency.
        dict(name="score_one", kind="score", dtype="fp32", R=1, V=32000, top=5, mode="plain"),
        # A prompt's tokens, rows of odd length, with twenty alternatives, temperatures and masks.
        dict(name="score_prompt", kind="score", dtype="bf16", R=2048, V=50257, top=20,
             mode="masked"),
        # A short sequence's loss in full precision.
        dict(name="score_grad_short", kind="score_grad", dtype="fp32", R=32, V=32000,
             mode="plain"),
        # A training batch on sampled tokens, with an entropy term and rows without a target.
        dict(name="score_grad_batch", kind="score_grad", dtype="bf16", R=4096, V=50257,
             mode="masked"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["rotate", "rotate_grad", "chunk", "chunk", "chunk", "score", "score_grad"])
    if kind in ("rotate", "rotate_grad"):
        G = rng.choice([1, 1, 2, 4, 8])
        Hk = rng.choice([h for h in (1, 2, 3, 4, 8, 12, 16) if h * G <= 32])
        d = rng.choice([32, 48, 64, 64, 80, 96, 128, 128, 256])
        d_rot = rng.choice([d, d, d // 2, d // 4 // 2 * 2])
        return dict(kind=kind, dtype=rng.choice(["bf16", "bf16", "fp32"]), G=G, H=Hk * G, d=d,
                    d_rot=d_rot, layout=rng.choice(["interleaved", "half"]),
                    reach=rng.choice([2048, 32768, 1 << 20]),
                    N=_log_int(rng, 1, (1 << 26) // (Hk * G * d)))
    if kind == "chunk":
        dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
        G = rng.choice([1, 1, 2, 3, 4, 8])
        Hk = rng.choice([h for h in (1, 2, 4, 8, 16) if h * G <= 32])
        B, T = _log_int(rng, 1, 48), _log_int(rng, 40, 8192)
        # what the plain form holds of scores, and the largest listed case's work
        most = (1 << 29) if dtype == "bf16" else (1 << 26)
        C = _log_int(rng, 1, max(1, min(T, 2048, most // (B * Hk * G * T))))
        return dict(kind=kind, dtype=dtype, G=G, H=Hk * G, B=B, C=C, N=B * C + rng.choice([0, 3]),
                    T=T, d=rng.choice([32, 64, 64, 72, 80, 128, 128]),
                    page=rng.choice([8, 16, 24, 64, 128]), layout=rng.choice(["pthd", "pthd", "phtd"]),
                    lam=round(rng.uniform(0.0, 1.0), 3))
    V = _log_int(rng, 2000, 131072)
    case = dict(kind=kind, dtype=rng.choice(["bf16", "fp32"]), V=V,
                R=_log_int(rng, 1, 100000000 // V), mode=rng.choice(["plain", "masked"]))
    if kind == "score":
        case["top"] = rng.choice([0, 1, 5, 20, 32])
    return case


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------
def _dt(case):
    return torch.float32 if case["dtype"] == "fp32" else torch.bfloat16


def _gen(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    return gen


def _frequencies(d_rot):
    """Radians per position of every pair, the slow ones interpolated for a longer context."""
    f = 1.0e4 ** (-torch.arange(0, d_rot, 2, dtype=torch.float64, device="cuda") / d_rot)
    return torch.where(f < 2 * math.pi / 1024, f / 4, f)


def _prepare_rotate(case, gen):
    N, H, d = case["N"], case["H"], case["d"]
    Hk, dev = H // case["G"], "cuda"
    rand = lambda *shape: torch.randn(shape, generator=gen, device=dev)  # noqa: E731
    # heads whose projections have grown to different sizes
    size = torch.exp(rand(H + Hk) * 0.5)[:, None]
    s = {"p1": (rand(N, H, d) * size[:H]).to(_dt(case)), "p2": (rand(N, Hk, d) * size[H:]).to(_dt(case)),
         "w1": 1 + 0.2 * rand(d), "w2": 1 + 0.2 * rand(d)}
    # sequences one after the other, each from where it stands
    owner = torch.sort(torch.randint(0, max(1, N // 300 + 1), (N,), generator=gen, device=dev))[0]
    begin = torch.randint(0, max(1, case["reach"] - N), (int(owner.max()) + 1,), generator=gen, device=dev)
    first = torch.searchsorted(owner, owner)
    s["positions"] = (begin[owner] + torch.arange(N, device=dev) - first).to(torch.int32)
    s["freqs"], s["half"], s["scale"] = _frequencies(case["d_rot"]), case["layout"] == "half", 1.1
    if case["kind"] == "rotate_grad":
        s["dq"], s["dk"] = rand(N, H, d).to(_dt(case)), rand(N, Hk, d).to(_dt(case))
    return s


def _pages(case, gen, n, mean=0.0):
    """n pages of a cache [n, page, Hk, d], stored token-major or head-major within a page; every
    channel has a mean of its own."""
    Hk, page, d = case["H"] // case["G"], case["page"], case["d"]
    shape = (n, page, Hk, d) if case["layout"] == "pthd" else (n, Hk, page, d)
    x = torch.randn(shape, generator=gen, device="cuda")
    x = x.add_(torch.randn(d, generator=gen, device="cuda") * mean).to(_dt(case))
    return x if case["layout"] == "pthd" else x.transpose(1, 2)


def _prepare_chunk(case, gen):
    B, C, N, H, T, d, page = (case[k] for k in ("B", "C", "N", "H", "T", "d", "page"))
    dev, i32 = "cuda", torch.int32
    # new tokens of each request, in a large batch one for half of them, as far as the buffer goes
    counts = torch.randint(max(1, C * 3 // 4), C + 1, (B,), generator=gen, device=dev)
    if B >= 16:
        what = torch.rand(B, generator=gen, device=dev)
        counts = torch.where(what < 0.5, torch.ones_like(counts),
                             torch.randint(1, C + 1, (B,), generator=gen, device=dev))
    counts = torch.where(counts.cumsum(0) <= N, counts, torch.zeros_like(counts))
    # rows in the cache, the new ones among them
    lengths = torch.maximum(counts, torch.randint(max(1, T // 2), T + 1, (B,), generator=gen, device=dev))
    if B >= 3:
        lengths[1] = counts[1]  # a prompt's first piece
    ends = counts.cumsum(0)
    t = torch.arange(N, device=dev)
    b = torch.searchsorted(ends, t, right=True).clamp(max=B - 1)
    position = (lengths - counts)[b] + t - (ends - counts)[b]
    position = torch.where(t < ends[-1], position, torch.full_like(t, -1))  # the buffer's padding
    used = (lengths + page - 1) // page
    cols, total = (T + page - 1) // page, int(used.sum())
    perm = torch.randperm(total + 2, generator=gen, device=dev).to(i32)
    col = torch.arange(cols, device=dev)
    first = used.cumsum(0) - used
    table = torch.where(col[None, :] < used[:, None],
                        perm[(first[:, None] + col[None, :]).clamp(max=total + 1)],
                        torch.full((), -1, dtype=i32, device=dev))
    return {"k": _pages(case, gen, total + 2), "v": _pages(case, gen, total + 2, mean=0.5),
            "q": torch.randn((N, H, d), generator=gen, device=dev).to(_dt(case)),
            "table": table.contiguous(), "positions": position.to(i32), "C": C,
            "starts": torch.cat([torch.zeros_like(ends[:1]), ends]).to(i32), "lam": case["lam"]}


def _prepare_score(case, gen):
    R, V = case["R"], case["V"]
    dev = "cuda"
    # a broad body and a few likely tokens, sharper in some rows than in others
    x = torch.randn((R, V), generator=gen, device=dev) * 2.0
    few = torch.randint(0, V, (R, 64), generator=gen, device=dev)
    x.scatter_add_(1, few, 4.0 + 8.0 * torch.rand((R, 64), generator=gen, device=dev))
    x.mul_(0.7 + 0.8 * torch.rand((R, 1), generator=gen, device=dev))
    # given tokens: mostly likely ones, some from anywhere
    pick = torch.randint(0, 64, (R, 1), generator=gen, device=dev)
    target = few.gather(1, pick)[:, 0]
    any_token = torch.randint(0, V, (R,), generator=gen, device=dev)
    target = torch.where(torch.rand(R, generator=gen, device=dev) < 0.2, any_token, target)
    s = {"temperature": None, "top": case.get("top", 0)}
    if case["mode"] == "masked":
        values = torch.tensor([0.7, 1.0, 1.0, 1.3], device=dev)
        s["temperature"] = values[torch.randint(0, 4, (R,), generator=gen, device=dev)]
        # a grammar leaves one token in eight and the given one: -inf in some rows, the type's
        # lowest in others; one row in sixteen has no given token
        mask = torch.rand((R, V), generator=gen, device=dev) > 1 / 8
        mask.scatter_(1, target[:, None], False)
        rows = torch.arange(R, device=dev)
        x.masked_fill_(mask & (rows[:, None] % 4 == 1), -math.inf)
        x.masked_fill_(mask & (rows[:, None] % 4 == 3), torch.finfo(_dt(case)).min)
        target = torch.where(rows % 16 == 5, torch.full_like(target, -1), target)
    s["logits"], s["targets"] = x.to(_dt(case)), target.to(torch.int32)
    if case["kind"] == "score_grad":
        # what the forward left, and advantages that fall on one token each and on the entropy
        e = _plain_score({**s, "top": 0})
        s["logz"], s["entropy"] = e["logz"], e["entropy"]
        s["dlogprob"] = torch.randn(R, generator=gen, device=dev)
        s["dentropy"] = torch.full((R,), 0.01, device=dev) if case["mode"] == "masked" else None
    return s


def prepare(case, seed):
    make = {"rotate": _prepare_rotate, "rotate_grad": _prepare_rotate, "chunk": _prepare_chunk,
            "score": _prepare_score, "score_grad": _prepare_score}[case["kind"]]
    s = make(case, _gen(seed))
    s["kind"] = case["kind"]
    return s


# ---------------------------------------------------------------------------
# One pass in elementary operations
# ---------------------------------------------------------------------------
def _cos_sin(s):
    """Of position * frequency modulo 2 pi: positions reach a million, so the product is in 64 bits."""
    a = torch.remainder(s["positions"].double()[:, None] * s["freqs"], 2 * math.pi).float()[:, None, :]
    return torch.cos(a) * s["scale"], torch.sin(a) * s["scale"]


def _turned(x, cos, sin, half):
    """The first 2 * cos.shape[-1] channels of x turned, the others as they are."""
    c = cos.shape[-1]
    r, rest = x[..., :2 * c], x[..., 2 * c:]
    a, b = (r[..., :c], r[..., c:]) if half else (r[..., 0::2], r[..., 1::2])
    a, b = a * cos - b * sin, a * sin + b * cos
    r = torch.cat((a, b), -1) if half else torch.stack((a, b), -1).reshape(r.shape)
    return torch.cat((r, rest), -1)


def _plain_rotate(s):
    cos, sin = _cos_sin(s)
    out = {}
    for name, x, w in (("q", s["p1"], s["w1"]), ("k", s["p2"], s["w2"])):
        x = x.float()
        n = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * w
        out[name] = _turned(n, cos, sin, s["half"]).to(s["p1"].dtype)
    return out


def _plain_rotate_grad(s):
    cos, sin = _cos_sin(s)
    out = {}
    for i, dy, x, w in ((1, s["dq"], s["p1"], s["w1"]), (2, s["dk"], s["p2"], s["w2"])):
        x = x.float()
        r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
        xhat = x * r
        dn = _turned(dy.float(), cos, -sin, s["half"])
        out[f"dw{i}"] = (dn * xhat).sum((0, 1), dtype=torch.float64).float()
        dn = dn * w
        out[f"dp{i}"] = (r * (dn - xhat * (dn * xhat).mean(-1, keepdim=True))).to(s["p1"].dtype)
    return out


def _plain_chunk(s):
    page, C = s["k"].shape[1], s["C"]
    N, H, d = s["q"].shape
    B, Hk = s["table"].shape[0], s["k"].shape[2]
    dev = s["q"].device
    # the requests' rows of the pages, [B, Hk, 1, T, d]
    T = s["table"].shape[1] * page
    t = torch.arange(T, device=dev)
    entry = s["table"].long().clamp(min=0)[:, t // page]
    k, v = (s[n][entry, t % page].float().permute(0, 2, 1, 3) for n in ("k", "v"))
    # their new tokens' queries, [B, Hk, G C, d], a request's places beyond its tokens idle
    starts = s["starts"].long()
    at = starts[:-1, None] + torch.arange(C, device=dev)
    live = at < starts[1:, None]
    at = at.clamp(max=N - 1)
    p = torch.where(live, s["positions"].long()[at], torch.full_like(at, -1))
    G = H // Hk
    q = s["q"].float()[at].view(B, C, Hk, G, d).permute(0, 2, 3, 1, 4).reshape(B, Hk, G * C, d)
    p = p[:, None, None, :].expand(B, Hk, G, C).reshape(B, Hk, G * C, 1)
    U = torch.matmul(q, k.transpose(2, 3)) * (1.0 / math.sqrt(d))
    S = torch.sigmoid(U.gather(3, p.clamp(min=0)) / TAU_S)
    E = U / (1.0 + torch.exp(-U))
    del U
    E.masked_fill_(t >= p, -math.inf)
    m = E.amax(3, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    P = E.sub_(m).exp_()
    l = P.sum(3, keepdim=True)
    z = torch.matmul(P, v)
    A = m + torch.log(l) - s["lam"] * torch.log((p + 1).clamp(min=1).float())
    g = torch.sigmoid(A - S)
    own_v = v.gather(2, p.clamp(min=0).expand(B, Hk, G * C, d))
    y = own_v + g * (torch.where(l > 0, z / l, own_v) - own_v)
    logz = torch.logaddexp(S, A)
    # back to the tokens' order; the buffer's padding is zero, its logz -inf
    y = y.view(B, Hk, G, C, d).permute(0, 3, 1, 2, 4).reshape(B * C, H, d)
    logz = logz.view(B, Hk, G, C).permute(0, 3, 1, 2).reshape(B * C, H)
    to = torch.where(live, at, torch.full_like(at, N)).reshape(-1)
    Y = torch.zeros((N + 1, H, d), device=dev).index_copy_(0, to, y)[:N]
    Z = torch.full((N + 1, H), -math.inf, device=dev).index_copy_(0, to, logz)[:N]
    none = (torch.arange(N, device=dev) >= starts[-1])[:, None]
    return {"y": torch.where(none[:, :, None], torch.zeros_like(Y), Y).to(s["q"].dtype),
            "logz": torch.where(none, torch.full_like(Z, -math.inf), Z)}


def _plain_score(s):
    x, target = s["logits"].float(), s["targets"].long()
    scale = torch.ones_like(x[:, :1]) if s["temperature"] is None else (1.0 / s["temperature"])[:, None]
    top = x.amax(1, keepdim=True)
    t = (x - top) * scale
    w = torch.exp(t)
    l = w.sum(1)
    mean = torch.where(w > 0, w * t, torch.zeros_like(w)).sum(1) / l
    logl = torch.log(l)
    chosen = t.gather(1, target.clamp(min=0)[:, None])[:, 0] - logl
    out = {"logprob": torch.where(target >= 0, chosen, torch.zeros_like(chosen)),
           "entropy": logl - mean, "logz": top[:, 0] * scale[:, 0] + logl}
    if s["top"]:
        # (in the order of the logits themselves: the lowest index of equal ones first)
        values, order = torch.sort(x, dim=1, descending=True, stable=True)
        values, order = values[:, :s["top"]], order[:, :s["top"]]
        out["top_tokens"] = torch.where(values == -math.inf, torch.full_like(order, -1), order).int()
        out["top_logprobs"] = (values - top) * scale - logl[:, None]
    return out


def _plain_score_grad(s):
    x, target = s["logits"].float(), s["targets"].long()
    scale = torch.ones_like(x[:, :1]) if s["temperature"] is None else (1.0 / s["temperature"])[:, None]
    logp = x * scale - s["logz"][:, None]
    p = torch.exp(logp)
    given = torch.where(target >= 0, s["dlogprob"], torch.zeros_like(s["dlogprob"]))[:, None]
    dx = -given * p
    if s["dentropy"] is not None:
        dx -= s["dentropy"][:, None] * torch.where(p > 0, p * (logp + s["entropy"][:, None]),
                                                  torch.zeros_like(p))
    dx.scatter_add_(1, target.clamp(min=0)[:, None], given)
    return {"dlogits": (dx * scale).to(s["logits"].dtype)}


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------
def run(s):
    kind = s["kind"]
    if not own:
        return {"rotate": _plain_rotate, "rotate_grad": _plain_rotate_grad, "chunk": _plain_chunk,
                "score": _plain_score, "score_grad": _plain_score_grad}[kind](s)
    from paper_2608_20172_gb300 import binding
    if kind in ("rotate", "rotate_grad"):
        rotary = binding.Rotary(s["freqs"], "half" if s["half"] else "interleaved", s["scale"])
        if kind == "rotate":
            q, k = binding.norm_rope(s["p1"], s["p2"], rotary, s["positions"], s["w1"], s["w2"],
                                     eps=EPS)
            return {"q": q, "k": k}
        dp1, dp2, dw1, dw2 = binding.norm_rope_grad(s["dq"], s["dk"], s["p1"], s["p2"], rotary,
                                                    s["positions"], s["w1"], s["w2"], eps=EPS)
        return {"dw1": dw1, "dp1": dp1, "dw2": dw2, "dp2": dp2}
    if kind == "chunk":
        y, logz = binding.paged_chunk(s["q"], s["k"], s["v"], s["table"], s["starts"],
                                      s["positions"], s["lam"], TAU_S)
        return {"y": y, "logz": logz}
    if kind == "score":
        r = binding.logprobs(s["logits"], s["targets"], temperature=s["temperature"], top=s["top"])
        out = {"logprob": r.logprob, "entropy": r.entropy, "logz": r.logz}
        if s["top"]:
            out["top_tokens"], out["top_logprobs"] = r.top_tokens, r.top_logprobs
        return out
    return {"dlogits": binding.logprobs_grad(s["logits"], s["targets"], s["logz"], s["entropy"],
                                             s["dlogprob"], s["dentropy"],
                                             temperature=s["temperature"])}


# ---------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    kind = case["kind"]
    e = 4 if case["dtype"] == "fp32" else 2
    if kind in ("rotate", "rotate_grad"):
        n = case["N"] * (case["H"] + case["H"] // case["G"]) * case["d"]
        if kind == "rotate":
            return {"bytes": 2 * n * e + 4 * case["N"], "flops": 7 * n}
        return {"bytes": 3 * n * e + 4 * case["N"], "flops": 13 * n}
    if kind == "chunk":
        B, C, H, d, T = (case[k] for k in ("B", "C", "H", "d", "T"))
        # mean new tokens of a request and rows of its history
        tokens = (C + 3) / 4 if B >= 16 else C * 7 / 8
        rows = max(T * 3 / 4, C / 2)
        total = min(B * tokens, case["N"])
        seen = rows - min(tokens, rows) / 2
        return {"bytes": int(2 * B * rows * (H // case["G"]) * d * e + 2 * total * H * d * e
                             + 4 * total * H), "flops": int(4 * total * seen * H * d)}
    n = case["R"] * case["V"]
    if kind == "score":
        return {"bytes": n * e + case["R"] * (16 + 8 * case["top"]), "flops": 5 * n}
    return {"bytes": 2 * n * e + 24 * case["R"], "flops": 7 * n}


# ---------------------------------------------------------------------------
# The same in 64 bits
# ---------------------------------------------------------------------------
def _rotated(x, w, s):
    """The definition for one head's rows in 64 bits, with complex numbers."""
    c = s["freqs"].numel()
    n = x / torch.sqrt((x * x).sum(-1, keepdim=True) / x.shape[-1] + EPS) * w
    turn = torch.polar(torch.full((), s["scale"], dtype=torch.float64, device=x.device),
                       s["positions"].double()[:, None] * s["freqs"])[:, None]
    if s["half"]:
        r = torch.complex(n[..., :c].contiguous(), n[..., c:2 * c].contiguous()) * turn
        return torch.cat((r.real, r.imag, n[..., 2 * c:]), -1)
    r = torch.complex(n[..., 0:2 * c:2].contiguous(), n[..., 1:2 * c:2].contiguous()) * turn
    return torch.cat((torch.view_as_real(r).flatten(-2), n[..., 2 * c:]), -1)


def _exact_rotate(s):
    return {"q": _rotated(s["p1"].double(), s["w1"].double(), s),
            "k": _rotated(s["p2"].double(), s["w2"].double(), s)}


def _exact_rotate_grad(s):
    """By reverse mode through the definition."""
    out = {}
    with torch.enable_grad():
        for i, dy in ((1, s["dq"]), (2, s["dk"])):
            x = s[f"p{i}"].double().requires_grad_()
            w = s[f"w{i}"].double().requires_grad_()
            dx, dw = torch.autograd.grad(_rotated(x, w, s), (x, w), dy.double())
            out[f"dw{i}"], out[f"dp{i}"] = dw.detach(), dx.detach()
    return out


def _exact_chunk(s):
    """Request by request and some rows at a time, the rows of R and F written out as defined."""
    N, H, d = s["q"].shape
    page, Hk, f8 = s["k"].shape[1], s["k"].shape[2], torch.float64
    y = torch.zeros((N, H, d), dtype=f8, device="cuda")
    logz = torch.full((N, H), -math.inf, dtype=f8, device="cuda")
    starts, positions = s["starts"].tolist(), s["positions"].long()
    for b in range(len(starts) - 1):
        if starts[b] == starts[b + 1]:
            continue
        n = int(positions[starts[b + 1] - 1]) + 1
        pages = s["table"][b, :-(-n // page)].long()
        K, V = (x[pages].reshape(-1, Hk, d)[:n].to(f8).permute(1, 0, 2) for x in (s["k"], s["v"]))
        j = torch.arange(n, device="cuda")
        for first in range(starts[b], starts[b + 1], 256):
            rows = slice(first, min(first + 256, starts[b + 1]))
            p = positions[rows]
            q = s["q"][rows].to(f8).reshape(-1, Hk, H // Hk, d)
            U = torch.einsum("thgd,hjd->thgj", q, K) / math.sqrt(d)
            R = U * torch.sigmoid(U) - s["lam"] * torch.log((p + 1).to(f8))[:, None, None, None]
            p = p[:, None, None, None]
            R = torch.where(j == p, torch.sigmoid(U / TAU_S), R)
            R = torch.where(j > p, torch.full((), -math.inf, dtype=f8, device="cuda"), R)
            lz = torch.logsumexp(R, 3)
            F = torch.exp(R - lz[..., None])
            y[rows] = torch.einsum("thgj,hjd->thgd", F, V).reshape(-1, H, d)
            logz[rows] = lz.reshape(-1, H)
    return {"y": y, "logz": logz}


def _log_softmax(s, x):
    t = torch.ones(x.shape[0], dtype=x.dtype, device=x.device) if s["temperature"] is None else \
        s["temperature"].double()
    x = x / t[:, None]
    logz = torch.logsumexp(x, 1)
    return x - logz[:, None], logz


def _entropy(logp):
    """-sum p log p, a token of no probability adding nothing."""
    finite = torch.where(logp < -1e4, torch.zeros_like(logp), logp)
    return -(torch.exp(logp) * finite).sum(1)


def _exact_score(s):
    logp, logz = _log_softmax(s, s["logits"].double())
    target = s["targets"].long()
    chosen = logp.gather(1, target.clamp(min=0)[:, None])[:, 0]
    out = {"logprob": torch.where(target >= 0, chosen, torch.zeros_like(chosen)),
           "entropy": _entropy(logp), "logz": logz}
    if s["top"]:
        # largest value first, then the lowest index: two stable passes over the rows
        by_value = torch.argsort(-s["logits"].double(), dim=1, stable=True)[:, :s["top"]]
        out["top_logprobs"] = logp.gather(1, by_value)
        out["top_tokens"] = torch.where(out["top_logprobs"] == -math.inf, torch.full_like(by_value, -1),
                                        by_value).int()
        out = {k: out[k] for k in ("logprob", "entropy", "logz", "top_tokens", "top_logprobs")}
    return out


def _exact_score_grad(s):
    """By reverse mode through the definition, some rows at a time."""
    out = []
    for rows in torch.arange(s["logits"].shape[0], device="cuda").split(512):
        part = {"temperature": None if s["temperature"] is None else s["temperature"][rows]}
        with torch.enable_grad():
            x = s["logits"][rows].double().requires_grad_()
            # (the lowest value of the type stands for no probability: its gradient is 0)
            logp, _ = _log_softmax(part, x.clamp(min=-1e30))
            target = s["targets"][rows].long()
            chosen = logp.gather(1, target.clamp(min=0)[:, None])[:, 0]
            loss = (torch.where(target >= 0, s["dlogprob"][rows].double(), 0.0) * chosen).sum()
            if s["dentropy"] is not None:
                loss = loss + (s["dentropy"][rows].double() * _entropy(logp)).sum()
            out.append(torch.autograd.grad(loss, x)[0].detach())
    return {"dlogits": torch.cat(out)}


def exact(case, seed):
    s = prepare(case, seed)
    return {"rotate": _exact_rotate, "rotate_grad": _exact_rotate_grad, "chunk": _exact_chunk,
            "score": _exact_score, "score_grad": _exact_score_grad}[case["kind"]](s)
