"""Plain 64-bit Relation rows of new tokens over a request's rows (numpy), and paged caches, for tests."""
import math

import numpy as np
import torch

U = 2.0 ** -24  # half a step of fp32
INF = math.inf


def rows(q, pos, K, V, lam, tau=2.0):
    """Tokens q [n, H, d] at positions pos (negative or past the rows: padding) over K, V [T, Hk, d] in fp64: Y, logZ, and
    of every row what the errors are counted in: sum F |v| [n, H, d], and the largest |u| and sum |q k| /
    sqrt(d)."""
    n, H, d = q.shape
    G = H // K.shape[1]
    Y, Z = np.zeros((n, H, d)), np.full((n, H), -INF)
    W, big = np.zeros((n, H, d)), np.zeros((n, H, 2))
    for t in range(n):
        p = int(pos[t])
        if not 0 <= p < len(K):
            continue
        for h in range(H):
            k, v = K[:p + 1, h // G], V[:p + 1, h // G]
            with np.errstate(all="ignore"):
                u = k @ q[t, h] / math.sqrt(d)
                r = u / (1 + np.exp(-u)) - lam * math.log(p + 1)
                r[p] = 1 / (1 + math.exp(-u[p] / tau)) if not math.isnan(u[p]) else math.nan
                m = r.max()
                Z[t, h] = m + math.log(np.exp(r - m).sum())
                f = np.exp(r - Z[t, h])
                Y[t, h], W[t, h] = f @ v, f @ np.abs(v)
                big[t, h] = np.abs(u).max(), (np.abs(k) @ np.abs(q[t, h])).max() / math.sqrt(d)
    return Y, Z, W, big


def bounds(Y, Z, W, big, d, dtype, lam, top):
    """Bounds of the errors of Y and logZ.  An evidence is off by a rounding a term of its sum of d; SiLU in
    bf16 by 8e-6 u / 2 (the tanh instruction's measured error, at most 7.9e-6, on a factor of u / 2), in fp32 by
    8 u (e^x and a division, 2 ulp each) of itself; the exponent's product and difference and 2^x by 8 u of
    |u| and 1.  Weights are off by as much of themselves, l like them, Y by twice that of sum F |v|, with the
    rounding of Y, and in bf16 of every weight.  logZ: the evidences' error, the logarithms' (2 ulp of values
    up to log of the position), lambda's product and the sums."""
    umax, size = big[..., 0], big[..., 1]
    step = torch.finfo(dtype).eps / 2
    e = (d + 8) * U * size + (8e-6 / 2 if dtype is torch.bfloat16 else 16 * U) * umax + 24 * U * (1 + umax)
    y = 1.01 * step * np.abs(Y) + (2.1 * e[..., None] + (1.01 * step if dtype is torch.bfloat16 else 0)) * W
    finite = np.where(np.isfinite(Z), np.abs(Z), 0)
    return y, e + U * (4 * finite + 8 * (1 + abs(lam)) * math.log(int(top) + 2) + 32)


class Cache:
    """Requests whose rows lie in scattered pages; `layout` "pthd" or "phtd", rows `pad` elements apart."""

    def __init__(self, lengths, Hk, d, dtype, page, *, seed=0, layout="pthd", pad=0, device="cuda:0", mean=0.3,
                 key_scale=1.0):
        rng = np.random.default_rng(seed)
        self.lengths, self.page, self.dtype, self.d = lengths, page, dtype, d
        used = [-(-n // page) for n in lengths]
        n_pages, cols = sum(used) + 2, max(used + [1])
        shape = (n_pages, page, Hk, d + pad) if layout == "pthd" else (n_pages, Hk, page, d + pad)
        self.store = []
        for scale, mu in ((key_scale, 0.0), (1.0, mean)):
            x = torch.from_numpy(rng.standard_normal(shape) * scale + mu).to(dtype)
            self.store.append(x if layout == "pthd" else x.transpose(1, 2))
        perm = rng.permutation(n_pages)
        self.table = np.full((len(lengths), cols), -1, np.int32)
        at = 0
        for b, u in enumerate(used):
            self.table[b, :u] = perm[at:at + u]
            at += u
        self.device = device
        self.upload()

    def upload(self):
        """The pages on the device, as they are now, with their strides."""
        put = lambda x: torch.empty_strided(x.size(), x.stride(), dtype=x.dtype, device=self.device).copy_(  # noqa: E731
            x)[..., :self.d]
        self.k, self.v = (put(x) for x in self.store)
        self.block_table = torch.from_numpy(self.table).to(self.device)

    def place(self, b, row):
        return int(self.table[b, row // self.page]), row % self.page

    def request(self, b):
        """K and V [n, Hk, d] of request b in fp64."""
        n = self.lengths[b]
        at = self.table[b, :-(-n // self.page)]
        return [x.double().numpy()[at].reshape(-1, *x.shape[2:])[:n, :, :self.d] for x in self.store]


def tokens(counts, lengths, n):
    """starts and positions of requests whose last `count` rows are the step's tokens, in a buffer of n."""
    starts = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    positions = np.full(n, -1, np.int32)
    for b, (c, m) in enumerate(zip(counts, lengths)):
        positions[starts[b]:starts[b + 1]] = np.arange(m - c, m)[:max(0, n - starts[b])]
    return starts, positions
