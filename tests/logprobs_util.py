"""Plain 64-bit log probabilities, entropies, top alternatives and the logits' gradient (numpy), for tests."""
import math

import numpy as np

U = 2.0 ** -24  # half a step of fp32


def row(x, target, T=1.0, top=0):
    """(logprob, entropy, logz, top tokens, top log probabilities) of one row in fp64."""
    none = [-1] * top, [-math.inf] * top
    if np.isnan(x).any() or not (T > 0 and math.isfinite(T)):
        return math.nan, math.nan, math.nan, none[0], [math.nan] * top
    m = x.max()
    if m == -math.inf:
        return (0.0 if target < 0 else -math.inf), 0.0, -math.inf, *none
    if m == math.inf:
        n = int((x == m).sum())
        logp, logz, h = np.where(x == m, -math.log(n), -math.inf), math.inf, math.log(n)
    else:
        t = (x - m) / T
        logl = math.log(np.exp(t).sum())
        logp, logz = t - logl, m / T + logl
        p = np.exp(logp)
        h = -(p[p > 0] * logp[p > 0]).sum()
    order = np.argsort(-x, kind="stable")[:top]
    order = [int(i) for i in order if x[i] > -math.inf]
    short = top - len(order)
    return ((0.0 if target < 0 else math.nan if target >= len(x) else logp[target]), h, logz,
            order + [-1] * short, [logp[i] for i in order] + [-math.inf] * short)


def bounds(x, T):
    """Bounds of the fp32 errors of (a row's log l, a term's log p of t).  A weight's exponent is a difference
    and two products (3 u |t|) and 2^x 2 ulp (4 u); a thread adds up at most V / 128 weights and 16 more
    additions join the threads; log adds an ulp.  The entropy's mean of t carries as much of itself and of t."""
    m = x[np.isfinite(x)].max() if np.isfinite(x).any() else 0.0
    t = np.where(np.isfinite(x), (x - m) / T, 0.0)
    w = np.where(np.isfinite(x), np.exp(t), 0.0)
    mean = (w * np.abs(t)).sum() / max(w.sum(), 1e-300)
    logl = math.log(max(w.sum(), 1e-300))
    l_err = U * (3 * mean + 24 + len(x) / 128) + 2 * U * abs(logl)
    mean2 = (w * t * t).sum() / max(w.sum(), 1e-300)
    h_err = l_err * (1 + mean) + U * (3 * mean2 + (24 + len(x) / 128) * mean)
    return l_err, h_err, abs(m / T)


def grad_row(x, target, T, g, h, k):
    """(gradient, bound of its fp32 error before the last rounding) of g logprob + h entropy + k logz."""
    if target < 0:
        g = 0.0
    _, H, logz, *_ = row(x, target, T)
    V = len(x)
    if math.isnan(logz) or target >= V:
        return np.full(V, math.nan), np.zeros(V)
    if logz == -math.inf:
        return np.zeros(V), np.zeros(V)
    far = abs(logz) > 1e30  # +inf, or nothing but the type's lowest: equal ones share the probability
    if far:
        p = np.where(x == x.max(), math.exp(-H), 0.0)
        logp = np.where(p > 0, -H, 0.0)
    else:
        logp = x / T - logz
        p = np.exp(logp)
        logp = np.where(p > 0, logp, 0.0)
    d = p * (k - g - h * (logp + H))
    # log p is off by roundings of x / T, of logz and of itself, p by as much of itself and 4 u more
    size = 0.0 if far else 2 * np.where(p > 0, np.abs(np.where(np.isfinite(x), x, 0) / T), 0) + 3 * abs(logz)
    lp_err = U * (size + 2 * np.abs(logp) + 2 * H)
    err = p * ((lp_err + 8 * U) * (abs(k) + abs(g) + abs(h) * (np.abs(logp) + H)) + abs(h) * lp_err)
    if target >= 0:
        d[target] += g
        err[target] += 2 * U * abs(g)
    return d / T, (err + 2 * U * np.abs(d)) / T
