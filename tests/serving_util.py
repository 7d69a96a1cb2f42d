"""Plain 64-bit implementations of the serving operators (numpy, request by request), for tests."""
import math

import numpy as np


def plan(lengths, counts, table, free, state, page, n_tokens):
    """(slots, positions, starts, lengths, state, table, free) after one step."""
    table, ring = table.copy(), free.copy()
    n_pages, cols = len(free), table.shape[1]
    head, avail = (int(x) for x in state)
    if not (0 <= head < n_pages and 0 <= avail <= n_pages):
        head = avail = 0
    slots = np.full(n_tokens, -1, np.int64)
    positions = np.full(n_tokens, -1, np.int32)
    starts, out, wanted, taken, given = [0], [], 0, 0, 0
    for b, (n, c) in enumerate(zip(lengths.tolist(), counts.tolist())):
        first = starts[-1]
        starts.append(min(first + max(c, 0), 2**31 - 1))
        if not 0 <= n <= cols * page:
            out.append(n)
            continue
        held = -(-n // page)
        if c < 0:
            for j in range(held):
                if avail + given < n_pages:
                    ring[(head + avail + given) % n_pages] = table[b, j]
                given += 1
            out.append(0)
            continue
        if n + c > cols * page or first + c > n_tokens:
            out.append(n)
            continue
        need = -(-(n + c) // page) - held
        if need and wanted + need > avail:
            wanted += need
            out.append(n)
            continue
        for j in range(need):
            table[b, held + j] = free[(head + wanted + j) % n_pages]
        wanted += need
        taken = max(taken, wanted) if wanted <= avail else taken
        for j in range(c):
            slots[first + j] = int(table[b, (n + j) // page]) * page + (n + j) % page
            positions[first + j] = n + j
        out.append(n + c)
    count = min(avail + given, n_pages) - taken
    return (slots, positions, np.array(starts, np.int32), np.array(out, np.int32),
            np.array([(head + taken) % n_pages, count], np.int32), table, ring)


def rope(x, positions, base):
    """Interleaved pairs of [N, H, d] turned by position * base^(-2c/d)."""
    d = x.shape[-1]
    a = positions.astype(np.float64)[:, None, None] * base ** (-2.0 * np.arange(d // 2) / d)
    c, s = np.cos(a), np.sin(a)
    out = np.empty_like(x)
    out[..., 0::2] = x[..., 0::2] * c - x[..., 1::2] * s
    out[..., 1::2] = x[..., 0::2] * s + x[..., 1::2] * c
    return out


def givens(x, theta, pairing):
    out = x.copy()
    H = x.shape[1]
    for k, th in enumerate(theta):
        a, b = (2 * k, 2 * k + 1) if pairing == 0 else (2 * k + 1, (2 * k + 2) % H)
        out[:, a] = math.cos(th) * x[:, a] - math.sin(th) * x[:, b]
        out[:, b] = math.sin(th) * x[:, a] + math.cos(th) * x[:, b]
    return out


def decode_row(q, K, V, lam, tau=2.0):
    """Y [H, d] and logZ [H] of the last row for q [H, d] over K, V [n, Hk, d]."""
    H, d = q.shape
    n, Hk = K.shape[:2]
    y, logz = np.empty((H, d)), np.empty(H)
    for h in range(H):
        k, v = K[:, h // (H // Hk)], V[:, h // (H // Hk)]
        u = k @ q[h] / math.sqrt(d)
        r = u / (1 + np.exp(-u)) - lam * math.log(n)
        r[n - 1] = 1 / (1 + math.exp(-u[n - 1] / tau))
        m = r.max()
        logz[h] = m + math.log(np.exp(r - m).sum())
        y[h] = np.exp(r - logz[h]) @ v
    return y, logz


def kept_tokens(x, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """The kept tokens of one row in ascending order and their weights, the largest 1."""
    if temperature == 0:
        temperature, top_k = 1.0, 1
    y = x.astype(np.float64) / temperature
    w = np.exp(y - y.max())
    order = np.argsort(-y, kind="stable")
    n = min(top_k, len(x)) if top_k > 0 else len(x)
    order = order[:n]
    if top_p < 1:
        c = np.cumsum(w[order])
        order = order[:max(1, int(((c - w[order]) < top_p * c[-1]).sum()))]
    order = order[:max(1, int((w[order] >= min(min_p, 1.0)).sum()))]
    kept = np.sort(order)
    return kept, w[kept]
