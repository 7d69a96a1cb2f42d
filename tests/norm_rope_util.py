"""Plain 64-bit norm with rotation and its gradient (numpy), for tests."""
import numpy as np

U = 2.0 ** -24  # half a step of fp32


def angles(positions, freqs):
    """positions * freqs modulo 2 pi in extended precision."""
    two_pi = 8 * np.arctan(np.longdouble(1))
    a = positions.astype(np.longdouble)[:, None] * freqs.astype(np.longdouble)
    return np.remainder(a, two_pi).astype(np.float64)


def pairs(d, d_rot, half):
    """The channels a and b of every pair."""
    p = np.arange(d_rot // 2)
    return (p, p + d_rot // 2) if half else (2 * p, 2 * p + 1)


def turn(n, positions, freqs, half, scale, sign=1.0):
    """Rows n [N, H, d] turned by their positions (sign -1: back)."""
    a, b = pairs(n.shape[-1], 2 * len(freqs), half)
    ang = angles(positions, freqs)[:, None, :]
    c, s = scale * np.cos(ang), sign * scale * np.sin(ang)
    out = n.copy()
    out[..., a] = n[..., a] * c - n[..., b] * s
    out[..., b] = n[..., a] * s + n[..., b] * c
    return out


def norm_rope(x, w, positions, freqs, half, scale, norm, eps):
    """(result, bound of the fp32 arithmetic's error).  With u = 2^-24: the mean square's sum has at most
    16 + 5 roundings and a division, halved by the root; rsqrtf is off by 2 ulp (4 u), two products follow:
    18 u of n.  A turn's angle, a part of a turn rounded to fp32, is off by at most pi u, sincospif by 2 ulp,
    the factor and the two products and their sum by one each: 11 u of |a| + |b|."""
    r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps) if norm else np.ones(x.shape[:-1] + (1,))
    n = x * r * w
    y = turn(n, positions, freqs, half, scale)
    size = np.abs(n)
    a, b = pairs(x.shape[-1], 2 * len(freqs), half)
    both = (size[..., a] + size[..., b]) * max(1.0, abs(scale))
    size[..., a], size[..., b] = both, both
    pad = (positions < 0)[:, None, None]
    # (the double frequency's product with a far position)
    far = 2.0 ** -52 * np.abs(positions).max() * (np.abs(freqs).max() if len(freqs) else 0)
    return np.where(pad, 0.0, y), size * (32 * U + far)


def norm_rope_grad(dy, x, w, positions, freqs, half, scale, norm, eps):
    """(dx, dw, bound of dx's error, bound of dw's): u turned back is off by 11 U of its pair, x^ by 18 U,
    the mean of x^ w u by 24 U more of the mean of its terms' sizes, and a few roundings; a column's sum over
    the rows by a rounding an addition (rows / 4 and 16 at most in one chain) beside its terms' errors."""
    pad = (positions < 0)[:, None, None]
    dy = np.where(pad, 0.0, dy)
    r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps) if norm else np.ones(x.shape[:-1] + (1,))
    xh = x * r
    u = turn(dy, positions, freqs, half, scale, -1.0)
    size = np.abs(dy)
    a, b = pairs(x.shape[-1], 2 * len(freqs), half)
    both = (size[..., a] + size[..., b]) * max(1.0, abs(scale))
    size[..., a], size[..., b] = both, both
    dw = (u * xh).sum((0, 1))
    dw_size = (size * np.abs(xh)).sum((0, 1))
    mean = (xh * w * u).mean(-1, keepdims=True) if norm else 0.0
    mean_size = (np.abs(xh * w) * size).mean(-1, keepdims=True) if norm else 0.0
    dx = r * (w * u - xh * mean)
    rows = x.shape[0] * x.shape[1]
    return (np.where(pad, 0.0, dx), dw, 100 * U * r * (np.abs(w) * size + np.abs(xh) * mean_size),
            (48 + rows / 4) * U * dw_size)
