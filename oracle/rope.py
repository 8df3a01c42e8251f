"""fp64 reference of rotary positions: frequencies of every scaling, rows of pairs turned by their positions."""
import math

import numpy as np

PLAIN, LINEAR, TURNS, PAIRS = range(4)


def turns(dim, base=10000.0, scaling=PLAIN, factor=1.0, context=0.0, low=1.0, high=32.0):
    """Turns per position of the dim / 2 pairs."""
    out = []
    for i in range(dim // 2):
        f = base ** (-2.0 * i / dim)
        if scaling == LINEAR:
            f /= factor
        elif scaling == TURNS:
            n = context * f / (2 * math.pi)  # turns in the context
            w = 0.0 if n <= low else 1.0 if n >= high else (n - low) / (high - low)
            f = f * w + f / factor * (1 - w)
        elif scaling == PAIRS:
            def p(r):
                return dim / 2 * math.log(context / (2 * math.pi * r)) / math.log(base)
            a, b = max(math.floor(p(high)), 0), min(math.ceil(p(low)), dim - 1)
            b = max(b, a + 0.001)
            w = 1.0 if i <= a else 0.0 if i >= b else 1 - (i - a) / (b - a)
            f = f * w + f / factor * (1 - w)
        out.append(f / (2 * math.pi))
    return np.array(out)


def pairs(dim, interleaved):
    i = np.arange(dim // 2)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + dim // 2)


def rotate(x, pos, per, interleaved=False, mscale=1.0, transpose=False):
    """x [n, heads, d] with row r turned by pos[r] * per turns of each pair; and sum of |terms| of every element."""
    x = np.asarray(x, np.float64)
    y, ab = x.copy(), np.zeros_like(x)
    a, b = pairs(2 * len(per), interleaved)
    ang = 2 * math.pi * np.mod(np.asarray(pos, np.float64)[:, None] * per, 1.0)
    c, s = np.cos(ang)[:, None] * mscale, np.sin(ang)[:, None] * (-mscale if transpose else mscale)
    u, v = x[..., a], x[..., b]
    y[..., a], y[..., b] = u * c - v * s, v * c + u * s
    ab[..., a] = ab[..., b] = (np.abs(u) + np.abs(v)) * abs(mscale)
    return y, ab
