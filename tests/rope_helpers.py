"""Inputs and tolerances of the tests of rotary positions."""
import numpy as np

from oracle import rope as OR
from paper_2608_29058_amd import _rs

PLAIN = dict(scaling=OR.PLAIN)


class Rot:
    """A rotation as the oracle and as the library has it."""

    def __init__(self, dim, inter=False, mscale=1.0, **kw):
        self.per = OR.turns(dim, **kw)
        self.dim, self.inter, self.mscale = dim, inter, mscale
        self.rope = _rs.Rope(dim, layout=_rs.RS_ROPE_INTERLEAVED if inter else _rs.RS_ROPE_HALF, mscale=mscale, **kw)

    def oracle(self, x, pos, transpose=False):
        return OR.rotate(x, pos, self.per, self.inter, self.mscale, transpose)


def half_step(dtype):
    return 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24


def check(got, want, ab, dtype, rot, pos):
    """got against the oracle's rows.  In u = 2^-24 of |x_1| + |x_2| times mscale: the angle of a quarter turn at most is off
    by 2 u (its rounding to fp32, the factor pi / 2 and the product, of 0.79), the series by 1.2 u, mscale and the product
    with it by 2 u, two products and a sum by 2 u: 8 u.  The fp64 angle, in whole, by 2^-50 of itself (the frequency's
    rounding here and there, two products).  Then half a step of the type."""
    got = np.asarray(got, np.float64)
    far = np.abs(np.asarray(pos, np.float64)).max(initial=0.0) * 2 * np.pi * rot.per.max() * 2.0 ** -50
    tol = half_step(dtype) * np.abs(want) * (1 + 2.0 ** -8) + (2.0 ** -21 + far) * ab * 1.01
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (np.argwhere(bad)[:4], got[bad][:4], want[bad][:4], tol[bad][:4])


def bits(t):
    import torch
    return t.contiguous().view(torch.int16 if t.dtype is torch.bfloat16 else torch.int32)


def rows(seed, n, heads, d, dtype, layout="token", device="cuda"):
    """[n, heads, d] on the device, and its values."""
    import torch
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(n, heads, d, generator=g).to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    t = x.to(device)
    if layout == "head":
        t = t.transpose(0, 1).contiguous().transpose(0, 1)
    elif layout == "wide":  # rows inside a fused projection
        w = torch.full((n, heads + 3, d), 9.0, dtype=t.dtype, device=device)
        w[:, 2:2 + heads] = t
        t = w[:, 2:2 + heads]
    return t, x.double().numpy()
