"""Rotary positions in 64 bits (angles in the host's 64-bit-mantissa long double), with the
bounds that the library's results have to keep.

What the kernels round: a cosine or sine is off by 1.6 2^-24, its product with `mul` by 2^-24 of
it; a result is two products and a sum, one of the products rounded apart: in all less than
2^-21 mul (|x1| + |x2|). Then U = half a step of the output's type."""
import math

import numpy as np
import torch

F = 2.0 ** -21
TAU = 2 * np.arctan2(np.longdouble(0), np.longdouble(-1))


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def freqs(dim, base=10000.0, scaling=None, factor=1.0, low=1.0, high=32.0, context=4096.0):
    L = np.longdouble
    i = np.arange(dim // 2).astype(L)
    b = L(base)
    if scaling == "base" and dim > 2:
        b = b * L(factor) ** (L(dim) / L(dim - 2))
    f = b ** (-2 * i / dim)
    slow = f / L(factor)
    if scaling == "linear":
        return slow
    if scaling == "turns":
        w = np.clip((context * f / TAU - low) / (L(high) - low), 0, 1)
        return f * w + slow * (1 - w)
    if scaling == "pairs":
        at = lambda n: dim * np.log(context / (TAU * L(n))) / (2 * np.log(L(base)))
        a, e = max(L(0), np.floor(at(high))), min(L(dim - 1), np.ceil(at(low)))
        w = np.clip((i - a) / max(e - a, L("0.001")), 0, 1)
        return f * (1 - w) + slow * w
    return f


def cos_sin(pos, f):
    """float64 [..., pairs] of integer positions (any size) and long double frequencies."""
    a = np.asarray(pos, dtype=np.longdouble)[..., None] * f
    a = a - TAU * np.round(a / TAU)
    return (torch.from_numpy(np.cos(a).astype(np.float64)),
            torch.from_numpy(np.sin(a).astype(np.float64)))


def columns(dim, order):
    i = torch.arange(dim // 2)
    return (i, i + dim // 2) if order == "halves" else (2 * i, 2 * i + 1)


def rotate(x, pos, f, dim, order, mul=1.0, back=False):
    """x [batch][heads][rows][D] on the CPU, pos [batch][rows]: (result, bound before the
    output's rounding), float64."""
    x = x.double()
    c, s = (t[:, None] * mul for t in cos_sin(pos, f))
    if back:
        s = -s
    one, two = columns(dim, order)
    y, bound = x.clone(), torch.zeros_like(x)
    u, v = x[..., one], x[..., two]
    y[..., one], y[..., two] = u * c - v * s, v * c + u * s
    bound[..., one] = bound[..., two] = F * abs(mul) * (u.abs() + v.abs())
    return y, bound


def check(name, got, want, bound):
    got = got.cpu()
    u = half_step(got.dtype)
    off = (got.double() - want).abs() - bound * (1 + u) - u * want.abs() - 1e-38
    assert torch.isfinite(got).all(), name
    assert off.numel() == 0 or float(off.max()) <= 0, (name, float(off.max()))
