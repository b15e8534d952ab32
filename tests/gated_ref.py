"""The gated feed-forward block and its gradients in 64 bits, with the bounds that the
library's results have to keep.

U is half a step of bf16 (2^-8 of the value) for what is rounded to bf16, 2^-24 for
fp32 inputs. A sum of n fp32 products is off by at most (n + 8) 2^-24 of the sum of their
sizes, in any order. The gate in fp32 (a base-2 exponential of an argument below 2^6, one
reciprocal, a few products) is off by at most A = 2^-16 of |act| and of 1 for its
derivative; the activations' slopes stay below 1.2. So
  G, U    s = (K + 8) 2^-24 |X||W|
  H       1.2 s_G |U| + |act| s_U + A |act||U|
  dG, dU  U |dG| + A |dH||U|,  U |dU| + A |dH||act|      (e_G, e_U)
  dX      e_G |Wg|^T + e_U |Wu|^T + (2 N + 8) 2^-24 (|dG||Wg|^T + |dU||Wu|^T)
  dW      |X|^T e + (M + 8) 2^-24 |X|^T |dG|
and U of the value itself where an output is bf16, 2^-24 where it is fp32.
"""
import math

import torch

U_BF, U_F32, A = 2.0 ** -8, 2.0 ** -24, 2.0 ** -16
E = 2.0 ** -24


def act(x, kind):
    """(act(x), act'(x)) in 64 bits."""
    if kind == "relu":
        return torch.clamp(x, min=0.0), (x > 0).double()
    if kind == "silu":
        z = 1 / (1 + torch.exp(-x))
        return x * z, z * (1 + x * (1 - z))
    c = math.sqrt(2 / math.pi)
    t = torch.tanh(c * (x + 0.044715 * x ** 3))
    return 0.5 * x * (1 + t), 0.5 * (1 + t) + 0.5 * x * (1 - t * t) * c * (1 + 3 * 0.044715 * x * x)


def mm(a, b):
    return torch.mm(a.contiguous(), b.contiguous())


def forward(X, Wg, Wu, kind):
    """{name: (value, bound)} of H, G and U."""
    X, Wg, Wu = X.double(), Wg.double(), Wu.double()
    k = X.shape[1]
    G, U = mm(X, Wg), mm(X, Wu)
    sG, sU = ((k + 8) * E * mm(X.abs(), W.abs()) for W in (Wg, Wu))
    a = act(G, kind)[0]
    return {"H": (a * U, 1.2 * sG * U.abs() + a.abs() * sU + A * (a * U).abs()), "G": (G, sG),
            "U": (U, sU)}


def backward(dH, X, Wg, Wu, G, U, kind):
    """{name: (value, bound)} of dX, dWg and dWu from the given G and U."""
    u = U_BF if X.dtype == torch.bfloat16 else U_F32
    dH, X, Wg, Wu, G, U = (t.double() for t in (dH, X, Wg, Wu, G, U))
    m, n = G.shape
    a, d = act(G, kind)
    dG, dU = dH * U * d, dH * a
    eG = u * dG.abs() + A * (dH * U).abs()
    eU = u * dU.abs() + A * (dH * a).abs()
    # the products read the rounded dG and dU, up to u larger
    eX = mm(eG, Wg.abs().t()) + mm(eU, Wu.abs().t()) + (2 * n + 8) * E * (1 + u) * (
        mm(dG.abs(), Wg.abs().t()) + mm(dU.abs(), Wu.abs().t()))
    Xt = X.t()
    eW = [mm(Xt.abs(), e) + (m + 8) * E * (1 + u) * mm(Xt.abs(), v.abs()) for e, v in
          ((eG, dG), (eU, dU))]
    return {"dX": (mm(dG, Wg.t()) + mm(dU, Wu.t()), eX), "dWg": (mm(Xt, dG), eW[0]),
            "dWu": (mm(Xt, dU), eW[1])}


def check(name, got, want, bound):
    out = U_BF if got.dtype == torch.bfloat16 else U_F32
    assert got.shape == want.shape and torch.isfinite(got).all(), name
    room = bound * (1 + out) + out * torch.clamp(want.abs(), min=2.0 ** -126) + 1e-30
    off = (got.double() - want).abs()
    assert bool((off <= room).all()), (name, float((off / room).max()), float(off.max()))
