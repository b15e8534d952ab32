"""Softmax attention and its gradients in 64 bits, one head of one sequence at a
time, with the bounds that the library's results have to keep.

The bounds follow from what the kernels round. A bf16 operand or output is off by at
most half a step, U = 2^-8 of its value; every other quantity is fp32, where sums of
up to a few thousand terms and an exponential of a score below 2^5 stay within
F = 2^-14 of the sum of their terms' sizes (2^-24 a term and rounding, 2^5 2^-23 for the
exponent's argument). So
  O   = P V         U P|V| (P rounded) + F P|V|
  dV  = P^T dO      U P^T|dO| + F P^T|dO|
  dS  = P (dP - D)  F P (|dO||V|^T + sum|dO||O|) in fp32, then U |dS|
  dQ  = scale dS K  scale (U |dS| + F P (...)) |K|, dK the same with |Q|
and U of the value itself where the output is bf16 (half a step of the smallest normal
number where it is smaller than that).
"""
import math

import torch

U, F = 2.0 ** -8, 2.0 ** -14


def seen(nq, nk, causal, window, device):
    last = torch.arange(nq, device=device)[:, None] + (nk - nq)
    key = torch.arange(nk, device=device)[None, :]
    m = torch.ones((nq, nk), dtype=torch.bool, device=device)
    if causal:
        m &= key <= last
    if window:
        m &= key > last - window
    return m


def _mm(a, b):
    return torch.mm(a.contiguous(), b.contiguous())


def lengths(lens, B, n):
    return [min(max(int(x), 0), n) for x in lens] if lens is not None else [n] * B


def forward(Q, K, V, scale, causal, window, len_q, len_k):
    """(O, bound of O, lse) of the rows in use; others 0, 0, -inf."""
    B, H, sq, D = Q.shape
    g = H // max(K.shape[1], 1)
    dev = dict(dtype=torch.float64, device=Q.device)
    O, bound = torch.zeros((B, H, sq, D), **dev), torch.zeros((B, H, sq, D), **dev)
    lse = torch.full((B, H, sq), -math.inf, **dev)
    for b, (nq, nk) in enumerate(zip(lengths(len_q, B, sq), lengths(len_k, B, K.shape[2]))):
        if nq == 0 or nk == 0:
            continue
        m = seen(nq, nk, causal, window, Q.device)
        for h in range(H):
            q, k, v = (x.double() for x in (Q[b, h, :nq], K[b, h // g, :nk], V[b, h // g, :nk]))
            x = (_mm(q, k.t()) * scale).masked_fill(~m, -math.inf)
            z = torch.logsumexp(x, 1)
            P = torch.exp(x - torch.where(z == -math.inf, 0.0, z)[:, None])
            lse[b, h, :nq], O[b, h, :nq] = z, _mm(P, v)
            bound[b, h, :nq] = (U + F) * _mm(P, v.abs())
    return O, bound, lse


def backward(dO, Q, K, V, O, lse, scale, causal, window, len_q, len_k):
    """((dQ, bound), (dK, bound), (dV, bound)) from the given O and lse."""
    B, H, sq, D = Q.shape
    Hk, sk = K.shape[1:3]
    g = H // max(Hk, 1)
    z = lambda s: torch.zeros(s, dtype=torch.float64, device=Q.device)
    dQ, bQ = z(Q.shape), z(Q.shape)
    dK, bK, dV, bV = z(K.shape), z(K.shape), z(K.shape), z(K.shape)
    for b, (nq, nk) in enumerate(zip(lengths(len_q, B, sq), lengths(len_k, B, sk))):
        if nq == 0 or nk == 0:
            continue
        m = seen(nq, nk, causal, window, Q.device)
        for h in range(H):
            c = h // g
            q, do, o = (x[b, h, :nq].double() for x in (Q, dO, O))
            k, v = K[b, c, :nk].double(), V[b, c, :nk].double()
            l = lse[b, h, :nq].double()
            P = torch.exp(_mm(q, k.t()) * scale - torch.where(l == -math.inf, 0.0, l)[:, None])
            P = P.masked_fill(~m | (l == -math.inf)[:, None], 0.0)
            dS = P * (_mm(do, v.t()) - (do * o).sum(1, keepdim=True))
            e = U * dS.abs() + F * P * (_mm(do.abs(), v.abs().t()) +
                                        (do * o).abs().sum(1, keepdim=True))
            dQ[b, h, :nq], bQ[b, h, :nq] = scale * _mm(dS, k), scale * _mm(e, k.abs())
            dK[b, c, :nk] += scale * _mm(dS.t(), q)
            bK[b, c, :nk] += scale * _mm(e.t(), q.abs())
            dV[b, c, :nk] += _mm(P.t(), do)
            bV[b, c, :nk] += (U + F) * _mm(P.t(), do.abs())
    return (dQ, bQ), (dK, bK), (dV, bV)


def check(name, got, want, bound):
    out = U * torch.clamp(want.abs(), min=2.0 ** -126) if got.dtype == torch.bfloat16 else \
        2.0 ** -24 * want.abs()
    # the output's rounding is of the computed value: (1 + U) covers it
    off = (got.double() - want).abs() - (bound * (1 + U) + out + 1e-30)
    assert torch.isfinite(got).all(), name
    worst = float(off.max()) if off.numel() else -1.0
    assert worst <= 0, (name, worst, float(((got.double() - want).abs() / (bound + out + 1e-30)).max()))
