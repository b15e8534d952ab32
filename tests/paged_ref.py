"""Appending to a paged cache and attention over it, on the host or in 64 bits on the device, one
sequence at a time. Bounds as in attn_core_ref.py: U a rounding to bf16, F what fp32 sums and
exponentials add."""
import math

import torch

from attn_core_ref import F, U, check  # noqa: F401  (check is for the tests)


def lengths(n, cap_rows, len_q=None, row_q=None):
    """(batch, first row, rows) of each sequence."""
    if row_q is not None:
        out = []
        for b in range(n):
            a = min(max(int(row_q[b]), 0), cap_rows)
            out.append((0, a, max(min(max(int(row_q[b + 1]), a), cap_rows) - a, 0)))
        return out
    return [(b, 0, cap_rows if len_q is None else min(max(int(len_q[b]), 0), cap_rows))
            for b in range(n)]


def places(seqs, len_k, table, pages, P):
    """[(batch, row, page, slot, place)] of the new tokens, page None where none is stored."""
    out = []
    for b, (x, first, n) in enumerate(seqs):
        for i in range(n):
            t = int(len_k[b]) - n + i
            page = None
            if 0 <= t < len(table[b]) * P and 0 <= table[b][t // P] < pages:
                page = table[b][t // P]
            out.append((x, first + i, page, t % P, t))
    return out


def attend(Q, kc, vc, table, len_k, seqs, scale, causal, window):
    """(O, bound, lse, rows that belong to a sequence) in 64 bits."""
    B, H, S, D = Q.shape
    pages, Hk, P, _ = kc.shape
    g = H // max(Hk, 1)
    dev = dict(dtype=torch.float64, device=Q.device)
    O, bound = torch.zeros((B, H, S, D), **dev), torch.zeros((B, H, S, D), **dev)
    lse = torch.full((B, H, S), -math.inf, **dev)
    used = torch.zeros((B, S), dtype=torch.bool, device=Q.device)
    for b, (x, first, n) in enumerate(seqs):
        used[x, first:first + n] = True
        lk = min(max(int(len_k[b]), 0), len(table[b]) * P)
        if n == 0 or lk == 0:
            continue
        ids = torch.tensor(table[b][:(lk + P - 1) // P], device=Q.device).long()
        good = ((ids >= 0) & (ids < pages)).repeat_interleave(P)[:lk]
        i = torch.arange(n, device=Q.device)[:, None] + (lk - n)
        j = torch.arange(lk, device=Q.device)[None, :]
        m = good[None, :].expand(n, lk).clone()
        if causal:
            m &= j <= i
        if window:
            m &= j > i - window
        seen = m.any(0)
        ids = torch.where((ids >= 0) & (ids < pages), ids, torch.zeros_like(ids))
        for h in range(Hk):
            k, v = (c[ids, h].reshape(-1, D)[:lk].double() for c in (kc, vc))
            # what nobody sees is not read
            k, v = (torch.where(seen[:, None], t, torch.zeros_like(t)) for t in (k, v))
            for e in range(h * g, h * g + g):
                q = Q[x, e, first:first + n].double()
                w = (torch.mm(q, k.t().contiguous()) * scale).masked_fill(~m, -math.inf)
                z = torch.logsumexp(w, 1)
                p = torch.exp(w - torch.where(z == -math.inf, 0.0, z)[:, None])
                lse[x, e, first:first + n] = z
                O[x, e, first:first + n] = torch.mm(p, v)
                bound[x, e, first:first + n] = (U + F) * torch.mm(p, v.abs())
    return O, bound, lse, used
