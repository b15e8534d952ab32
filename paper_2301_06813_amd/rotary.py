"""Rotary positions of rank r's query and key heads, from torch tensors.

Convenience over the binding (``sbp_rope_turns``, ``sbp_rope_fwd``, ``sbp_rope_bwd``): takes
4-D tensors [batch][heads][rows][head_dim] (any strides with unit column stride, e.g. parts
of a fused QKV activation), allocates the outputs and makes the call. All computation
happens in libsbp.so.

Q and K hold every head (``scope`` SBP_GLOBAL: rank r of p takes its share of the key heads,
and the query heads that share them) or rank r's heads (SBP_LOCAL).
"""
from __future__ import annotations

import functools

import torch

from . import sbp
from .attention import rank_heads
from .streams import on_stream, same_device


class Rope:
    """A rotation of a head's first `dim` columns: its frequencies base^(-2 i / dim), on the
    device, made once.

    order    which columns make a pair: "halves" (i, i + dim / 2) or "pairs" (2 i, 2 i + 1)
    scaling  for contexts `factor` times the `context` a model was trained on: "linear",
             "base", "turns" (pairs with `high` or more turns over the context keep their
             frequency, those with `low` or fewer are slowed down) or "pairs" (the same by the
             pairs' numbers); see sbp_rope_scaling_t
    mul      factor of the rotated columns
    """

    def __init__(self, dim: int, base: float = 10000.0, order: str = "halves", scaling=None,
                 factor: float = 1.0, low: float = 1.0, high: float = 32.0, context: float = 4096.0,
                 mul: float = 1.0, device=None):
        turns = sbp.sbp_rope_turns(dim, base, sbp.ROPE_SCALINGS[scaling], factor, low, high, context)
        self.dim, self.order, self.mul = dim, order, mul
        wrapped = [t - (1 << 64) if t >> 63 else t for t in turns]   # torch has no uint64 products
        self.turns = torch.tensor(wrapped, dtype=torch.int64,
                                  device="cuda" if device is None else device)
        self.view = sbp.sbp_rope_t(self.turns.data_ptr(), dim, sbp.ROPE_ORDERS[order], mul)


def places(pos, batch: int, rows: int):
    """sbp_places_t of positions [batch] (of the sequences' first rows) or [batch][rows], int32
    on the device (kept alive by the caller); None: row i at i."""
    if pos is None:
        return None
    if pos.dtype != torch.int32:
        raise ValueError("positions are int32")
    if pos.shape == (batch,):
        return sbp.sbp_places_t(pos.data_ptr(), pos.stride(0), 0)
    if pos.shape != (batch, rows) or (rows > 1 and pos.stride(1) != 1):
        raise ValueError("one position per sequence, or per row with unit stride")
    return sbp.sbp_places_t(pos.data_ptr(), pos.stride(0), 1)


def fwd(rope: Rope, Q, K=None, p: int = 1, r: int = 0, *, pos=None, out=None, out_dtype=None,
        scope=sbp.SBP_GLOBAL, stream=None):
    """(Qo, Ko) of rank r's heads: Q and K rotated by their rows' positions (``places``), in
    their dtype (or out_dtype), or in the tensors `out`, which may be the rank's parts of Q and
    K themselves. Without K, Ko is None."""
    return _turn(sbp.sbp_rope_fwd, rope, Q, K, p, r, pos, out, out_dtype, scope, stream)


def bwd(rope: Rope, dQo, dKo=None, p: int = 1, r: int = 0, *, pos=None, out=None, out_dtype=None,
        scope=sbp.SBP_GLOBAL, stream=None):
    """(dQ, dK) from the gradients of fwd's outputs (scope SBP_LOCAL where they hold the
    rank's heads only)."""
    return _turn(sbp.sbp_rope_bwd, rope, dQo, dKo, p, r, pos, out, out_dtype, scope, stream)


def _turn(call, rope, Q, K, p, r, pos, out, out_dtype, scope, stream):
    if stream is not None and stream != sbp.current_stream():
        return on_stream(stream, functools.partial(_turn, call, rope, Q, K, p, r, pos, out, out_dtype,
                                                   scope, None))
    B, H, S, D = Q.shape
    same_device(Q, K, pos, rope.turns, *(out or ()))
    Hk = H if K is None else K.shape[1]
    hq, hk = (H, Hk) if p == 1 or scope != sbp.SBP_GLOBAL else rank_heads(H, Hk, p, r)[1::2]
    q = sbp.view4(Q, scope)
    k = None if K is None else sbp.view4(K, scope)
    if out is None:
        # one block for both, [batch][rows][heads][dim] with K's heads behind Q's
        n = hq if K is None else hq + hk
        t = Q.new_empty((B, S, n, D), dtype=out_dtype) if out_dtype else Q.new_empty((B, S, n, D))
        ld = max(n, 1) * D
        dt, at, sb = sbp._dtype_of(t), t.data_ptr(), max(S, 1) * ld
        strides = sb, D, ld, 1
        qo = sbp.sbp_view4_t(at, B, hq, S, D, sb, D, ld, dt, sbp.SBP_LOCAL)
        if K is None:
            ko, out = None, (t.as_strided((B, hq, S, D), strides), None)
        else:
            ko = sbp.sbp_view4_t(at + hq * D * t.element_size(), B, hk, S, D, sb, D, ld, dt,
                                 sbp.SBP_LOCAL)
            out = (t.as_strided((B, hq, S, D), strides),
                   t.as_strided((B, hk, S, D), strides, hq * D))
    else:
        qo, ko = (None if t is None else sbp.view4(t, sbp.SBP_LOCAL) for t in out)
    call(q, k, rope.view, places(pos, B, S), qo, ko, p, r, None)
    return out
