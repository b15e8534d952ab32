"""Softmax attention of rank r's heads, from torch tensors.

Convenience over the binding (``sbp_attn_core_fwd``, ``sbp_attn_core_bwd``): takes
4-D tensors [batch][heads][rows][head_dim] (any strides with unit column stride,
e.g. parts of a fused QKV activation), allocates the outputs and makes the call.
All computation happens in libsbp.so.

Q, K and V hold every head (``scope`` SBP_GLOBAL: rank r of p takes its share of the
key heads, and the query heads that share them) or rank r's heads (SBP_LOCAL). The
backward call's O, lse and dO may be either.
"""
from __future__ import annotations

import functools
import math

import torch

from . import sbp
from .streams import on_stream, same_device

_EMPTY = torch.empty


def rank_heads(heads: int, kv_heads: int, p: int, r: int):
    """(first query head, query heads, first key head, key heads) of rank r."""
    group = heads // kv_heads if kv_heads else 1
    hk = kv_heads // p + (r < kv_heads % p)
    k0 = r * (kv_heads // p) + min(r, kv_heads % p)
    return k0 * group, hk * group, k0, hk


def _opts(Q, scale, causal, window, len_q, len_k):
    for t in (len_q, len_k):
        if t is not None and t.shape != Q.shape[:1]:
            raise ValueError("one length per sequence")
    if scale is None:
        scale = 1.0 / math.sqrt(Q.shape[-1])
    return sbp.attn_opts(scale, causal, window, len_q, len_k)


def _local(x, full, scope):
    """View of an operand over query heads: LOCAL when it holds the rank's heads only."""
    return sbp.view4(x, scope if x.shape[1] == full else sbp.SBP_LOCAL)


def _rows(lse, full, scope):
    """View of the rows' statistics, [batch][heads][rows] or with one column."""
    if lse.dim() != 3:
        return _local(lse, full, scope)
    sb, sh, ld = lse.stride()
    if lse.shape[2] <= 1:   # as in sbp.view
        ld = max(ld, 1)
    return sbp.sbp_view4_t(lse.data_ptr(), *lse.shape, 1, sb, sh, ld, sbp._dtype_of(lse),
                           scope if lse.shape[1] == full else sbp.SBP_LOCAL)


def _new(like, B, heads, rows, D, dtype):
    """A tensor [batch][heads][rows][head_dim], [batch][rows][heads][head_dim] in memory
    (what a projection reads), and its view."""
    t = like.new_empty((B, rows, heads, D), dtype=dtype)
    ld = max(heads, 1) * D
    return t.transpose(1, 2), sbp.sbp_view4_t(t.data_ptr(), B, heads, rows, D, max(rows, 1) * ld, D,
                                              ld, sbp._dtype_of(t), sbp.SBP_LOCAL)


def core_fwd(Q, K, V, p: int = 1, r: int = 0, *, scale=None, causal: bool = False,
             window: int = 0, len_q=None, len_k=None, lse: bool = True, out=None,
             out_dtype=None, scope=sbp.SBP_GLOBAL, stream=None, ws=None):
    """(O, lse): O [batch][local heads][rows][head_dim] in Q's dtype (or out_dtype, or
    the given tensor `out`) and the rows' log-sum-exp [batch][local heads][rows] in
    fp32, which the backward pass reads (None with lse=False)."""
    if stream is not None and stream != sbp.current_stream():
        return on_stream(stream, functools.partial(
            core_fwd, scale=scale, causal=causal, window=window, len_q=len_q, len_k=len_k, lse=lse,
            out=out, out_dtype=out_dtype, scope=scope, ws=ws), Q, K, V, p, r)
    B, H, sq, D = Q.shape
    same_device(Q, K, V, len_q, len_k, out, ws)
    hq = rank_heads(H, K.shape[1], p, r)[1] if scope == sbp.SBP_GLOBAL else H
    if out is None:
        out, o = _new(Q, B, hq, sq, D, out_dtype or Q.dtype)
    else:
        o = sbp.view4(out, sbp.SBP_LOCAL)
    z = _EMPTY((B, hq, sq), dtype=torch.float32, device=Q.device) if lse else None
    n = max(sq, 1)
    rows = sbp.sbp_view4_t(z.data_ptr(), B, hq, sq, 1, max(hq, 1) * n, n, 1, sbp.SBP_F32,
                           sbp.SBP_LOCAL) if lse else None
    sbp.sbp_attn_core_fwd(sbp.view4(Q, scope), sbp.view4(K, scope), sbp.view4(V, scope),
                          _opts(Q, scale, causal, window, len_q, len_k),
                          o, rows, p, r, None, ws)
    return out, z


def bwd_workspace_bytes(B: int, hq: int, sq: int) -> int:
    """Workspace that the backward call cannot do without."""
    return 8 * ((B * hq * sq + 3) // 4 * 4)


def core_bwd(dO, Q, K, V, O, lse, p: int = 1, r: int = 0, *, scale=None, causal: bool = False,
             window: int = 0, len_q=None, len_k=None, out=None, grad_dtype=None,
             accumulate: bool = False, scope=sbp.SBP_GLOBAL, stream=None, ws=None):
    """(dQ, dK, dV) of rank r's heads, in the inputs' dtype (or grad_dtype), or in the
    three given tensors `out` (accumulate: added to their fp32 contents). lse is
    [batch][heads][rows] as core_fwd returns it."""
    if stream is not None and stream != sbp.current_stream():
        return on_stream(stream, functools.partial(
            core_bwd, scale=scale, causal=causal, window=window, len_q=len_q, len_k=len_k, out=out,
            grad_dtype=grad_dtype, accumulate=accumulate, scope=scope, ws=ws), dO, Q, K, V, O, lse,
            p, r)
    B, H, sq, D = Q.shape
    Hk, sk = K.shape[1:3]
    same_device(dO, Q, K, V, O, lse, len_q, len_k, ws, *(out or ()))
    hq, hk = (H, Hk) if scope != sbp.SBP_GLOBAL else rank_heads(H, Hk, p, r)[1::2]
    if out is None:
        if accumulate:
            raise ValueError("accumulate needs the tensors to add to")
        dt = grad_dtype or Q.dtype
        (dq, vq), (dk, vk), (dv, vv) = (_new(Q, B, hq, sq, D, dt), _new(Q, B, hk, sk, D, dt),
                                        _new(Q, B, hk, sk, D, dt))
        out = dq, dk, dv
    else:
        vq, vk, vv = (sbp.view4(t, sbp.SBP_ACCUMULATE if accumulate else sbp.SBP_LOCAL) for t in out)
    need = bwd_workspace_bytes(B, hq, sq)
    if ws is None and need > sbp.SBP_WORKSPACE_BYTES:
        # more rows than the kept workspace has room for: one of this call's own
        ws = _EMPTY(need, dtype=torch.uint8, device=Q.device)
    sbp.sbp_attn_core_bwd(_local(dO, H, scope), sbp.view4(Q, scope), sbp.view4(K, scope),
                          sbp.view4(V, scope), _local(O, H, scope), _rows(lse, H, scope),
                          _opts(Q, scale, causal, window, len_q, len_k), vq, vk, vv, p, r, None,
                          ws)
    return out
