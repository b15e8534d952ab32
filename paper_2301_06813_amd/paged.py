"""A paged cache of keys and values: appending a step's tokens, with rotary positions applied
on the way, and the attention of the new tokens over it, from torch tensors.

Convenience over the binding (``sbp_paged_append``, ``sbp_paged_attn``). All computation happens
in libsbp.so.

New tokens come padded, [sequences][heads][rows][head_dim] (len_q: the rows in use), or
packed, [1][heads][rows][head_dim] with row_q [sequences + 1]: sequence b has rows
row_q[b] .. row_q[b + 1] - 1. table [sequences][width] names the pages of a sequence's tokens in
order; len_k counts a sequence's tokens, the new ones included, of which the table has to have
room for all (past it append and attend count places differently: sbp_pages_t). All are int32 on
the device and read when the calls run, so that captured graphs see their new contents. Where the
host knows a step's longest sequence, table[:, :its pages] lets attend choose the kernel for that
length (64 single tokens over up to 1000 keys, 64 heads over 8 of 128: 45 us, 51 with room for 32768).

Q, K and V hold every head (``scope`` SBP_GLOBAL) or rank r's heads (SBP_LOCAL), the cache
likewise (``Cache``'s scope).
"""
from __future__ import annotations

import functools
import math

import torch

from . import sbp
from .attention import _EMPTY, _new, rank_heads
from .streams import on_stream, same_device


def _pages(table, len_k, len_q, row_q) -> sbp.sbp_pages_t:
    seqs, width = table.shape
    if table.dtype != torch.int32 or (table.stride(1) != 1 and width > 1):
        raise ValueError("the table is int32 with unit column stride")
    for t, n in ((len_k, seqs), (len_q, seqs), (row_q, seqs + 1)):
        if t is not None and t.shape != (n,):
            raise ValueError("one length per sequence, and one first row more than sequences")
    ld = table.stride(0)
    return sbp.sbp_pages_t(table.data_ptr(), max(ld, width) if seqs <= 1 else ld, seqs, width,
                           sbp._lens(len_k), sbp._lens(len_q), sbp._lens(row_q))


class Cache:
    """Keys and values, [pages][heads][tokens of a page][head_dim] views in bf16 of any strides
    with unit column stride: a page's memory may be [token][head][dim] or [head][token][dim],
    keys and values parts of one tensor. The tensors are the caller's and are kept."""

    def __init__(self, k, v, scope=sbp.SBP_GLOBAL):
        if k.shape != v.shape or k.dim() != 4:
            raise ValueError("keys and values are [pages][heads][tokens][head_dim]")
        self.k, self.v, self.scope = k, v, scope
        self._views = sbp.view4(k, scope), sbp.view4(v, scope)

    def append(self, K, V, table, len_k, p: int = 1, r: int = 0, *, Q=None, rope=None, len_q=None,
               row_q=None, out=None, out_dtype=None, scope=sbp.SBP_GLOBAL, stream=None):
        """Stores the new tokens' K and V at places len_k - n .. len_k - 1 of their sequences,
        K rotated by them with a rotary.Rope. With Q, returns rank r's heads of it, rotated
        (in Q's dtype, or out_dtype, or in the tensor `out`, which may be the rank's part of
        Q); else None. Rows that no sequence uses are left as they are."""
        if stream is not None and stream != sbp.current_stream():
            return on_stream(stream, lambda: (self.append(
                K, V, table, len_k, p, r, Q=Q, rope=rope, len_q=len_q, row_q=row_q, out=out,
                out_dtype=out_dtype, scope=scope),))[0]
        same_device(K, V, Q, table, len_k, len_q, row_q, out, self.k, self.v,
                    None if rope is None else rope.turns)
        qo = None
        if Q is not None:
            B, H, S, D = Q.shape
            if out is None:
                hq = H if p == 1 or scope != sbp.SBP_GLOBAL else rank_heads(H, K.shape[1], p, r)[1]
                out, qo = _new(Q, B, hq, S, D, out_dtype or Q.dtype)
            else:
                qo = sbp.view4(out, sbp.SBP_LOCAL)
        elif out is not None:
            raise ValueError("out without Q")
        sbp.sbp_paged_append(sbp.view4(K, scope), sbp.view4(V, scope),
                             _pages(table, len_k, len_q, row_q),
                             None if rope is None else rope.view, *self._views,
                             None if Q is None else sbp.view4(Q, scope), qo, p, r, None)
        return out

    def attend(self, Q, table, len_k, p: int = 1, r: int = 0, *, scale=None, causal: bool = True,
               window: int = 0, len_q=None, row_q=None, lse: bool = True, out=None, out_dtype=None,
               stream=None, ws=None):
        """(O, lse): attention of the new tokens' rows of Q (of the cache's scope) over their
        sequences' tokens in the cache; O [batch][local heads][rows][head_dim] in Q's dtype (or
        out_dtype, or the given tensor `out`), lse [batch][local heads][rows] in fp32 (None with
        lse=False). Packed rows that no sequence uses are left as they are."""
        if stream is not None and stream != sbp.current_stream():
            return on_stream(stream, functools.partial(
                self.attend, scale=scale, causal=causal, window=window, len_q=len_q, row_q=row_q,
                lse=lse, out=out, out_dtype=out_dtype, ws=ws), Q, table, len_k, p, r)
        B, H, S, D = Q.shape
        same_device(Q, table, len_k, len_q, row_q, out, ws, self.k, self.v)
        if not -(1 << 31) <= window < 1 << 31:
            raise ValueError("a window is an int32")
        hq = H if p == 1 or self.scope != sbp.SBP_GLOBAL else rank_heads(H, self.k.shape[1], p, r)[1]
        if out is None:
            out, o = _new(Q, B, hq, S, D, out_dtype or Q.dtype)
        else:
            o = sbp.view4(out, sbp.SBP_LOCAL)
        z = rows = None
        if lse:
            z = _EMPTY((B, hq, S), dtype=torch.float32, device=Q.device)
            n = max(S, 1)
            rows = sbp.sbp_view4_t(z.data_ptr(), B, hq, S, 1, max(hq, 1) * n, n, 1, sbp.SBP_F32,
                                   sbp.SBP_LOCAL)
        sbp.sbp_paged_attn(sbp.view4(Q, self.scope), *self._views,
                           _pages(table, len_k, len_q, row_q),
                           1.0 / math.sqrt(D) if scale is None else scale, causal, window, o, rows,
                           p, r, None, ws)
        return out, z
