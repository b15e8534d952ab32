"""Rank-r local products of one SBP linear, from torch tensors.

Convenience over the binding: picks the input states of a named signature,
asks the library for the output states (``sbp_signature``) and local output
shape (``sbp_shard_index``), allocates the output and calls the entry point.
All computation happens in libsbp.so.

Signatures are the 1-D factors of AutoDDL's SBP matmul (Sec. 4.2):
DP (S(0),B)->S(0), COL (B,S(1))->S(1), KS (S(1),S(0))->P, and by linearity
PB (P,B)->P, BP (B,P)->P, BB (B,B)->B. On a device mesh an nd signature is
one of them per mesh axis (the 3-D rule of Sec. 4.2 is ("DP", "COL", "KS"));
the ``*_nd`` functions take (factors, mesh, coord).
"""
from __future__ import annotations

import functools

import torch

from . import sbp
from .streams import on_stream, same_device

OPS = ("fwd", "bwd_data", "bwd_weight")


def input_layouts(sig: str, p: int, r: int):
    """States of X and W under signature sig."""
    if sig == "DP":
        return sbp.split(0, p, r), sbp.broadcast(p, r)
    if sig == "COL":
        return sbp.broadcast(p, r), sbp.split(1, p, r)
    if sig == "KS":
        return sbp.split(1, p, r), sbp.split(0, p, r)
    if sig == "PB":
        return sbp.partial(p, r), sbp.broadcast(p, r)
    if sig == "BP":
        return sbp.broadcast(p, r), sbp.partial(p, r)
    if sig == "BB":
        return sbp.broadcast(p, r), sbp.broadcast(p, r)
    raise ValueError("unknown signature %r" % sig)


def layouts(sig: str, p: int, r: int) -> dict:
    x, w = input_layouts(sig, p, r)
    y, dy, dx, dw = sbp.sbp_signature(x, w)
    return {"x": x, "w": w, "y": y, "dy": dy, "dx": dx, "dw": dw}


def layouts_for(lin, wl, r) -> dict:
    """States of one linear of a workload on rank r (for a mesh workload, r
    is the device's mesh coordinate)."""
    if wl.mesh:
        return nd_layouts(lin.factors, wl.mesh, r)
    return layouts(lin.sig, wl.p, r)


# states of X and W on one mesh axis, per factor
FACTOR_STATES = {"DP": ("S0", "B"), "COL": ("B", "S1"), "KS": ("S1", "S0"), "PB": ("P", "B"),
                 "BP": ("B", "P"), "BB": ("B", "B")}


def nd_input_layouts(factors, mesh, coord):
    """nd states of X and W: factor f on mesh axis a puts X and W in the
    states FACTOR_STATES[f] on that axis."""
    xs = [FACTOR_STATES[f][0] for f in factors]
    ws = [FACTOR_STATES[f][1] for f in factors]
    return sbp.nd_layout(xs, mesh, coord), sbp.nd_layout(ws, mesh, coord)


def nd_layouts(factors, mesh, coord) -> dict:
    x, w = nd_input_layouts(factors, mesh, coord)
    y, dy, dx, dw = sbp.sbp_nd_signature(x, w)
    return {"x": x, "w": w, "y": y, "dy": dy, "dx": dx, "dw": dw}


def shard(l, rows: int, cols: int):
    """The library's share of a rows x cols tensor in 1-D or nd state l."""
    if isinstance(l, sbp.sbp_nd_layout_t):
        return sbp.sbp_nd_shard_index(l, rows, cols)
    return sbp.sbp_shard_index(l, rows, cols)


def is_partial(l) -> bool:
    if isinstance(l, sbp.sbp_nd_layout_t):
        return any(l.kind[a] == sbp.SBP_PARTIAL for a in range(l.ndim))
    return l.kind == sbp.SBP_PARTIAL


def out_shape(op: str, L: dict, M: int, K: int, N: int):
    """Local output shape of op for the device's share of global X (MxK), W (KxN)."""
    if op == "fwd":
        return shard(L["x"], M, K).rows, shard(L["w"], K, N).cols
    if op == "bwd_data":
        return shard(L["dy"], M, N).rows, shard(L["w"], K, N).rows
    if op == "bwd_weight":
        return shard(L["x"], M, K).cols, shard(L["dy"], M, N).cols
    raise ValueError(op)


def out_state(op: str, L: dict):
    return L[{"fwd": "y", "bwd_data": "dx", "bwd_weight": "dw"}[op]]


def out_dtype(op: str, L: dict, in_dtype):
    """fp32 for Partial-sum outputs and fp32 inputs, else the input dtype."""
    if is_partial(out_state(op, L)) or in_dtype == torch.float32:
        return torch.float32
    return in_dtype


def alloc_out(op: str, sig: str, p: int, r: int, M: int, K: int, N: int, in_dtype, device):
    return alloc_out_L(op, layouts(sig, p, r), M, K, N, in_dtype, device)


def alloc_out_L(op: str, L: dict, M: int, K: int, N: int, in_dtype, device):
    rows, cols = out_shape(op, L, M, K, N)
    return torch.empty((rows, cols), dtype=out_dtype(op, L, in_dtype), device=device)


def run(op: str, sig: str, p: int, r: int, X, W, dY, out, stream=None):
    """Launch rank r's local product op of signature sig on global X, W, dY
    (torch tensors; a tensor the op does not read may be None) into `out`;
    returns the output state."""
    return run_L(op, layouts(sig, p, r), X, W, dY, out, stream)


def run_L(op: str, L: dict, X, W, dY, out, stream=None, accumulate=False, ws=None):
    """As run, for the states in L (1-D or nd). accumulate: add the product
    to out's fp32 contents (gradient accumulation); ws: the workspace
    argument of the binding (None: its default workspace)."""
    nd = isinstance(L["x"], sbp.sbp_nd_layout_t)
    o = sbp.view(out, sbp.SBP_ACCUMULATE if accumulate else sbp.SBP_LOCAL)
    if op == "fwd":
        fn = sbp.sbp_nd_linear_fwd if nd else sbp.sbp_linear_fwd
        return fn(sbp.view(X), L["x"], sbp.view(W), L["w"], o, stream, ws)
    if op == "bwd_data":
        fn = sbp.sbp_nd_linear_bwd_data if nd else sbp.sbp_linear_bwd_data
        return fn(sbp.view(dY), L["dy"], sbp.view(W), L["w"], o, stream, ws)
    if op == "bwd_weight":
        fn = sbp.sbp_nd_linear_bwd_weight if nd else sbp.sbp_linear_bwd_weight
        return fn(sbp.view(X), L["x"], sbp.view(dY), L["dy"], o, stream, ws)
    raise ValueError(op)


def run_bwd(sig: str, p: int, r: int, X, W, dY, dX, dW, stream=None):
    """Both backward products of rank r in one call (sbp_linear_bwd); returns
    the (dX, dW) states."""
    return run_bwd_L(layouts(sig, p, r), X, W, dY, dX, dW, stream)


def run_bwd_L(L: dict, X, W, dY, dX, dW, stream=None, accumulate_dw=False, ws=None):
    """Both backward products in one call; accumulate_dw adds dW to its fp32
    contents (gradient accumulation over micro-batches)."""
    fn = sbp.sbp_nd_linear_bwd if isinstance(L["x"], sbp.sbp_nd_layout_t) else sbp.sbp_linear_bwd
    return fn(sbp.view(dY), L["dy"], sbp.view(X), L["x"], sbp.view(W), L["w"],
              sbp.view(dX, sbp.SBP_LOCAL),
              sbp.view(dW, sbp.SBP_ACCUMULATE if accumulate_dw else sbp.SBP_LOCAL), stream, ws)


def call_bwd(sig: str, p: int, r: int, X, W, dY, stream=None):
    """Allocate dX and dW and run both backward products; returns (dX, dW, states)."""
    if stream is not None and stream != sbp.current_stream():
        return on_stream(stream, call_bwd, sig, p, r, X, W, dY)
    M, K = X.shape
    N = W.shape[1]
    dX = alloc_out("bwd_data", sig, p, r, M, K, N, X.dtype, X.device)
    dW = alloc_out("bwd_weight", sig, p, r, M, K, N, X.dtype, X.device)
    st = run_bwd(sig, p, r, X, W, dY, dX, dW, stream)
    return dX, dW, st


def call(op: str, sig: str, p: int, r: int, X, W, dY, stream=None):
    """Allocate the output and run; returns (out, state)."""
    if stream is not None and stream != sbp.current_stream():
        return on_stream(stream, call, op, sig, p, r, X, W, dY)
    ref = X if X is not None else dY
    M = (X if X is not None else dY).shape[0]
    K = X.shape[1] if X is not None else W.shape[0]
    N = W.shape[1] if W is not None else dY.shape[1]
    out = alloc_out(op, sig, p, r, M, K, N, ref.dtype, ref.device)
    st = run(op, sig, p, r, X, W, dY, out, stream)
    return out, st


def call_nd(op: str, factors, mesh, coord, X, W, dY, stream=None):
    """nd form of call: the device at mesh coordinate coord under the per-axis
    factors; returns (out, nd state)."""
    if stream is not None and stream != sbp.current_stream():
        return on_stream(stream, call_nd, op, factors, mesh, coord, X, W, dY)
    L = nd_layouts(factors, mesh, coord)
    ref = X if X is not None else dY
    M = ref.shape[0]
    K = X.shape[1] if X is not None else W.shape[0]
    N = W.shape[1] if W is not None else dY.shape[1]
    out = alloc_out_L(op, L, M, K, N, ref.dtype, ref.device)
    st = run_L(op, L, X, W, dY, out, stream)
    return out, st


def call_bwd_nd(factors, mesh, coord, X, W, dY, stream=None):
    """nd form of call_bwd; returns (dX, dW, states)."""
    if stream is not None and stream != sbp.current_stream():
        return on_stream(stream, call_bwd_nd, factors, mesh, coord, X, W, dY)
    L = nd_layouts(factors, mesh, coord)
    M, K = X.shape
    N = W.shape[1]
    dX = alloc_out_L("bwd_data", L, M, K, N, X.dtype, X.device)
    dW = alloc_out_L("bwd_weight", L, M, K, N, X.dtype, X.device)
    st = run_bwd_L(L, X, W, dY, dX, dW, stream)
    return dX, dW, st


# ------------------------------------------------ gated feed-forward block
def gated_fwd_L(L: dict, X, Wg, Wu, act: str = "silu", save: bool = True, stream=None, ws=None):
    """(H, G, U) of the device's shares of global X, Wg and Wu under the states in L
    (``layouts`` or ``nd_layouts``): H = act(X Wg) * (X Wu), and the projections that the
    backward pass reads (None with save=False)."""
    M, K = X.shape
    return _gated_fwd(L, _gated_sizes(L, M, K, Wg.shape[1]), X, Wg, Wu, act, save, stream, ws)


def _gated_sizes(L: dict, M: int, K: int, N: int):
    """Rows and columns of the device's shares of X and of the weights."""
    x, w = shard(L["x"], M, K), shard(L["w"], K, N)
    return x.rows, x.cols, w.rows, w.cols


@functools.lru_cache(maxsize=1024)
def _gated_states(sig: str, p: int, r: int, M: int, K: int, N: int):
    """layouts(sig, p, r) and _gated_sizes of them. (Five calls of the library, half of the
    host's time for a small product; they depend on these numbers only.)"""
    L = layouts(sig, p, r)
    return L, _gated_sizes(L, M, K, N)


def _gated_fwd(L, sizes, X, Wg, Wu, act, save, stream, ws):
    if stream is not None and stream != sbp.current_stream():
        return on_stream(stream, _gated_fwd, L, sizes, X, Wg, Wu, act, save, None, ws)
    same_device(X, Wg, Wu, ws)
    nd = isinstance(L["x"], sbp.sbp_nd_layout_t)
    m, n = sizes[0], sizes[3]
    x = sbp.view(X)

    def new():   # a tensor and its view
        t = X.new_empty((m, n))
        return t, sbp.raw_view(t.data_ptr(), m, n, max(n, 1), x.dtype, sbp.SBP_LOCAL)

    H, h = new()
    # the fp32 path has no form without the projections in memory
    (G, g), (U, u) = (new(), new()) if save or x.dtype == sbp.SBP_F32 else ((None,) * 2,) * 2
    fn = sbp.sbp_nd_gated_fwd if nd else sbp.sbp_gated_fwd
    fn(x, L["x"], sbp.view(Wg), sbp.view(Wu), L["w"], sbp.ACTS[act], h, g, u, None, ws)
    return (H, G, U) if save else (H, None, None)


def gated_bwd_L(L: dict, dH, X, Wg, Wu, G, U, act: str = "silu", out=None, grad_dtype=None,
                accumulate: bool = False, stream=None, ws=None):
    """(dX, dWg, dWu) of the device's shares, from the upstream gradient dH (global, or the
    device's share) and the G and U of gated_fwd. They are in the inputs' dtype where no
    partial sum of several devices forbids it (or in grad_dtype), or go to the three given
    tensors `out` (accumulate: added to their fp32 contents)."""
    M, K = X.shape
    return _gated_bwd(L, _gated_sizes(L, M, K, Wg.shape[1]), dH, X, Wg, Wu, G, U, act, out,
                      grad_dtype, accumulate, stream, ws)


def _gated_bwd(L, sizes, dH, X, Wg, Wu, G, U, act, out, grad_dtype, accumulate, stream, ws):
    if stream is not None and stream != sbp.current_stream():
        return on_stream(stream, _gated_bwd, L, sizes, dH, X, Wg, Wu, G, U, act, out, grad_dtype,
                         accumulate, None, ws)
    same_device(dH, X, Wg, Wu, G, U, ws, *(out or ()))
    nd = isinstance(L["x"], sbp.sbp_nd_layout_t)
    M, N = X.shape[0], Wg.shape[1]
    m, k, kw, n = sizes

    x = sbp.view(X)

    def new(rows, cols, state):   # a tensor and its view
        t = X.new_empty((rows, cols), dtype=grad_dtype or (torch.float32 if partial_devices(state) > 1
                                                           else X.dtype))
        return t, sbp.raw_view(t.data_ptr(), rows, cols, max(cols, 1), sbp._dtype_of(t),
                               sbp.SBP_LOCAL)

    if out is None:
        if accumulate:
            raise ValueError("accumulate needs the tensors to add to")
        (dx, vx), (dg, vg), (du, vu) = (new(m, k, L["dx"]), new(kw, n, L["dw"]), new(kw, n, L["dw"]))
        out = dx, dg, du
    else:
        vx, vg, vu = (sbp.view(t, sbp.SBP_ACCUMULATE if accumulate else sbp.SBP_LOCAL) for t in out)
    pre = X.new_empty((2, m, n))   # dG, dU
    at = pre.data_ptr()
    half = lambda i: sbp.raw_view(at + i * m * n * X.element_size(), m, n, max(n, 1), x.dtype,
                                  sbp.SBP_LOCAL)
    mine = lambda t: sbp.view(t, sbp.SBP_GLOBAL if t.shape == (M, N) else sbp.SBP_LOCAL)
    fn = sbp.sbp_nd_gated_bwd if nd else sbp.sbp_gated_bwd
    fn(mine(dH), L["dy"], x, L["x"], sbp.view(Wg), sbp.view(Wu), L["w"], sbp.ACTS[act], mine(G),
       mine(U), half(0), half(1), vx, vg, vu, None, ws)
    return out


def partial_devices(l) -> int:
    """Devices over which a 1-D or nd state is a partial sum (1: the tensor is whole)."""
    if isinstance(l, sbp.sbp_nd_layout_t):
        n = 1
        for a in range(l.ndim):
            n *= l.p[a] if l.kind[a] == sbp.SBP_PARTIAL else 1
        return n
    return l.p if l.kind == sbp.SBP_PARTIAL else 1


def gated_fwd(sig: str, p: int, r: int, X, Wg, Wu, act: str = "silu", save: bool = True,
              stream=None, ws=None):
    """gated_fwd_L under signature sig ("DP", "COL" or "BB") on rank r of p."""
    M, K = X.shape
    return _gated_fwd(*_gated_states(sig, p, r, M, K, Wg.shape[1]), X, Wg, Wu, act, save,
                      stream, ws)


def gated_bwd(sig: str, p: int, r: int, dH, X, Wg, Wu, G, U, act: str = "silu", out=None,
              grad_dtype=None, accumulate: bool = False, stream=None, ws=None):
    """gated_bwd_L under signature sig on rank r of p."""
    M, K = X.shape
    return _gated_bwd(*_gated_states(sig, p, r, M, K, Wg.shape[1]), dH, X, Wg, Wu, G, U, act,
                      out, grad_dtype, accumulate, stream, ws)
