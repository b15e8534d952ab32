"""One Transformer layer's shares, forward and backward, of every device of a tensor-parallel
group: column-split projections of Q, K and V, softmax attention of the device's heads,
row-split output projection, gated block, row-split down projection. The devices run one
after the other on one GPU; sums of their partial outputs stand for the all-reduces."""
import math

import pytest
import torch

import attn_core_ref
import gated_ref
from paper_2301_06813_amd import attention, inputs, linear, sbp

from helpers import say

pytestmark = pytest.mark.gpu
BF, F32, F64 = torch.bfloat16, torch.float32, torch.float64
WEIGHTS = ("q", "k", "v", "o", "g", "u", "d")


def make(B, S, D, heads, kv, dm, hid):
    rn = lambda shape, std, seed: inputs.randn(shape, std, seed, BF, "cuda")
    shapes = {"q": (dm, heads * D), "k": (dm, kv * D), "v": (dm, kv * D), "o": (heads * D, dm),
              "g": (dm, hid), "u": (dm, hid), "d": (hid, dm)}
    W = {n: rn(s, s[0] ** -0.5, 7 + i) for i, (n, s) in enumerate(shapes.items())}
    return rn((B * S, dm), 1.0, 1), rn((B * S, dm), 1.0, 2), W


def heads_of(t, B, S, D):
    """[batch * rows][heads * D] as [batch][heads][rows][D]."""
    return t.view(B, S, -1, D).permute(0, 2, 1, 3)


def flat(t):
    B, h, S, D = t.shape
    return t.permute(0, 2, 1, 3).reshape(B * S, h * D)


def row_split(op, p, r, X, W, dY):
    """A product of a row-split (KS) linear whose X is the device's share already."""
    L = linear.layouts("KS", p, r)
    M, K, N = (X if X is not None else dY).shape[0], W.shape[0], W.shape[1]
    out = linear.alloc_out(op, "KS", p, r, M, K, N, BF, "cuda")
    o = sbp.view(out, sbp.SBP_LOCAL)
    if op == "fwd":
        sbp.sbp_linear_fwd(sbp.view(X, sbp.SBP_LOCAL), L["x"], sbp.view(W), L["w"], o)
    elif op == "bwd_data":
        sbp.sbp_linear_bwd_data(sbp.view(dY), L["dy"], sbp.view(W), L["w"], o)
    else:
        sbp.sbp_linear_bwd_weight(sbp.view(X, sbp.SBP_LOCAL), L["x"], sbp.view(dY), L["dy"], o)
    return out


def layer(p, B, S, D, x, dy, W, seen):
    """(y, dx, {weight: gradient}) of the layer; seen(kind, tensors) gets each stage."""
    s = 1 / math.sqrt(D)
    kw = dict(scale=s, causal=True, scope=sbp.SBP_LOCAL)
    kept, total = [], 0
    for r in range(p):
        q, k, v = (heads_of(linear.call("fwd", "COL", p, r, x, W[n], None)[0], B, S, D) for n in "qkv")
        o, lse = attention.core_fwd(q, k, v, p, r, **kw)
        seen("attn", (q, k, v, o, lse, s))
        total = total + row_split("fwd", p, r, flat(o), W["o"], None).float()
        kept.append((q, k, v, o, lse))
    h = (x.float() + total).to(BF)
    total = 0
    for r in range(p):
        H, G, U = linear.gated_fwd("COL", p, r, h, W["g"], W["u"])
        n = G.shape[1]
        mine = slice(r * n, (r + 1) * n)
        seen("gated", (h, W["g"][:, mine], W["u"][:, mine], H, G, U))
        total = total + row_split("fwd", p, r, H, W["d"], None).float()
        kept[r] += (H, G, U)
    y = (h.float() + total).to(BF)

    grads = {n: [] for n in WEIGHTS}
    total = 0
    for r in range(p):
        H, G, U = kept[r][5:]
        dH = row_split("bwd_data", p, r, None, W["d"], dy)
        grads["d"].append(row_split("bwd_weight", p, r, H, W["d"], dy))
        dX, dWg, dWu = linear.gated_bwd("COL", p, r, dH, h, W["g"], W["u"], G, U)
        n = G.shape[1]
        mine = slice(r * n, (r + 1) * n)
        seen("gated_bwd", (dH, h, W["g"][:, mine], W["u"][:, mine], G, U, dX, dWg, dWu))
        grads["g"].append(dWg)
        grads["u"].append(dWu)
        total = total + dX.float()
    dh = (dy.float() + total).to(BF)
    total = dh.float()
    for r in range(p):
        q, k, v, o, lse = kept[r][:5]
        do = heads_of(row_split("bwd_data", p, r, None, W["o"], dh), B, S, D)
        grads["o"].append(row_split("bwd_weight", p, r, flat(o), W["o"], dh))
        g = attention.core_bwd(do, q, k, v, o, lse, p, r, **kw)
        seen("attn_bwd", (do, q, k, v, o, lse, s, *g))
        L = linear.layouts("COL", p, r)
        for n, t in zip("qkv", g):
            d = flat(t)
            dx = linear.alloc_out("bwd_data", "COL", p, r, *x.shape, W[n].shape[1], BF, "cuda")
            dw = linear.alloc_out("bwd_weight", "COL", p, r, *x.shape, W[n].shape[1], BF, "cuda")
            share = sbp.view(d, sbp.SBP_LOCAL)
            sbp.sbp_linear_bwd_data(share, L["dy"], sbp.view(W[n]), L["w"], sbp.view(dx, sbp.SBP_LOCAL))
            sbp.sbp_linear_bwd_weight(sbp.view(x), L["x"], share, L["dy"], sbp.view(dw, sbp.SBP_LOCAL))
            total = total + dx.float()
            grads[n].append(dw)
    return y, total, {n: torch.cat(g, 0 if n in "od" else 1) for n, g in grads.items()}


def check_stage(kind, t):
    """A stage against 64 bits, from the tensors that it read."""
    if kind == "attn":
        q, k, v, o, lse, s = t
        want, bound, wl = attn_core_ref.forward(q, k, v, s, True, 0, None, None)
        attn_core_ref.check("O", o, want, bound)
        assert float((lse.double() - wl).abs().max()) <= 2.0 ** -14
    elif kind == "attn_bwd":
        do, q, k, v, o, lse, s, *g = t
        for n, got, (want, bound) in zip(("dQ", "dK", "dV"), g, attn_core_ref.backward(
                do, q, k, v, o, lse, s, True, 0, None, None)):
            attn_core_ref.check(n, got, want, bound)
    elif kind == "gated":
        h, g, u, H, G, U = t
        for (n, (want, bound)), got in zip(gated_ref.forward(h, g, u, "silu").items(), (H, G, U)):
            gated_ref.check(n, got, want, bound)
    else:
        dH, h, g, u, G, U, *out = t
        for (n, (want, bound)), got in zip(gated_ref.backward(dH, h, g, u, G, U, "silu").items(), out):
            gated_ref.check(n, got, want, bound)


def reference(B, S, D, x, dy, W):
    """The whole layer and its gradients in 64 bits (on the CPU)."""
    x = x.cpu().to(F64).requires_grad_()
    W = {n: w.cpu().to(F64).requires_grad_() for n, w in W.items()}
    q, k, v = (heads_of(x @ W[n], B, S, D) for n in "qkv")
    g = q.shape[1] // k.shape[1]
    k, v = k.repeat_interleave(g, 1), v.repeat_interleave(g, 1)
    z = q @ k.transpose(2, 3) / math.sqrt(D)
    z = z.masked_fill(torch.ones(S, S).triu(1).bool(), -math.inf)
    h = x + flat(torch.softmax(z, 3) @ v) @ W["o"]
    y = h + (torch.nn.functional.silu(h @ W["g"]) * (h @ W["u"])) @ W["d"]
    grads = torch.autograd.grad(y, (x, *W.values()), dy.cpu().to(F64))
    return y.detach(), grads[0], dict(zip(W, grads[1:]))


# every output lies at most 13 roundings to bf16 from the inputs (dWq: Q, K, V, P, O, the
# projection and h; G and U, H; dH, dG, dX and dh, dO, dS, dQ), each at most 2^-8 of what is
# rounded. Their sum, and as much again for sums that are smaller than their terms, bounds
# the distance in norm; a share that is left out or taken twice changes an output by a
# large part of its own norm.
FAR = 2 * 13 * 2.0 ** -8


@pytest.mark.parametrize("p", [1, 2])
@pytest.mark.parametrize("dims", [(2, 72, 32, 4, 2, 128, 256), (1, 200, 128, 2, 2, 256, 384),
                                  (3, 33, 40, 4, 4, 96, 136)],
                         ids=["grouped", "wide heads", "odd"])
def test_layer(dims, p):
    B, S, D = dims[:3]
    x, dy, W = make(*dims)
    say("layer", dims, p)

    def seen(kind, t):
        torch.cuda.synchronize()
        check_stage(kind, t)

    y, dx, grads = layer(p, B, S, D, x, dy, W, seen)
    wy, wx, wg = reference(B, S, D, x, dy, W)
    rel = lambda got, want: float((got.cpu().to(F64) - want).norm() / want.norm())
    assert rel(y, wy) <= FAR and rel(dx, wx) <= FAR
    for n in WEIGHTS:
        assert grads[n].shape == W[n].shape
        assert rel(grads[n], wg[n]) <= FAR, n


def test_layer_captured():
    # the layer as one graph: every replay writes the eager results, with eager calls of
    # the same operators between the replays
    dims = (2, 72, 32, 4, 2, 128, 256)
    x, dy, W = make(*dims)
    run = lambda: layer(2, *dims[:3], x, dy, W, lambda *a: None)
    y, dx, grads = run()
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        run()                         # the stream's workspace is there before the capture
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    say("capture")
    with torch.cuda.graph(graph, stream=st):
        y2, dx2, grads2 = run()
    for rep in range(3):
        for t in (y2, dx2, *grads2.values()):
            t.fill_(5)
        graph.replay()
        run()
        torch.cuda.synchronize()
        say("replay", rep)
        assert torch.equal(y, y2) and torch.equal(dx, dx2)
        assert all(torch.equal(grads[n], grads2[n]) for n in WEIGHTS)


def test_two_graphs_share_a_workspace():
    # an attention pass and a gated pass captured into graphs of their own that share one
    # workspace, replayed in turn on one stream: row statistics go there, and partials
    B, S, D = 1, 1500, 64
    rn = lambda shape, seed: inputs.randn(shape, 1.0, seed, BF, "cuda")
    Q, K, V, dO = (rn((B, 4, S, D), 40 + i) for i in range(4))
    X, Wg, Wu, dH = rn((40, 4096), 50), rn((4096, 96), 51), rn((4096, 96), 52), rn((40, 96), 53)
    ws = torch.empty(sbp.SBP_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")

    def attn():
        O, lse = attention.core_fwd(Q, K, V, ws=ws)
        return (O, lse, *attention.core_bwd(dO, Q, K, V, O, lse, ws=ws))

    def gated():
        H, G, U = linear.gated_fwd("COL", 1, 0, X, Wg, Wu, ws=ws)
        return (H, G, U, *linear.gated_bwd("COL", 1, 0, dH, X, Wg, Wu, G, U, ws=ws))

    sbp.sbp_profile_begin(32)
    want = [f() for f in (attn, gated)]
    names = " ".join(n for n, _ in sbp.sbp_profile_end(32))
    assert all(n in names for n in ("attn_core_stat", "gated_join"))
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    graphs, got = [torch.cuda.CUDAGraph() for _ in range(2)], []
    say("capture two")
    for g, f in zip(graphs, (attn, gated)):
        with torch.cuda.graph(g, stream=st):
            got.append(f())
    for rep in range(3):
        for out in got:
            for t in out:
                t.fill_(9)
        with torch.cuda.stream(st):
            torch.cuda.current_stream().wait_stream(torch.cuda.default_stream())
            for g in (graphs if rep % 2 else graphs[::-1]):
                g.replay()
        torch.cuda.synchronize()
        say("replay", rep)
        assert all(torch.equal(a, b) for w, o in zip(want, got) for a, b in zip(w, o))
