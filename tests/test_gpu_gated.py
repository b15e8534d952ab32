"""GPU tests of the gated feed-forward block against 64 bits (gated_ref.py derives the
bounds), and bit-exact on small integers: tile edges, one row, odd and strided operands,
every kernel form, signatures and device meshes, fp32, accumulating gradients, workspaces,
streams and graphs."""
import numpy as np
import pytest
import torch

import gated_ref as ref
import oracle
from paper_2301_06813_amd import inputs, linear, sbp

from helpers import out_bits, say

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
ACTS = ("silu", "gelu", "relu")


def rn(shape, std, seed, dtype=BF):
    return inputs.randn(shape, std, seed, dtype, "cuda")


def make(M, K, N, seed, dtype=BF):
    return (rn((M, K), 1.0, seed, dtype), rn((K, N), max(K, 1) ** -0.5, seed + 1, dtype),
            rn((K, N), max(K, 1) ** -0.5, seed + 2, dtype), rn((M, N), 1.0, seed + 3, dtype))


def both(X, Wg, Wu, dH, act="silu", ws=None, G=None, U=None, grad_dtype=None):
    H, g, u = linear.gated_fwd("COL", 1, 0, X, Wg, Wu, act, ws=ws)
    torch.cuda.synchronize()
    for (n, (want, bound)), got in zip(ref.forward(X, Wg, Wu, act).items(), (H, g, u)):
        ref.check(n, got, want, bound)
    G, U = g if G is None else G, u if U is None else U
    out = linear.gated_bwd("COL", 1, 0, dH, X, Wg, Wu, G, U, act, ws=ws, grad_dtype=grad_dtype)
    torch.cuda.synchronize()
    for (n, (want, bound)), got in zip(ref.backward(dH, X, Wg, Wu, G, U, act).items(), out):
        ref.check(n, got, want, bound)
    return (H, g, u), out


SHAPES = [(1, 64, 64), (1, 1024, 4096), (2, 8, 8), (3, 72, 200), (8, 512, 72), (17, 4096, 136),
          (64, 64, 64), (63, 200, 65), (130, 200, 72), (129, 33, 257), (257, 1000, 1375), (300, 1, 7),
          (5, 3, 1), (513, 256, 520), (1024, 512, 1024), (4096, 128, 2048), (32, 8192, 256),
          (2048, 64, 2056), (700, 2048, 96)]


@pytest.mark.parametrize("shape", SHAPES, ids=["x".join(map(str, s)) for s in SHAPES])
@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_shapes(shape, dtype):
    M, K, N = shape
    T = make(M, K, N, 10, dtype)
    for act in ACTS if M * N < 1 << 18 else ACTS[:1]:
        say("gated", shape, act, dtype)
        both(*T, act)


def ints(shape, hi, seed):
    return inputs.randint(shape, -hi, hi, seed, BF, "cuda")


EXACT = [(1, 64, 64), (64, 128, 64), (65, 72, 200), (200, 520, 264), (260, 130, 77), (4096, 64, 2048),
         (48, 4096, 64), (1000, 24, 136)]


@pytest.mark.parametrize("shape", EXACT, ids=["x".join(map(str, s)) for s in EXACT])
def test_exact_on_integers(shape):
    # relu on integers: every sum is a whole number below 2^24, so each output is the exact
    # value, rounded once
    M, K, N = shape
    X, Wg, Wu = ints((M, K), 1, 20), ints((K, N), 1, 21), ints((K, N), 1, 22)
    say("exact", shape)
    H, G, U = linear.gated_fwd("COL", 1, 0, X, Wg, Wu, "relu")
    g, u = ref.mm(X.double(), Wg.double()), ref.mm(X.double(), Wu.double())
    want = {"H": torch.clamp(g, min=0) * u, "G": g, "U": u}
    assert float(want["H"].abs().max()) < 2 ** 24
    for (n, w), got in zip(want.items(), (H, G, U)):
        assert np.array_equal(out_bits(got), oracle.round_bf16(w.cpu().numpy())), n
    only = linear.gated_fwd("COL", 1, 0, X, Wg, Wu, "relu", save=False)
    assert torch.equal(only[0], H) and only[1] is None
    # dG and dU are whole numbers of at most 9
    dH, G, U = ints((M, N), 3, 23), ints((M, N), 3, 24), ints((M, N), 3, 25)
    out = linear.gated_bwd("COL", 1, 0, dH, X, Wg, Wu, G, U, "relu", grad_dtype=F32)
    bf = linear.gated_bwd("COL", 1, 0, dH, X, Wg, Wu, G, U, "relu")
    dG = dH.double() * U.double() * (G.double() > 0)
    dU = dH.double() * torch.clamp(G.double(), min=0)
    Xt = X.double().t()
    want = (ref.mm(dG, Wg.double().t()) + ref.mm(dU, Wu.double().t()), ref.mm(Xt, dG), ref.mm(Xt, dU))
    for n, got, b, w in zip(("dX", "dWg", "dWu"), out, bf, want):
        assert torch.equal(got.double(), w), n
        assert np.array_equal(out_bits(b), oracle.round_bf16(w.cpu().numpy())), n


def test_empty():
    for M, K, N in ((0, 64, 64), (5, 0, 9), (5, 64, 0)):
        for dtype in (BF, F32):
            say("empty", M, K, N, dtype)
            (H, g, u), (dX, dWg, dWu) = both(*make(M, K, N, 30, dtype))
            for t in (H, g, u, dX, dWg, dWu):
                assert float(t.double().abs().sum()) == 0


def test_strided_and_unaligned():
    # the two projections as halves of one matrix, rows padded, starts inside a
    # 16-byte block; what lies beside the outputs stays as it is
    M, K, N = 150, 264, 328
    for off, pad in ((0, 8), (1, 3), (4, 4)):
        fused = rn((K, 2 * N + pad + off), K ** -0.5, 40)
        Wg, Wu = fused[:, off:off + N], fused[:, off + N:off + 2 * N]
        X = rn((M, K + pad), 1.0, 41)[:, off and 2:][:, :K]
        dH = rn((M, N + pad + off), 1.0, 42)[:, off:off + N]
        say("strided", off, pad)
        (H, G, U), grads = both(X, Wg, Wu, dH)
        L = linear.layouts("COL", 1, 0)
        lo = lambda t: sbp.view(t, sbp.SBP_LOCAL)
        one = [torch.full((M + 1, N + pad), 7.0, dtype=BF, device="cuda") for _ in range(3)]
        v = [t[1:, off:off + N] for t in one]
        sbp.sbp_gated_fwd(sbp.view(X), L["x"], sbp.view(Wg), sbp.view(Wu), L["w"], sbp.SBP_ACT_SILU,
                          *(lo(t) for t in v))
        for t, w, b in zip(v, (H, G, U), one):
            assert torch.equal(t, w)
            assert (b[0] == 7).all() and (b[:, :off] == 7).all() and (b[:, off + N:] == 7).all()
        out = [torch.full((M, K + pad), 7.0, dtype=BF, device="cuda")[:, :K],
               torch.full((K, N + pad), 7.0, dtype=BF, device="cuda")[:, :N],
               torch.full((K, N + pad + 8), 7.0, dtype=BF, device="cuda")[:, :N]]   # another stride
        linear.gated_bwd("COL", 1, 0, dH, X, Wg, Wu, G, U, out=out)
        torch.cuda.synchronize()
        for (n, (want, bound)), got in zip(ref.backward(dH, X, Wg, Wu, G, U, "silu").items(), out):
            ref.check(n, got, want, bound)
            base = got._base if got._base is not None else got
            assert (base[:, got.shape[1]:] == 7).all()


@pytest.mark.parametrize("sig", ["DP", "COL", "BB"])
def test_signatures_every_rank(sig):
    M, K, N = 70, 96, 150
    X, Wg, Wu, dH = make(M, K, N, 50)
    for p in (1, 2, 3):
        for r in range(p):
            L = linear.layouts(sig, p, r)
            x, w = linear.shard(L["x"], M, K), linear.shard(L["w"], K, N)
            rows, cols = slice(x.row_off, x.row_off + x.rows), slice(w.col_off, w.col_off + w.cols)
            say("signature", sig, p, r)
            H, G, U = linear.gated_fwd(sig, p, r, X, Wg, Wu, "gelu")
            for (n, (want, bound)), got in zip(
                    ref.forward(X[rows], Wg[:, cols], Wu[:, cols], "gelu").items(), (H, G, U)):
                ref.check(n, got, want, bound)
            wants = ref.backward(dH[rows, cols], X[rows], Wg[:, cols], Wu[:, cols], G, U, "gelu")
            for d in (dH, dH[rows, cols]):            # global, and this rank's share
                out = linear.gated_bwd(sig, p, r, d, X, Wg, Wu, G, U, "gelu")
                for (n, (want, bound)), got in zip(wants.items(), out):
                    ref.check(n, got, want, bound)
                    st = L["dx"] if n == "dX" else L["dw"]
                    assert got.dtype == (F32 if linear.partial_devices(st) > 1 else BF)


def test_device_mesh():
    M, K, N = 60, 64, 88
    X, Wg, Wu, dH = make(M, K, N, 60)
    for factors in (("DP", "COL"), ("COL", "DP"), ("BB", "COL")):
        for c in ((0, 0), (1, 0), (0, 1), (1, 1)):
            L = linear.nd_layouts(factors, (2, 2), c)
            x, w = linear.shard(L["x"], M, K), linear.shard(L["w"], K, N)
            rows, cols = slice(x.row_off, x.row_off + x.rows), slice(w.col_off, w.col_off + w.cols)
            say("mesh", factors, c)
            H, G, U = linear.gated_fwd_L(L, X, Wg, Wu)
            for (n, (want, bound)), got in zip(
                    ref.forward(X[rows], Wg[:, cols], Wu[:, cols], "silu").items(), (H, G, U)):
                ref.check(n, got, want, bound)
            out = linear.gated_bwd_L(L, dH, X, Wg, Wu, G, U)
            for (n, (want, bound)), got in zip(
                    ref.backward(dH[rows, cols], X[rows], Wg[:, cols], Wu[:, cols], G, U,
                                 "silu").items(), out):
                ref.check(n, got, want, bound)


@pytest.mark.parametrize("shape", [(200, 136, 264), (96, 50, 75), (64, 2048, 64), (4096, 64, 64)],
                         ids=["aligned", "odd", "long k", "long m"])
@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_accumulation(shape, dtype):
    M, K, N = shape
    X, Wg, Wu, dH = make(M, K, N, 70, dtype)
    _, G, U = linear.gated_fwd("COL", 1, 0, X, Wg, Wu)
    for ws in (None, sbp.NO_WORKSPACE):
        new = [torch.empty(s, dtype=F32, device="cuda") for s in ((M, K), (K, N), (K, N))]
        old = [rn(t.shape, 1.0, 80 + i, F32) for i, t in enumerate(new)]
        out = [t.clone() for t in old]
        say("accumulate", shape, dtype, ws is None)
        linear.gated_bwd("COL", 1, 0, dH, X, Wg, Wu, G, U, out=out, accumulate=True, ws=ws)
        torch.cuda.synchronize()
        wants = ref.backward(dH, X, Wg, Wu, G, U, "silu")
        for (n, (want, bound)), got, was in zip(wants.items(), out, old):
            # adding to the contents rounds twice more (fp32 dX: once per product)
            extra = 3 * ref.E * (was.double().abs() + want.abs() + bound)
            ref.check(n, got, want + was.double(), bound + extra)


def test_no_workspace():
    for shape in ((16, 4096, 96), (4096, 72, 136), (8, 200, 75)):
        say("no workspace", shape)
        both(*make(*shape, 90), ws=sbp.NO_WORKSPACE)


def test_extreme_preactivations():
    # gates far out on both sides: act and its slope stay finite and reach their limits
    M, K, N = 16, 8, 24
    X, Wg, Wu, dH = make(M, K, N, 95)
    far = torch.tensor([-1e30, -3e4, -200.0, -30.0, 30.0, 200.0, 3e4, 1e30], device="cuda")
    G = far.repeat(3)[None].expand(M, N).contiguous().to(BF)
    U = rn((M, N), 1.0, 96)
    for act in ACTS:
        say("extremes", act)
        out = linear.gated_bwd("COL", 1, 0, dH, X, Wg, Wu, G, U, act, grad_dtype=F32)
        a, d = ref.act(G.double(), act)
        a, d = torch.nan_to_num(a, 0.0), torch.where(G < 0, 0.0, 1.0).double()
        dG, dU = dH.double() * U.double() * d, dH.double() * torch.where(G < 0, 0.0, a)
        want = ref.mm(X.double().t(), dG)
        bound = ref.U_BF * ref.mm(X.double().abs().t(), dG.abs()) * (1 + 2.0 ** -6) + 1e-6
        ref.check("dWg", out[1], want, bound)
        assert torch.isfinite(out[2]).all()


def test_deterministic_streams_and_graph():
    M, K, N = 300, 1024, 200
    X, Wg, Wu, dH = make(M, K, N, 110)
    Xt = rn((1, K), 1.0, 114)
    H, G, U = linear.gated_fwd("COL", 1, 0, X, Wg, Wu)
    g = linear.gated_bwd("COL", 1, 0, dH, X, Wg, Wu, G, U)
    h1 = linear.gated_fwd("COL", 1, 0, Xt, Wg, Wu, save=False)[0]
    st = torch.cuda.Stream()
    ws = torch.empty(sbp.SBP_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    say("side stream")
    with torch.cuda.stream(st):
        H2, G2, U2 = linear.gated_fwd("COL", 1, 0, X, Wg, Wu)
        g2 = linear.gated_bwd("COL", 1, 0, dH, X, Wg, Wu, G2, U2)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((H, G, U, *g), (H2, G2, U2, *g2)))
    graph = torch.cuda.CUDAGraph()
    say("capture")
    with torch.cuda.graph(graph, stream=st):
        H3, G3, U3 = linear.gated_fwd("COL", 1, 0, X, Wg, Wu, ws=ws)
        g3 = linear.gated_bwd("COL", 1, 0, dH, X, Wg, Wu, G3, U3, ws=ws)
        h3 = linear.gated_fwd("COL", 1, 0, Xt, Wg, Wu, save=False, ws=ws)[0]
    for rep in range(4):
        for t in (H3, G3, U3, h3, *g3):
            t.fill_(3)
        graph.replay()
        linear.gated_fwd("COL", 1, 0, Xt, Wg, Wu)     # eager work between the replays
        torch.cuda.synchronize()
        say("replay", rep)
        assert all(torch.equal(a, b) for a, b in zip((H, G, U, h1, *g), (H3, G3, U3, h3, *g3)))


def test_gradients_against_differences():
    # loss = sum(dH * H) of the 64-bit reference along random directions: central
    # differences with step 2^-10, whose error is of the order 2^-20 of the third
    # derivative, far below the gradients' own bounds
    M, K, N = 24, 40, 56
    X, Wg, Wu, dH = make(M, K, N, 120, F32)
    for act in ("silu", "gelu"):
        H, G, U = linear.gated_fwd("COL", 1, 0, X, Wg, Wu, act)
        grads = linear.gated_bwd("COL", 1, 0, dH, X, Wg, Wu, G, U, act)
        # G and U are inputs rounded to fp32 sums: (K + 8) 2^-24 of their sums' sizes, and
        # the loss's slopes and curvatures in them stay below a few times |dH| (1 + |U|)
        args = [X.double(), Wg.double(), Wu.double()]
        loss = lambda a: float((ref.forward(*a, act)["H"][0] * dH.double()).sum())
        bounds = ref.backward(dH, X, Wg, Wu, G, U, act)
        for i, n in enumerate(("dX", "dWg", "dWu")):
            d = rn(args[i].shape, 1.0, 130 + i, F32).double()
            h = 2.0 ** -10
            up, dn = list(args), list(args)
            up[i], dn[i] = args[i] + h * d, args[i] - h * d
            want = (loss(up) - loss(dn)) / (2 * h)
            got = float((grads[i].double() * d).sum())
            size = float((bounds[n][1] * d.abs()).sum())
            curve = h * h * float((grads[i].double() * d).abs().sum()) * 8
            say("difference", act, n, got, want, size + curve)
            assert abs(got - want) <= size + curve


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("shape", [(150, 264, 328), (70, 51, 45), (33, 130, 66), (40, 68, 1030)],
                         ids=["aligned", "odd", "even", "wide"])
def test_weights_with_strides_of_their_own(shape, dtype):
    # each weight and each of dH, G and U in rows of its own length, with and without a
    # workspace (fp32 operands may be copied there for wider loads)
    M, K, N = shape
    rows = lambda r, c, pad, seed, std: rn((r, c + pad), std, seed, dtype)[:, :c]
    X = rows(M, K, 8, 131, 1.0)
    Wg, Wu = rows(K, N, 8, 132, K ** -0.5), rows(K, N, 24, 133, K ** -0.5)
    dH, G, U = (rows(M, N, 8 * i, 134 + i, 1.0) for i in range(3))
    for ws in (None, sbp.NO_WORKSPACE):
        say("own strides", shape, dtype, ws is None)
        both(X, Wg, Wu, dH, ws=ws, G=G, U=U)


WIDE = (1 << 21) + 4     # elements from row to row, past what the pipelined kernels' offsets reach


@pytest.mark.parametrize("which", ["X", "weights", "all"])
@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_rows_far_apart(dtype, which):
    # operands with leading dimensions past 2^21: bf16 through registers; fp32 gradients as two
    # pairs of products, the second of which adds its dX to the first's
    M, K, N = 70, 72, 96
    T = make(M, K, N, 140, dtype)
    wide = torch.empty(80 * WIDE, dtype=dtype, device="cuda")

    def far(t, i):          # the same matrix with its rows WIDE apart
        v = wide.as_strided(t.shape, (WIDE, 1), 128 * i)
        v.copy_(t)
        return v

    X, Wg, Wu, dH = (far(t, i) if which == "all" or (which == "X") == (i == 0) and i < 3 else t
                     for i, t in enumerate(T))
    say("rows far apart", dtype, which)
    sbp.sbp_profile_begin(32)
    (H, G, U), grads = both(X, Wg, Wu, dH)
    names = " ".join(n for n, _ in sbp.sbp_profile_end(32))
    if dtype == F32:
        assert "gemm_f32_gated_bwd" not in names
    if which == "all":
        G, U = far(G, 4), far(U, 5)
        both(X, Wg, Wu, dH, G=G, U=U)
    wants = ref.backward(dH, X, Wg, Wu, G, U, "silu")
    old = [rn(t.shape, 1.0, 150 + i, F32) for i, t in enumerate(grads)]
    for ws in (None, sbp.NO_WORKSPACE):
        say("accumulating", ws is None)
        out = [t.clone() for t in old]
        linear.gated_bwd("COL", 1, 0, dH, X, Wg, Wu, G, U, out=out, accumulate=True, ws=ws)
        torch.cuda.synchronize()
        for (n, (want, bound)), got, was in zip(wants.items(), out, old):
            # adding to the contents rounds twice more (fp32 dX: once per product)
            extra = 3 * ref.E * (was.double().abs() + want.abs() + bound)
            ref.check(n, got, want + was.double(), bound + extra)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_offsets_past_32_bits(dtype):
    # an operand whose rows lie on both sides of 2^31 elements, and outputs that do
    if torch.cuda.mem_get_info()[0] < 48 << 30:
        pytest.skip("needs 48 GiB of device memory")
    M, K, N = 70, 72, 96
    X, Wg, Wu, dH = make(M, K, N, 160, dtype)
    ld = (1 << 31) // 40 + 8          # row 40 starts past 2^31
    say("offsets", dtype)
    wide = torch.empty(72 * ld, dtype=dtype, device="cuda")
    far = lambda buf, t: buf.as_strided(t.shape, (ld, 1))
    want_f = ref.forward(X, Wg, Wu, "silu")
    H, G, U = linear.gated_fwd("COL", 1, 0, X, Wg, Wu)
    want_b = ref.backward(dH, X, Wg, Wu, G, U, "silu")
    for i in range(3):
        T = [X, Wg, Wu]
        T[i] = far(wide, T[i])
        T[i].copy_((X, Wg, Wu)[i])
        say("offsets of operand", i)
        for (n, (want, bound)), got in zip(want_f.items(), linear.gated_fwd("COL", 1, 0, *T)):
            ref.check(n, got, want, bound)
        for (n, (want, bound)), got in zip(want_b.items(),
                                           linear.gated_bwd("COL", 1, 0, dH, *T, G, U)):
            ref.check(n, got, want, bound)
    for i in range(3):
        out = [torch.empty_like(t) for t in (X, Wg, Wu)]
        out[i] = far(wide, out[i])
        say("offsets of gradient", i)
        linear.gated_bwd("COL", 1, 0, dH, X, Wg, Wu, G, U, out=out)
        for (n, (want, bound)), got in zip(want_b.items(), out):
            ref.check(n, got, want, bound)
    v, L, g, u = far(wide, H), linear.layouts("COL", 1, 0), torch.empty_like(G), torch.empty_like(U)
    say("offsets of H")
    sbp.sbp_gated_fwd(sbp.view(X), L["x"], sbp.view(Wg), sbp.view(Wu), L["w"], sbp.SBP_ACT_SILU,
                      *(sbp.view(t, sbp.SBP_LOCAL) for t in (v, g, u)))
    torch.cuda.synchronize()
    ref.check("H", v, *want_f["H"])


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_extreme_preactivations_every_gradient(act, dtype):
    # gates far out on both sides: all three gradients and H against the gate's limits, act(x) = x
    # or 0 and its slope 1 or 0 (at |x| of 200 and more SiLU and GELU are within 2^-100 of them)
    M, K, N = 16, 8, 24
    X, Wg, Wu, dH = make(M, K, N, 170, dtype)
    far = torch.tensor([-1e18, -3e4, -200.0, 200.0, 3e4, 1e18], device="cuda")
    G = far.repeat(4)[None].expand(M, N).contiguous().to(dtype)
    U = rn((M, N), 1.0, 171, dtype)
    say("extremes", act, dtype)
    out = linear.gated_bwd("COL", 1, 0, dH, X, Wg, Wu, G, U, act, grad_dtype=F32)
    on = (G > 0).double()
    a, u = G.double() * on, ref.U_BF if dtype == BF else ref.U_F32
    dG, dU = dH.double() * U.double() * on, dH.double() * a
    Xt, W = X.double().t(), (Wg.double().t(), Wu.double().t())
    want = (ref.mm(dG, W[0]) + ref.mm(dU, W[1]), ref.mm(Xt, dG), ref.mm(Xt, dU))
    e = [u * t.abs() + ref.A * s.abs() for t, s in ((dG, dH.double() * U.double()), (dU, dU))]
    sizes = (ref.mm(dG.abs(), W[0].abs()) + ref.mm(dU.abs(), W[1].abs()), ref.mm(Xt.abs(), dG.abs()),
             ref.mm(Xt.abs(), dU.abs()))
    off = (ref.mm(e[0], W[0].abs()) + ref.mm(e[1], W[1].abs()), ref.mm(Xt.abs(), e[0]),
           ref.mm(Xt.abs(), e[1]))
    terms = (2 * N, M, M)
    for n, got, w, b, s, t in zip(("dX", "dWg", "dWu"), out, want, off, sizes, terms):
        ref.check(n, got, w, b + (t + 8) * ref.E * (1 + u) * s + 2.0 ** -99)
    # H from such sums: one reduction index, whose products are exact
    X1, W1 = torch.ones((M, 1), dtype=dtype, device="cuda"), G[:1]
    Wu1 = rn((1, N), 1.0, 172, dtype)
    H, g, _ = linear.gated_fwd("COL", 1, 0, X1, W1, Wu1, act)
    assert torch.equal(g, G)
    h = a * Wu1.double()
    ref.check("H", H, h, ref.A * h.abs() + 2.0 ** -99)
