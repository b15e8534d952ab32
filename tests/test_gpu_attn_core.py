"""GPU tests of softmax attention, forward and backward, against 64 bits
(attn_core_ref.py derives the bounds): sizes around the tiles' edges, one query
row, grouped heads, head splits, masks that leave rows empty, padded batches,
strided and unaligned operands, fp32 and accumulating gradients, workspaces of
every kind, streams and graphs."""
import math

import pytest
import torch

import attn_core_ref as ref
from paper_2301_06813_amd import attention, sbp

from helpers import say

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def rn(shape, seed, dtype=BF):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def lens(v):
    return None if v is None else torch.tensor(v, dtype=torch.int32, device="cuda")


def tensors(B, H, Hk, sq, sk, D, seed, fused=False):
    if fused:
        act = rn((B, sq, H + 2 * Hk, D), seed).permute(0, 2, 1, 3)
        return act[:, :H], act[:, H:H + Hk], act[:, H + Hk:], rn((B, sq, H, D), seed + 3).permute(0, 2, 1, 3)
    return (rn((B, H, sq, D), seed), rn((B, Hk, sk, D), seed + 1), rn((B, Hk, sk, D), seed + 2),
            rn((B, H, sq, D), seed + 3))


def both(Q, K, V, dO, causal=False, window=0, lq=None, lk=None, out_dtype=None, ws=None, scale=None):
    D = Q.shape[-1]
    s = 1 / math.sqrt(D) if scale is None else scale
    kw = dict(scale=s, causal=causal, window=window, len_q=lens(lq), len_k=lens(lk), ws=ws)
    O, lse = attention.core_fwd(Q, K, V, out_dtype=out_dtype, **{**kw, "ws": None if ws is not None
                                and not isinstance(ws, sbp.sbp_workspace_t) else ws})
    torch.cuda.synchronize()
    wO, bO, wl = ref.forward(Q, K, V, s, causal, window, lq, lk)
    ref.check("O", O, wO, bO)
    empty = wl == -math.inf
    assert torch.equal(lse == -math.inf, empty)
    off = (lse.double() - wl)[~empty].abs()
    # scores below 2^5 in fp32, one logarithm: 2^-14 as in the bounds' F
    assert off.numel() == 0 or float(off.max()) <= 2.0 ** -14
    assert float(O[empty].abs().sum()) == 0.0
    g = attention.core_bwd(dO, Q, K, V, O, lse, grad_dtype=out_dtype, **{**kw, "ws": ws if not
                           isinstance(ws, sbp.sbp_workspace_t) else None})
    torch.cuda.synchronize()
    for n, got, (want, bound) in zip(("dQ", "dK", "dV"), g,
                                     ref.backward(dO, Q, K, V, O, lse, s, causal, window, lq, lk)):
        ref.check(n, got, want, bound)
    return O, lse, g


SHAPES = [  # B, H, Hk, sq, sk, D, causal, window
    (1, 1, 1, 1, 1, 64, False, 0), (1, 1, 1, 1, 1, 64, True, 0), (2, 3, 3, 1, 33, 64, True, 0),
    (1, 2, 2, 32, 32, 64, True, 0), (2, 2, 1, 31, 65, 64, False, 0), (1, 4, 2, 64, 64, 128, True, 0),
    (2, 3, 3, 197, 197, 64, False, 0), (1, 6, 2, 333, 333, 80, True, 100),
    (1, 2, 1, 129, 257, 128, True, 0), (1, 2, 2, 257, 129, 64, True, 0),   # rows that see nothing
    (3, 14, 2, 5, 300, 40, True, 0), (1, 7, 1, 2, 1000, 128, False, 0),
    (1, 2, 2, 100, 70, 1, False, 0), (1, 3, 3, 65, 130, 7, True, 0), (2, 2, 2, 66, 66, 36, True, 0),
    (1, 4, 4, 90, 90, 127, True, 17), (2, 1, 1, 300, 300, 72, False, 64), (1, 1, 1, 70, 70, 64, True, 1),
    (4, 16, 16, 512, 512, 64, True, 0), (2, 64, 64, 256, 256, 128, True, 0),
]


@pytest.mark.parametrize("fused", [False, True], ids=["apart", "fused"])
@pytest.mark.parametrize("shape", SHAPES, ids=["x".join(map(str, s)) for s in SHAPES])
def test_shapes(shape, fused):
    B, H, Hk, sq, sk, D, causal, window = shape
    if fused and sq != sk:
        pytest.skip("one activation holds equal rows of Q, K and V")
    say("attention", shape, fused)
    both(*tensors(B, H, Hk, sq, sk, D, 100, fused), causal, window)


def test_no_keys_and_no_rows():
    Q, K, V, dO = tensors(2, 4, 2, 9, 0, 64, 5)
    say("no keys")
    O, lse, (dQ, dK, dV) = both(Q, K, V, dO)
    assert float(O.abs().sum()) == 0 and dK.shape[2] == 0
    Q, K, V, dO = tensors(2, 4, 2, 0, 9, 64, 6)
    say("no rows")
    O, lse, (dQ, dK, dV) = both(Q, K, V, dO)
    assert float(dK.abs().sum()) == 0 and float(dV.abs().sum()) == 0 and O.shape[2] == 0


PADDED = [([70, 0, 33, 128], [70, 5, 33, 128]), ([1, 64, 65, 127], [128, 1, 0, 90]),
          ([128, 128, 128, 128], [0, 1, 31, 500]), ([-3, 700, 64, 2], [5, 128, -1, 128])]


@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 20)])
@pytest.mark.parametrize("lq,lk", PADDED, ids=["a", "b", "c", "clamped"])
@pytest.mark.parametrize("D", [64, 44])
def test_padded_batch(lq, lk, causal, window, D):
    # what lies past the lengths is never read, and its outputs are zero
    Q, K, V, dO = (t.contiguous() for t in tensors(4, 4, 2, 128, 128, D, 30))
    for b in range(4):
        nq, nk = min(max(lq[b], 0), 128), min(max(lk[b], 0), 128)
        for t, n in ((Q, nq), (dO, nq), (K, nk), (V, nk)):
            t[b, :, n:] = float("nan")
    say("padded", lq, lk, causal, window, D)
    s = 0.125
    kw = dict(scale=s, causal=causal, window=window, len_q=lens(lq), len_k=lens(lk))
    O, lse = attention.core_fwd(Q, K, V, **kw)
    wO, bO, wl = ref.forward(Q, K, V, s, causal, window, lq, lk)
    ref.check("O", O, wO, bO)
    assert torch.equal(lse == -math.inf, wl == -math.inf)
    g = attention.core_bwd(dO, Q, K, V, O, lse, **kw)
    for n, got, (want, bound) in zip(("dQ", "dK", "dV"), g,
                                     ref.backward(dO, Q, K, V, O, lse, s, causal, window, lq, lk)):
        ref.check(n, got, want, bound)
        for b in range(4):   # (a row that sees one key has dQ = 0 too, but as a difference)
            past = min(max((lq if n == "dQ" else lk)[b], 0), 128)
            assert float(got[b, :, past:].double().abs().sum()) == 0, (n, b)


def test_head_split_matches_whole():
    # every rank of 1..3 with uneven key heads, fused and local operands
    B, H, Hk, S, D = 2, 10, 5, 70, 64
    Q, K, V, dO = tensors(B, H, Hk, S, S, D, 50, True)
    O, lse, (dQ, dK, dV) = both(Q, K, V, dO, True)
    for p in (2, 3, 7):
        for r in range(p):
            q0, hq, k0, hk = attention.rank_heads(H, Hk, p, r)
            say("rank", r, "of", p, hq, hk)
            o, l = attention.core_fwd(Q, K, V, p, r, causal=True)
            assert o.shape == (B, hq, S, D)
            # GLOBAL and LOCAL forms of the backward call's other inputs
            for args in ((dO, Q, K, V, O, lse), (dO[:, q0:q0 + hq], Q, K, V, o, l)):
                g = attention.core_bwd(*args, p, r, causal=True)
                want = ref.backward(dO[:, q0:q0 + hq], Q[:, q0:q0 + hq], K[:, k0:k0 + hk],
                                    V[:, k0:k0 + hk], O[:, q0:q0 + hq], lse[:, q0:q0 + hq],
                                    1 / math.sqrt(D), True, 0, None, None)
                for n, got, (w, bound) in zip(("dQ", "dK", "dV"), g, want):
                    ref.check(n, got, w, bound)
            if hq:
                wO, bO, _ = ref.forward(Q[:, q0:q0 + hq], K[:, k0:k0 + hk], V[:, k0:k0 + hk],
                                        1 / math.sqrt(D), True, 0, None, None)
                ref.check("O", o, wO, bO)
    loc = attention.core_fwd(Q[:, 4:8], K[:, 2:4], V[:, 2:4], causal=True, scope=sbp.SBP_LOCAL)
    wO, bO, _ = ref.forward(Q[:, 4:8], K[:, 2:4], V[:, 2:4], 1 / math.sqrt(D), True, 0, None, None)
    ref.check("O", loc[0], wO, bO)


def test_fp32_outputs_and_accumulation():
    Q, K, V, dO = tensors(2, 4, 2, 75, 130, 64, 60)
    say("fp32 outputs")
    O, lse, g = both(Q, K, V, dO, True, out_dtype=F32)
    old = [rn(t.shape, 70 + i, F32) for i, t in enumerate(g)]
    out = [t.clone() for t in old]
    say("accumulating")
    for _ in range(2):
        attention.core_bwd(dO, Q, K, V, O, lse, causal=True, out=out, accumulate=True)
    torch.cuda.synchronize()
    for o, a, x in zip(out, old, g):
        torch.testing.assert_close(o, (a + x) + x, rtol=0, atol=0)


@pytest.mark.parametrize("dims", [(1, 8, 2, 3, 2000, 64), (2, 2, 2, 1, 4096, 128), (1, 1, 1, 40, 3000, 44),
                                  (1, 8, 1, 2000, 96, 64), (1, 4, 1, 1500, 40, 128)])
def test_split_over_workgroups(dims):
    # few rows or few keys: with no workspace (forward) or just the needed one (backward)
    # nothing is split; both ways agree with 64 bits
    T = tensors(*dims, 80)
    B, H, Hk, sq, sk, D = dims
    say("split", dims)
    both(*T)
    say("unsplit", dims)
    both(*T, ws=sbp.NO_WORKSPACE)
    need = attention.bwd_workspace_bytes(B, H, sq)
    both(*T, ws=torch.empty(need, dtype=torch.uint8, device="cuda"))
    O, lse = attention.core_fwd(*T[:3])
    with pytest.raises(sbp.SbpError) as ei:
        attention.core_bwd(T[3], *T[:3], O, lse, ws=torch.empty(need - 32, dtype=torch.uint8,
                                                                device="cuda"))
    assert ei.value.code == sbp.SBP_ERR_WORKSPACE


def test_unaligned_and_strided():
    # rows that start at odd elements, rows of odd length, repeated (stride 0) keys, and
    # outputs inside larger buffers whose other elements stay as they are
    B, H, S, D = 2, 3, 77, 64
    big = rn((B, H, S, D + 3), 90)
    Q, K, V = big[..., 1:D + 1], rn((B, H, S, D + 5), 91)[..., 5:], rn((1, 1, S, D), 92).expand(B, H, S, D)
    dO = rn((B, H, S, D + 1), 93)[..., :D]
    say("unaligned")
    O, lse, g = both(Q, K, V, dO, True)
    kw = dict(causal=True)
    bufO = torch.full((B, H, S + 1, D + 2), 7.0, dtype=BF, device="cuda")
    o, _ = attention.core_fwd(Q, K, V, out=bufO[:, :, 1:, 1:D + 1], **kw)
    assert torch.equal(o, O)
    assert (bufO[:, :, 0] == 7).all() and (bufO[..., 0] == 7).all() and (bufO[..., -1] == 7).all()
    # dQ, dK and dV as parts of one fused gradient
    fused = torch.zeros((B, S, 3, H, D), dtype=BF, device="cuda")
    parts = [fused[:, :, i].transpose(1, 2) for i in range(3)]
    say("fused gradient")
    attention.core_bwd(dO, Q, K, V, O, lse, out=parts, **kw)
    for x, y in zip(parts, g):
        assert torch.equal(x, y)


def test_large_scores_and_peaked_rows():
    # scores up to 2^5 scale: rows with one key far above the rest, keys that come in
    # rising and in falling order (the running maximum moves at every step, or never)
    B, H, S, D = 1, 2, 400, 64
    Q, K, V, dO = tensors(B, H, H, S, S, D, 95)
    ramp = torch.linspace(-1, 1, S, device="cuda")[:, None]
    for sign in (1, -1):
        Kr = (K.float() * 0.05 + sign * ramp * 2).to(BF)
        Qr = (Q.float().abs() * 0.3).to(BF)
        say("ramp", sign)
        both(Qr, Kr, V, dO)
        both(Qr, Kr, V, dO, True)


def test_deterministic_streams_and_graph():
    B, H, Hk, S, D = 2, 6, 2, 300, 64
    Q, K, V, dO = tensors(B, H, Hk, S, S, D, 110, True)
    O, lse = attention.core_fwd(Q, K, V, causal=True)
    g = attention.core_bwd(dO, Q, K, V, O, lse, causal=True)
    torch.cuda.synchronize()
    q1, k1, v1, _ = tensors(1, 8, 2, 1, 3000, 64, 111)      # a split forward in the same graph
    o1, l1 = attention.core_fwd(q1, k1, v1)
    st = torch.cuda.Stream()
    ws = torch.empty(sbp.SBP_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    say("side stream")
    with torch.cuda.stream(st):
        O2, lse2 = attention.core_fwd(Q, K, V, causal=True)
        g2 = attention.core_bwd(dO, Q, K, V, O2, lse2, causal=True)
    torch.cuda.synchronize()
    assert torch.equal(O, O2) and torch.equal(lse, lse2)
    assert all(torch.equal(a, b) for a, b in zip(g, g2))
    graph = torch.cuda.CUDAGraph()
    say("capture")
    with torch.cuda.graph(graph, stream=st):
        O3, lse3 = attention.core_fwd(Q, K, V, causal=True, ws=ws)
        g3 = attention.core_bwd(dO, Q, K, V, O3, lse3, causal=True, ws=ws)
        o3, l3 = attention.core_fwd(q1, k1, v1, ws=ws)
    for rep in range(4):
        for t in (O3, lse3, o3, l3, *g3):
            t.fill_(3)
        graph.replay()
        attention.core_fwd(q1, k1, v1)          # eager work between the replays
        torch.cuda.synchronize()
        say("replay", rep)
        assert torch.equal(O, O3) and torch.equal(lse, lse3) and torch.equal(o1, o3) and torch.equal(l1, l3)
        assert all(torch.equal(a, b) for a, b in zip(g, g3))


def test_gradients_against_differences():
    # d loss / d x along random directions, loss = sum(dO * O) in 64 bits of the reference
    # forward: the library's gradients predict its change. The step h = 2^-7 leaves a
    # second-order term h^2 of the third derivative (central differences), a few 1e-4 of
    # the sum of sizes; the gradients' own bounds are far larger
    B, H, Hk, S, D = 1, 4, 2, 50, 64
    Q, K, V, dO = tensors(B, H, Hk, S, S, D, 120)
    O, lse = attention.core_fwd(Q, K, V, causal=True)
    grads = attention.core_bwd(dO, Q, K, V, O, lse, causal=True, grad_dtype=F32)
    s = 1 / math.sqrt(D)
    bounds = [b for _, b in ref.backward(dO, Q, K, V, O, lse, s, True, 0, None, None)]

    def loss(q, k, v):
        return float((ref.forward(q, k, v, s, True, 0, None, None)[0] * dO.double()).sum())

    for i, name in enumerate(("Q", "K", "V")):
        x = [Q.double(), K.double(), V.double()]
        d = rn(x[i].shape, 130 + i, F32).double()
        h = 2.0 ** -7
        up, dn = list(x), list(x)
        up[i], dn[i] = x[i] + h * d, x[i] - h * d
        got = float((grads[i].double() * d).sum())
        want = (loss(*up) - loss(*dn)) / (2 * h)
        # O, which the gradients are computed from, is rounded to bf16: U |O| |dO| a row
        extra = float((ref.U * (O.double() * dO.double()).abs().sum(-1)).sum()) * s * 4
        room = float((bounds[i] * d.abs()).sum()) + extra
        say("difference", name, got, want, room)
        assert abs(got - want) <= room
        assert room < 0.5 * float((grads[i].double() * d).abs().sum())


FORMS = {("fwd", 64, 1), ("fwd", 64, 2), ("fwd", 64, 4), ("fwd", 128, 1), ("fwd", 128, 2, 8),
         ("fwd", 128, 2, 4), ("bwd", 64, 1), ("bwd", 64, 2), ("bwd", 128, 1), ("bwd", 128, 2)}


@pytest.mark.parametrize("pad", [0, 1], ids=["aligned", "unaligned"])
def test_every_form(pad):
    # sizes that reach every tile form of both passes, by 16-byte loads and through
    # registers; sequences of unequal lengths, whose last tiles are partly filled
    reached = set()
    for D, dim in ((64, 64), (128, 128), (40, 64), (120, 128)):
        for B, H, Hk, S, causal, window in ((2, 16, 16, 1024, False, 0), (2, 16, 16, 1024, True, 0),
                                            (2, 8, 8, 512, True, 0), (2, 8, 4, 512, True, 200),
                                            (1, 4, 4, 1500, True, 0)):
            if D % 64 and S == 1024:
                continue
            T = [rn((B, n, S, D + pad), 60 + i)[..., :D] for i, n in enumerate((H, Hk, Hk, H))]
            Q, K, V, dO = T
            lq, lk = ([S - 24, S // 2 + 1], [S - 34, S // 2 + 9]) if B == 2 else ([S - 3], [S])
            say("form", D, B, H, Hk, S, causal, window, pad)
            both(Q, K, V, dO, causal, window, lq, lk)
            sbp.sbp_profile_begin(16)
            O, lse = attention.core_fwd(Q, K, V, causal=causal, window=window)
            attention.core_bwd(dO, Q, K, V, O, lse, causal=causal, window=window)
            for name, _ in sbp.sbp_profile_end(16):
                kind, _, rest = name.replace("attn_core_", "").partition("_kernel<")
                if kind not in ("fwd", "bwd"):
                    continue
                v = [int(x) for x in rest.rstrip(">").split(",")]
                assert v[0] == dim and v[-1] == (pad == 0), name
                reached.add((kind, v[0], v[1], v[3]) if (kind, *v[:2]) == ("fwd", 128, 2) else
                            (kind, *v[:2]))
    assert reached == FORMS


@pytest.mark.parametrize("scale", [2.0 ** -100, 1e-20, 3.0, 2.0 ** 100])
def test_extreme_scales(scale):
    # scores near zero: every key has the same weight; and scores so large that one key has
    # it all (small integers, so that the largest score is the largest by far)
    Q, K, V, dO = tensors(1, 4, 2, 70, 90, 64, 70)
    if scale > 1:
        Q, K = torch.zeros_like(Q), torch.zeros_like(K)
        Q[..., 0], K[..., 0] = 1.0, 0.0
        K[:, :, 17, 0] = 64.0
    say("scale", scale)
    O, lse = attention.core_fwd(Q, K, V, scale=scale)
    g = attention.core_bwd(dO, Q, K, V, O, lse, scale=scale)
    torch.cuda.synchronize()
    v = V.double().repeat_interleave(2, 1)
    want = v[:, :, 17:18] if scale > 1 else v.mean(2, keepdim=True)
    # P rounded to bf16, sums of 90 terms in fp32, O rounded to bf16
    room = 2.0 ** -8 * (want.abs() + v.abs().amax(2, keepdim=True)) + 2.0 ** -14
    assert bool(((O.double() - want).abs() <= room).all())
    assert torch.isfinite(lse).all() and all(torch.isfinite(t).all() for t in g)
    # dV = P^T dO, within P's rounding and the result's
    P = torch.zeros((1, 4, 70, 90), dtype=torch.float64, device="cuda")
    P[..., 17] = 1.0
    P = P if scale > 1 else torch.full_like(P, 1 / 90)
    d = torch.zeros(V.shape, dtype=torch.float64, device="cuda")
    e = torch.zeros_like(d)
    for h in range(4):
        d[0, h // 2] += torch.mm(P[0, h].t().contiguous(), dO[0, h].double())
        e[0, h // 2] += torch.mm(P[0, h].t().contiguous(), dO[0, h].double().abs())
    assert bool(((g[2].double() - d).abs() <= (2.0 ** -8 + 2.0 ** -14) * (d.abs() + e) + 2.0 ** -14).all())


def test_offsets_past_32_bits():
    # a cache whose second sequence, and whose last rows, lie more than 2^31 elements in
    gap = 2 ** 31 + 64
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 24 GiB of device memory")
    S, D = 300, 64
    # rows 2^23 + 8 elements apart (by 16-byte loads through registers), sequences `gap`
    big = torch.empty(gap + 512 * 2 ** 14, dtype=BF, device="cuda")
    wide = torch.empty(S * (2 ** 23 + 8), dtype=BF, device="cuda")
    Q, dO = rn((2, 4, S, D), 81), rn((2, 4, S, D), 82)
    K0, V0 = rn((2, 2, S, D), 83), rn((2, 2, S, D), 84)
    K = big.as_strided((2, 2, S, D), (gap, S * D, D, 1))
    V = big.as_strided((2, 2, S, D), (gap, S * D, D, 1), 2 * S * D)
    K.copy_(K0)
    V.copy_(V0)
    say("offsets: sequences")
    O, lse = attention.core_fwd(Q, K, V, causal=True)
    g = attention.core_bwd(dO, Q, K, V, O, lse, causal=True)
    O0, lse0 = attention.core_fwd(Q, K0, V0, causal=True)
    g0 = attention.core_bwd(dO, Q, K0, V0, O0, lse0, causal=True)
    torch.cuda.synchronize()
    assert torch.equal(O, O0) and torch.equal(lse, lse0)
    assert all(torch.equal(a, b) for a, b in zip(g, g0))
    K = wide.as_strided((1, 2, S, D), (0, D, 2 ** 23 + 8, 1))
    V = wide.as_strided((1, 2, S, D), (0, D, 2 ** 23 + 8, 1), 2 * D)
    K.copy_(K0[:1])
    V.copy_(V0[:1])
    say("offsets: rows")
    O, lse = attention.core_fwd(Q[:1], K, V, causal=True)
    g = attention.core_bwd(dO[:1], Q[:1], K, V, O, lse, causal=True)
    torch.cuda.synchronize()
    wO, bO, wl = ref.forward(Q[:1], K0[:1], V0[:1], 0.125, True, 0, None, None)
    ref.check("O", O, wO, bO)
    for n, got, (want, bound) in zip(("dQ", "dK", "dV"), g, ref.backward(
            dO[:1], Q[:1], K0[:1], V0[:1], O, lse, 0.125, True, 0, None, None)):
        ref.check(n, got, want, bound)


@pytest.mark.parametrize("bad", [float("inf"), float("nan")], ids=["inf", "nan"])
@pytest.mark.parametrize("dims", [(2, 4, 2, 70, 90, 64), (2, 2, 1, 130, 200, 128), (1, 2, 2, 40, 4000, 64),
                                  (2, 4, 2, 70, 90, 44)], ids=["64", "128", "split", "unaligned"])
def test_rows_without_keys_beside_values_that_are_not_finite(dims, bad):
    # rows past their sequence's length, and rows that the mask leaves nothing, have zero
    # results whatever the keys and values inside the lengths hold; accumulated gradients stay
    B, H, Hk, sq, sk, D = dims
    Q, K, V, dO = tensors(*dims, 140)
    K[:, :, 2], V[:, :, 5] = bad, bad
    for nq, nk, causal, dead in ((sq - 9, sk - 30, False, slice(sq - 9, sq)),
                                 (sq - 9, sk, True, slice(sq - 9, sq)),
                                 (sq, sq - 20, True, slice(0, 20))):
        kw = dict(causal=causal, len_q=lens([nq] * B), len_k=lens([nk] * B))
        say("not finite", dims, bad, nq, nk, causal)
        O, lse = attention.core_fwd(Q, K, V, **kw)
        assert bool((O[:, :, dead] == 0).all()) and bool((lse[:, :, dead] == -math.inf).all())
        O0, lse0 = attention.core_fwd(Q, torch.zeros_like(K), torch.zeros_like(V), **kw)
        dQ, dK, dV = attention.core_bwd(dO, Q, K, V, O0, lse0, **kw)
        assert bool((dQ[:, :, dead] == 0).all())
        assert bool((dK[:, :, nk:] == 0).all()) and bool((dV[:, :, nk:] == 0).all())
        old = [rn(t.shape, 150 + i, F32) for i, t in enumerate((Q, K, V))]
        out = [t.clone() for t in old]
        attention.core_bwd(dO, Q, K, V, O0, lse0, out=out, accumulate=True, **kw)
        assert torch.equal(out[0][:, :, dead], old[0][:, :, dead])
        assert all(torch.equal(a[:, :, nk:], b[:, :, nk:]) for a, b in zip(out[1:], old[1:]))


def peaked(dims, peak, ties, seed, pad=0):
    """Scores that are exact: `peak` for the keys of `ties`, 0 for the others (scale 1)."""
    B, H, Hk, sq, sk, D = dims
    Q, K = (torch.zeros((B, h, s, D + pad), dtype=BF, device="cuda")[..., :D] for h, s in ((H, sq), (Hk, sk)))
    Q[..., 0] = 1.0
    K[:, :, ties, 0] = peak
    return Q, K, rn((B, Hk, sk, D + pad), seed)[..., :D], rn((B, H, sq, D), seed + 1)


@pytest.mark.parametrize("scale", [2.0 ** 10, 2.0 ** 20, 2.0 ** 30, 1e9, 2.0 ** 40, 2.0 ** 100])
@pytest.mark.parametrize("dims,pad", [((1, 4, 2, 70, 90, 64), 0), ((2, 2, 2, 300, 500, 128), 0),
                                      ((1, 2, 2, 70, 90, 40), 3)], ids=["64", "128", "unaligned"])
def test_maxima_of_any_size(dims, pad, scale):
    # the largest score far beyond 2^24: its weight is still one against itself. Three keys
    # share it, each with a third
    ties = [17, 40, 61]
    for peak in (3.0, 5.6875, -5.6875):
        Q, K, V, _ = peaked(dims, peak, ties, 160, pad)
        if peak < 0:          # every key but those three
            ties = [j for j in range(dims[4]) if j not in ties]
        say("maxima", dims, peak, scale)
        O, lse = attention.core_fwd(Q, K, V, scale=scale, out_dtype=F32)
        v = V.double().repeat_interleave(dims[1] // dims[2], 1)[:, :, ties]
        want = v.mean(2, keepdim=True)
        # weights of equal size, exact as operands: sums and a division in fp32
        assert bool(((O.double() - want).abs() <= ref.F * v.abs().mean(2, keepdim=True)).all())
        # one rounding of a sum of the largest score and a logarithm
        top = max(peak, 0.0) * scale
        far = (lse.double() - (top + math.log(len(ties)))).abs()
        assert float(far.max()) <= 2.0 ** -23 * top + 2.0 ** -20, float(far.max())


def test_large_queries_and_keys():
    # the same from large Q and K at an ordinary scale: scores of 3 2^34 D
    Q, K, V, _ = peaked((1, 4, 2, 70, 90, 64), 1.0, [17, 40, 61], 165)
    Q[:] = 2.0 ** 17
    K[:] = torch.where(K[..., :1] > 0, 3.0 * 2 ** 17, 2.0 ** 17)
    say("large Q and K")
    O, lse = attention.core_fwd(Q, K, V, scale=0.125, out_dtype=F32)
    v = V.double().repeat_interleave(2, 1)[:, :, [17, 40, 61]]
    assert bool(((O.double() - v.mean(2, keepdim=True)).abs() <= ref.F * v.abs().mean(2, keepdim=True)).all())
    top = 3.0 * 2 ** 34 * 64 * 0.125
    assert float((lse.double() - top).abs().max()) <= 2.0 ** -23 * top


@pytest.mark.parametrize("scale", [1.0, 2.0 ** 20, 2.0 ** 30, 1e9, 2.0 ** 100])
@pytest.mark.parametrize("dims", [(1, 8, 2, 3, 3000, 64), (1, 2, 2, 1, 4096, 128), (1, 1, 1, 40, 3000, 44)],
                         ids=["64", "128", "unaligned"])
def test_maxima_of_any_size_over_splits(dims, scale):
    # the largest score once in the first split of the keys, three times in the last one: each
    # of the four has a quarter, however small log 3 is beside it
    ties = [40, dims[4] - 60, dims[4] - 31, dims[4] - 9]
    for peak in (100.0, 181.0):
        Q, K, V, _ = peaked(dims, peak, ties, 170)
        say("maxima over splits", dims, peak, scale)
        sbp.sbp_profile_begin(8)
        O, lse = attention.core_fwd(Q, K, V, scale=scale, out_dtype=F32)
        assert any("join" in n for n, _ in sbp.sbp_profile_end(8))
        v = V.double().repeat_interleave(dims[1] // dims[2], 1)[:, :, ties]
        want = v.mean(2, keepdim=True)
        assert bool(((O.double() - want).abs() <= ref.F * v.abs().mean(2, keepdim=True)).all())
        far = (lse.double() - (peak * scale + math.log(4))).abs()
        assert float(far.max()) <= 2.0 ** -23 * peak * scale + 2.0 ** -20, float(far.max())


@pytest.mark.parametrize("scale", [2.0 ** 6, 1e3, 2.0 ** 10, 2.0 ** 14])
@pytest.mark.parametrize("dims", [(1, 4, 2, 70, 90, 64), (2, 2, 2, 300, 500, 128)], ids=["64", "128"])
def test_gradients_at_large_scores(dims, scale):
    # P from an fp32 lse is off by a factor of up to exp(2^-22 |lse|) = 1 + R; what follows from
    # it as in ref.backward's bounds
    B, H, Hk, sq, sk, D = dims
    ties = [17, 40, 61]
    for peak in (3.0, 5.6875):
        Q, K, V, dO = peaked(dims, peak, ties, 180)
        say("gradients at large scores", dims, peak, scale)
        O, lse = attention.core_fwd(Q, K, V, scale=scale)
        g = attention.core_bwd(dO, Q, K, V, O, lse, scale=scale, grad_dtype=F32)
        R = math.expm1(2.0 ** -22 * float(lse.max()))
        P = torch.zeros((sq, sk), dtype=torch.float64, device="cuda")
        P[:, ties] = 1 / 3
        want = [torch.zeros(t.shape, dtype=torch.float64, device="cuda") for t in (Q, K, V)]
        room = [torch.zeros_like(t) for t in want]
        mm = lambda a, b: torch.mm(a.contiguous(), b.contiguous())
        for b in range(B):
            for h in range(H):
                c = h * Hk // H
                q, k, v, do, o = (t.double() for t in (Q[b, h], K[b, c], V[b, c], dO[b, h], O[b, h]))
                D_ = (do * o).sum(1, keepdim=True)
                dS = P * (mm(do, v.t()) - D_)
                e = ref.U * dS.abs() + (R + ref.F) * P * (mm(do.abs(), v.abs().t()) +
                                                          (do * o).abs().sum(1, keepdim=True))
                for i, x in enumerate((scale * mm(dS, k), scale * mm(dS.t(), q), mm(P.t(), do))):
                    want[i][b, (h, c, c)[i]] += x
                for i, x in enumerate((scale * mm(e, k.abs()), scale * mm(e.t(), q.abs()),
                                       (R + ref.U + ref.F) * mm(P.t(), do.abs()))):
                    room[i][b, (h, c, c)[i]] += x
        for n, got, w, r in zip(("dQ", "dK", "dV"), g, want, room):
            ref.check(n, got, w, r)


def test_most_heads():
    # 2^23 key heads of one row without keys: as many workgroups of 256 threads, and no form of
    # 512 threads, fit one launch
    n, D = 1 << 23, 72
    if torch.cuda.mem_get_info()[0] < 8 << 30:
        pytest.skip("needs 8 GiB of device memory")
    Q = torch.ones((n, 1, 1, D), dtype=BF, device="cuda")
    K = torch.empty((n, 1, 0, D), dtype=BF, device="cuda")
    say("most heads")
    O, lse = attention.core_fwd(Q, K, K)
    torch.cuda.synchronize()
    assert int(torch.count_nonzero(O)) == 0 and bool((lse == -math.inf).all())
