"""Rotary positions, the paged cache and attention over it together, as a layer uses them: in
training (rotation, attention, and both backward, against 64 bits and as a captured graph), and in
serving (prompts in chunks and single tokens through a column-split projection, append and
attention, on every device of a tensor-parallel group, against the whole sequences at once)."""
import math

import pytest
import torch

import attn_core_ref as ref
import paged_ref as pref
import rope_ref
from paper_2301_06813_amd import attention, inputs, linear, paged, rotary, sbp

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def rn(shape, seed, std=1.0):
    return inputs.randn(shape, std, seed, BF, "cuda")


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("order", ["halves", "pairs"])
def test_training(order):
    """Rotated Q and K into attention and back: each stage against 64 bits from the operands that
    it was given, eagerly and from a graph."""
    B, H, Hk, S, D, rot = 2, 4, 2, 70, 64, 48
    act = rn((B, S, H + 2 * Hk, D), 1).permute(0, 2, 1, 3)
    Q, K, V = act[:, :H], act[:, H:H + Hk], act[:, H + Hk:]
    dO = rn((B, S, H, D), 2).permute(0, 2, 1, 3)
    rope, f, s = rotary.Rope(rot, order=order), rope_ref.freqs(rot), 1 / math.sqrt(D)
    pos = torch.arange(S).expand(B, S)

    def step():
        q, k = rotary.fwd(rope, Q, K)
        O, lse = attention.core_fwd(q, k, V, scale=s, causal=True)
        dq, dk, dv = attention.core_bwd(dO, q, k, V, O, lse, scale=s, causal=True)
        dQ, dK = rotary.bwd(rope, dq, dk)
        return q, k, O, lse, dq, dk, dv, dQ, dK

    q, k, O, lse, dq, dk, dv, dQ, dK = eager = step()
    for n, x, y, back in (("q", Q, q, False), ("k", K, k, False), ("dQ", dq, dQ, True), ("dK", dk, dK, True)):
        rope_ref.check(n, y, *rope_ref.rotate(x.cpu(), pos, f, rot, order, back=back))
    ref.check("O", O, *ref.forward(q, k, V, s, True, 0, None, None)[:2])
    for n, got, (want, bound) in zip(("dq", "dk", "dv"), (dq, dk, dv),
                                     ref.backward(dO, q, k, V, O, lse, s, True, 0, None, None)):
        ref.check(n, got, want, bound)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = step()
    for _ in range(3):
        for t in out:
            t.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, eager))


def test_gradient_through_attention_against_differences():
    """The chain's gradient for Q along a direction e, against (L(Q + h e) - L(Q - h e)) / 2 h of the
    64-bit chain, L = <dO, O>: the library's bf16 q, O and dq carry 2^-8 each, and sums of 64 x
    terms that hardly cancel, so a thirtieth of the gradient's size along e."""
    B, H, S, D = 1, 1, 40, 32
    Q, K, V, dO = (rn((B, H, S, D), 3 + i) for i in range(4))
    rope, f, s = rotary.Rope(D), rope_ref.freqs(D), 1 / math.sqrt(D)
    pos = torch.arange(S).expand(B, S)
    q, k = rotary.fwd(rope, Q, K)
    O, lse = attention.core_fwd(q, k, V, scale=s, causal=True)
    dq, dk, _ = attention.core_bwd(dO, q, k, V, O, lse, scale=s, causal=True)
    dQ, dK = rotary.bwd(rope, dq, dk)

    def loss(Q, K):
        q, _ = rope_ref.rotate(Q, pos, f, D, "halves")
        k, _ = rope_ref.rotate(K, pos, f, D, "halves")
        x = (q @ k.transpose(2, 3)) * s
        x = x.masked_fill(torch.triu(torch.ones(S, S, dtype=torch.bool), 1), -math.inf)
        return float((torch.softmax(x, -1) @ V.double().cpu() * dO.double().cpu()).sum())

    Qd, Kd, h = Q.double().cpu(), K.double().cpu(), 1e-4
    for seed, got, at in ((1, dQ, 0), (2, dK, 1)):
        e = torch.randn(Q.shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64)
        e = torch.where(got.double().cpu() >= 0, e.abs(), -e.abs())   # along the gradient: no cancelling
        up, down = [(Qd + z * e, Kd) if at == 0 else (Qd, Kd + z * e) for z in (h, -h)]
        want = (loss(*up) - loss(*down)) / (2 * h)
        have = float((got.double().cpu() * e).sum())
        assert abs(have - want) <= abs(want) / 30, (have, want)


class Layer:
    """A device's attention share: column-split projection of Q, K and V, its own cache."""

    def __init__(self, p, r, W, H, Hk, D, pages, P):
        self.p, self.r, self.W, self.D = p, r, W, D
        self.h, self.hk = H // p, Hk // p
        mem = torch.full((pages, 2, P, self.hk, D), math.nan, dtype=BF, device="cuda")
        self.cache = paged.Cache(*(mem[:, i].permute(0, 2, 1, 3) for i in range(2)), sbp.SBP_LOCAL)

    def heads(self, x):
        """Q, K and V of rows x, [1][heads][rows][D] each."""
        out = []
        for w, n in zip(self.W, (self.h, self.hk, self.hk)):
            y = linear.call("fwd", "COL", self.p, self.r, x, w, None)[0]
            out.append(y.view(1, -1, n, self.D).transpose(1, 2))
        return out

    def step(self, x, rope, table, len_k, row_q):
        q, k, v = self.heads(x)
        q = self.cache.append(k, v, table, len_k, Q=q, rope=rope, row_q=row_q, out=q,
                              scope=sbp.SBP_LOCAL)
        return self.cache.attend(q, table, len_k, row_q=row_q)[0]


@pytest.mark.parametrize("p", [1, 2])
@pytest.mark.parametrize("D,P", [(64, 16), (80, 10)])
def test_serving(p, D, P):
    """Three sequences: prompts of 50, 1 and 130 tokens in chunks of up to 48, then 5 tokens each,
    the short ones' tokens beside the long one's chunks. Every step's rows against the whole
    sequence at once: the same projections bit for bit, rotated by the library's other call
    (the same bits), and attention in 64 bits."""
    H, Hk, dm, total = 8, 2, 96, [55, 6, 135]
    W = [rn((dm, n * D), 10 + i, dm ** -0.5) for i, n in enumerate((H, Hk, Hk))]
    xs = [rn((n, dm), 20 + i) for i, n in enumerate(total)]
    rope = rotary.Rope(D, scaling="turns", factor=4.0, context=64.0, low=1.0, high=4.0)
    width = (max(total) + P - 1) // P
    perm = torch.randperm(3 * width + 2, generator=torch.Generator().manual_seed(5))[:3 * width]
    table = perm.view(3, width).to(torch.int32).cuda()
    # rows of each sequence's steps
    prompt, plan, done = [50, 1, 130], [], [0, 0, 0]
    while done != total:
        new = [min(48, q - d) if d < q else min(1, n - d) for d, q, n in zip(done, prompt, total)]
        plan.append(new)
        done = [d + n for d, n in zip(done, new)]
    assert len(plan) >= 6 and any(0 in new for new in plan)
    for r in range(p):
        layer = Layer(p, r, W, H, Hk, D, 3 * width + 2, P)
        got, done = [[], [], []], [0, 0, 0]
        for new in plan:
            x = torch.cat([x[d:d + n] for x, d, n in zip(xs, done, new)])
            done = [d + n for d, n in zip(done, new)]
            row_q = [0]
            for n in new:
                row_q.append(row_q[-1] + n)
            O = layer.step(x, rope, table, i32(done), i32(row_q))
            for b in range(3):
                got[b].append(O[:, :, row_q[b]:row_q[b + 1]].clone())
        for b in range(3):
            q, k, v = layer.heads(xs[b])
            q, k = rotary.fwd(rope, q, k, scope=sbp.SBP_LOCAL)
            want, bound, _ = ref.forward(q, k, v, 1 / math.sqrt(D), True, 0, None, None)
            O = torch.cat(got[b], 2)
            assert O.shape[2] == total[b]
            # products of other row counts may sum in another order: bf16 rows of q, k and v may
            # differ by a step where that falls on a border, 2^-7 of a score's and a value's terms
            s = 1 / math.sqrt(D)
            group = H // Hk
            ka, va = (t.abs().double().repeat_interleave(group, 1) for t in (k, v))
            terms = (q.abs().double() @ ka.transpose(2, 3)).amax(-1, keepdim=True) * s
            bound = bound + 2.0 ** -7 * (2 * terms + 1) * va.amax(2, keepdim=True)
            ref.check("O", O, want, bound)


def test_decoding_graph():
    """Append and attention of single tokens captured once and replayed as the sequences grow, with
    eager work between; another graph over the same workspace and cache beside it."""
    B, H, Hk, D, P, width = 4, 8, 2, 64, 16, 6
    kc, vc = rn((B * width, P, Hk, D), 1).permute(0, 2, 1, 3), rn((B * width, P, Hk, D), 2).permute(0, 2, 1, 3)
    keep = kc.clone(), vc.clone()
    table = torch.randperm(B * width, generator=torch.Generator().manual_seed(1)).view(B, width).to(torch.int32).cuda()
    lens = i32([16, 1, 40, 63])
    rope, act = rotary.Rope(D), rn((B, 1, H + 2 * Hk, D), 3)

    def step(cache, act, ws=None):
        x = act.permute(0, 2, 1, 3)
        q = cache.append(x[:, H:H + Hk], x[:, H + Hk:], table, lens, Q=x[:, :H], rope=rope)
        return cache.attend(q, table, lens, ws=ws)

    cache, ws = paged.Cache(kc, vc), torch.empty(1 << 21, dtype=torch.uint8, device="cuda")
    g, other = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = step(cache, act, ws)
    with torch.cuda.graph(other):
        again = cache.attend(act.permute(0, 2, 1, 3)[:, :H], table, lens, ws=ws)
    plain = paged.Cache(*keep)
    for t in range(4):
        act.copy_(rn(act.shape, 30 + t))
        lens.add_(1)
        g.replay()
        other.replay()
        want = step(plain, act, torch.empty(1 << 21, dtype=torch.uint8, device="cuda"))
        check = plain.attend(act.permute(0, 2, 1, 3)[:, :H], table, lens,
                             ws=torch.empty(1 << 21, dtype=torch.uint8, device="cuda"))
        torch.cuda.synchronize()
        assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])
        assert torch.equal(again[0], check[0]) and torch.equal(again[1], check[1])
        assert torch.equal(kc, keep[0]) and torch.equal(vc, keep[1])


@pytest.mark.parametrize("p", [1, 2])
@pytest.mark.parametrize("D,P", [(64, 16), (80, 10)])
def test_serving_steps_against_their_operands(p, D, P):
    """Every operator of test_serving's steps against 64 bits from the operands it was given, with no
    slack between them: projections as far from the whole sequence's as two roundings to bf16 and
    two orders of an fp32 sum, rotations, cached rows, and attention over the rows that the cache
    holds by (U + F) P |V|."""
    H, Hk, dm, total = 8, 2, 96, [55, 6, 135]
    W = [rn((dm, n * D), 40 + i, dm ** -0.5) for i, n in enumerate((H, Hk, Hk))]
    xs = [rn((n, dm), 50 + i) for i, n in enumerate(total)]
    kw = dict(scaling="turns", factor=4.0, context=64.0, low=1.0, high=4.0)
    rope, f, s = rotary.Rope(D, **kw), rope_ref.freqs(D, **kw), 1 / math.sqrt(D)
    width = (max(total) + P - 1) // P
    perm = torch.randperm(3 * width + 2, generator=torch.Generator().manual_seed(6))[:3 * width]
    host_table = perm.view(3, width).tolist()
    table, prompt = i32(host_table), [50, 1, 130]
    for r in range(p):
        layer, done = Layer(p, r, W, H, Hk, D, 3 * width + 2, P), [0, 0, 0]
        kc, vc = layer.cache.k, layer.cache.v
        whole = [layer.heads(x) for x in xs]
        sums = [[(x.abs().double() @ w[:, r * w.shape[1] // p:(r + 1) * w.shape[1] // p].abs().double())
                 .view(1, x.shape[0], -1, D).transpose(1, 2) for w in W] for x in xs]
        while done != total:
            new = [min(48, q - d) if d < q else min(1, n - d) for d, q, n in zip(done, prompt, total)]
            x = torch.cat([x[d:d + n] for x, d, n in zip(xs, done, new)])
            before, done = done, [d + n for d, n in zip(done, new)]
            row_q = [sum(new[:b]) for b in range(4)]
            seqs = pref.lengths(3, row_q[-1], None, row_q)
            q, k, v = layer.heads(x)
            for b, (_, first, n) in enumerate(seqs):
                for got, full, size in zip((q, k, v), whole[b], sums[b]):
                    rows, cols = slice(first, first + n), slice(before[b], done[b])
                    want = full[:, :, cols].double()
                    off = (got[:, :, rows].double() - want).abs()
                    lim = 2 * pref.U * want.abs() + 2 * dm * 2.0 ** -24 * (1 + 2 * pref.U) * size[:, :, cols]
                    # (the second rounding is of the first one's value)
                    assert bool((off <= lim * (1 + 2 * pref.U)).all())
            pos = torch.cat([torch.arange(a, e) for a, e in zip(before, done)])[None]
            wq, bq = rope_ref.rotate(q.cpu(), pos, f, D, "halves")
            wk, bk = rope_ref.rotate(k.cpu(), pos, f, D, "halves")
            q = layer.cache.append(k, v, table, i32(done), Q=q, rope=rope, row_q=i32(row_q), out=q,
                                   scope=sbp.SBP_LOCAL)
            rope_ref.check("q", q, wq, bq)
            for _, i, page, slot, t in pref.places(seqs, done, host_table, kc.shape[0], P):
                rope_ref.check("k", kc[page, :, slot], wk[0, :, i], bk[0, :, i])
                assert torch.equal(vc[page, :, slot], v[0, :, i])
            O, lse = layer.cache.attend(q, table, i32(done), row_q=i32(row_q))
            want, bound, wl, used = pref.attend(q, kc, vc, host_table, done, seqs, s, True, 0)
            assert bool(used.all())
            pref.check("O", O, want, bound)
            # scores below 2^5 in fp32, one logarithm
            assert float((lse.double() - wl).abs().max()) <= 2.0 ** -14
