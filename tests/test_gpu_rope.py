"""GPU tests of rotary positions against 64 bits (rope_ref.py derives the bounds): both orders,
parts of a head, every scaling, types, odd sizes, strides, places from none to 2^31, head
splits, in place, the gradient against the formula and against differences, streams and graphs."""
import pytest
import torch

import rope_ref as ref
from paper_2301_06813_amd import rotary, sbp
from paper_2301_06813_amd.attention import rank_heads

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def rn(shape, seed, dtype=BF):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def fused(B, S, H, Hk, D, seed, dtype=BF):
    act = rn((B, S, H + 2 * Hk, D), seed, dtype).permute(0, 2, 1, 3)
    return act[:, :H], act[:, H:H + Hk]


def grid(pos, B, S):
    """Positions [B][S] on the host."""
    i = torch.arange(S)[None, :].expand(B, S)
    if pos is None:
        return i
    pos = pos.cpu().long()
    return pos[:, None] + i if pos.dim() == 1 else pos


# B, S, H, Hk, D, rotated columns
SHAPES = [(1, 1, 1, 1, 2, 2), (16, 1, 16, 4, 64, 64), (2, 37, 3, 1, 128, 128), (3, 5, 6, 2, 80, 40),
          (2, 65, 4, 4, 64, 48), (1, 130, 7, 7, 96, 96), (2, 9, 2, 1, 33, 6), (1, 3, 2, 2, 111, 110),
          (5, 333, 6, 2, 80, 80), (1, 1, 70, 10, 128, 64), (1, 7, 4, 2, 1, 0), (2, 17, 2, 2, 20, 20)]


@pytest.mark.parametrize("order", ["halves", "pairs"])
@pytest.mark.parametrize("types", [(BF, BF), (BF, F32), (F32, F32)], ids=["bf", "bf-f", "f"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_both_directions(shape, types, order):
    B, S, H, Hk, D, rot = shape
    if rot == 0:
        pytest.skip("a head of one column has no pair")
    Q, K = fused(B, S, H, Hk, D, 3, types[0])
    rope = rotary.Rope(rot, order=order)
    f = ref.freqs(rot)
    first = torch.randint(0, 5000, (B,), dtype=torch.int32, device="cuda")
    rows = torch.randint(-100, 100000, (B, S), dtype=torch.int32, device="cuda")
    for pos in (None, first, rows):
        for call, back in ((rotary.fwd, False), (rotary.bwd, True)):
            got = call(rope, Q, K, pos=pos, out_dtype=types[1])
            for n, x, y in zip("QK", (Q, K), got):
                assert y.dtype == types[1] and y.shape == x.shape
                ref.check(n, y, *ref.rotate(x.cpu(), grid(pos, B, S), f, rot, order, back=back))
                # columns past the rotated ones are copied
                assert torch.equal(y[..., rot:], x[..., rot:].to(types[1]))


@pytest.mark.parametrize("scaling", [None, "linear", "base", "turns", "pairs"])
def test_scalings_and_factor_at_far_places(scaling):
    kw = dict(scaling=scaling, factor=8.0, low=1.0, high=32.0, context=4096.0, base=500000.0)
    rope = rotary.Rope(64, mul=1.25, **kw)
    f = ref.freqs(64, **kw)
    Q, K = fused(2, 40, 4, 2, 64, 5, F32)
    pos = torch.tensor([[0, 1, 2, 4095, 4096, 1 << 20, (1 << 20) + 1, 123456789] * 5,
                        [-1, -7, (1 << 31) - 1, -(1 << 31), 1 << 30, 7, 999999999, -5] * 5],
                       dtype=torch.int32, device="cuda")
    for y, x in zip(rotary.fwd(rope, Q, K, pos=pos), (Q, K)):
        ref.check("far", y, *ref.rotate(x.cpu(), grid(pos, 2, 40), f, 64, "halves", mul=1.25))
    # a first place from which rows pass 2^31
    first = torch.tensor([(1 << 31) - 3, -5], dtype=torch.int32, device="cuda")
    for y, x in zip(rotary.fwd(rope, Q, K, pos=first), (Q, K)):
        ref.check("past 2^31", y, *ref.rotate(x.cpu(), grid(first, 2, 40), f, 64, "halves", mul=1.25))


def test_gradient_against_differences():
    """<dY, R (x + h e) - R (x - h e)> / 2 h is the gradient's element: R is linear, so this holds
    up to rounding for any h; in fp32 with h = 1."""
    rope = rotary.Rope(12, order="pairs", mul=1.5)
    x, dy = rn((1, 2, 3, 16), 7, F32), rn((1, 2, 3, 16), 8, F32)
    pos = torch.tensor([[5, 1000, 77]], dtype=torch.int32, device="cuda")
    dx, _ = rotary.bwd(rope, dy, pos=pos)
    for h, i, col in ((0, 0, 0), (0, 1, 5), (1, 2, 11), (1, 0, 12), (1, 2, 15)):
        e = torch.zeros_like(x)
        e[0, h, i, col] = 1.0
        up, _ = rotary.fwd(rope, x + e, pos=pos)
        down, _ = rotary.fwd(rope, x - e, pos=pos)
        want = float((dy.double() * (up.double() - down.double())).sum()) / 2
        # two outputs a side that differ, each off by 2^-21 1.5 (|x1| + |x2| + 1) and 2^-24 of itself
        bound = float(dy.abs().max()) * 4 * (2.0 ** -21 * 1.5 * (2 * float(x.abs().max()) + 1) + 2.0 ** -22 * 8)
        assert abs(float(dx[0, h, i, col]) - want) <= bound


def test_turned_there_and_back():
    """bwd of fwd is mul^2 x: what training relies on, in fp32 bounds of both passes."""
    rope = rotary.Rope(64, mul=0.5)
    x = rn((2, 3, 50, 64), 9, F32)
    pos = torch.tensor([123456, 1 << 30], dtype=torch.int32, device="cuda")
    y, _ = rotary.fwd(rope, x, pos=pos)
    z, _ = rotary.bwd(rope, y, pos=pos)
    size = x.abs() + x.roll(32, -1).abs()
    assert float((z - 0.25 * x).abs().sub(2.0 ** -20 * size).max()) <= 0


@pytest.mark.parametrize("p", [2, 3, 8])
def test_head_split(p):
    """Rank r's heads, of global and of local views, are slices of the whole result."""
    Q, K = fused(2, 21, 15, 5, 48, 11)
    rope = rotary.Rope(48)
    wq, wk = rotary.fwd(rope, Q, K)
    for r in range(p):
        h0, h, k0, hk = rank_heads(15, 5, p, r)
        for scope in (sbp.SBP_GLOBAL, sbp.SBP_LOCAL):
            q, k = (Q, K) if scope == sbp.SBP_GLOBAL else (Q[:, h0:h0 + h], K[:, k0:k0 + hk])
            gq, gk = rotary.fwd(rope, q, k, p, r, scope=scope)
            assert torch.equal(gq, wq[:, h0:h0 + h]) and torch.equal(gk, wk[:, k0:k0 + hk])


@pytest.mark.parametrize("order", ["halves", "pairs"])
@pytest.mark.parametrize("layout", ["rows", "heads"])
def test_in_place(layout, order):
    """Q and K parts of one activation, rotated where they are; V's part stays."""
    H, Hk, D, S, B = 6, 2, 72, 19, 3
    act = rn((B, S, H + 2 * Hk, D) if layout == "rows" else (B, H + 2 * Hk, S, D), 13)
    x = act.permute(0, 2, 1, 3) if layout == "rows" else act
    rope = rotary.Rope(56, order=order)
    want = rotary.fwd(rope, x[:, :H], x[:, H:H + Hk])
    v = x[:, H + Hk:].clone()
    rotary.fwd(rope, x[:, :H], x[:, H:H + Hk], out=(x[:, :H], x[:, H:H + Hk]))
    assert torch.equal(x[:, :H], want[0]) and torch.equal(x[:, H:H + Hk], want[1])
    assert torch.equal(x[:, H + Hk:], v)
    # the rank's part of Q and K
    y = want[0].clone()
    rotary.fwd(rope, y, None, 2, 1, out=(y[:, 3:], None))
    assert torch.equal(y[:, :3], want[0][:, :3])
    assert torch.equal(y[:, 3:], rotary.fwd(rope, want[0])[0][:, 3:])


def test_unaligned_rows_and_strides():
    """Rows at odd elements and with odd strides; surroundings stay."""
    B, H, S, D = 2, 3, 11, 50
    for dt in (BF, F32):
        buf = rn((B, H, S, D + 3), 15, dt)
        x = buf[..., 1:1 + D]
        out = torch.full((B, H, S, D + 5), 7.0, dtype=dt, device="cuda")
        rope = rotary.Rope(34, order="halves")
        rotary.fwd(rope, x, out=(out[..., 3:3 + D], None))
        ref.check("odd", out[..., 3:3 + D], *ref.rotate(x.cpu(), grid(None, B, S), ref.freqs(34), 34,
                                                        "halves"))
        assert float((out[..., :3] - 7).abs().max()) == 0 and float((out[..., 3 + D:] - 7).abs().max()) == 0


def test_offsets_past_32_bits():
    """Batches whose strides pass 2^31 elements."""
    big = torch.empty((1 << 31) + 4096, dtype=BF, device="cuda")
    x = big.as_strided((2, 2, 3, 64), (1 << 31, 64, 128, 1))
    x.copy_(rn((2, 2, 3, 64), 17))
    small = x.clone()
    rope = rotary.Rope(64)
    want = rotary.fwd(rope, small)[0]
    assert torch.equal(rotary.fwd(rope, x)[0], want)
    rotary.fwd(rope, x, out=(x, None))
    assert torch.equal(x, want)


def test_not_finite_values_stay_in_their_pairs():
    rope = rotary.Rope(8, order="halves")
    x = torch.zeros((1, 1, 4, 12), device="cuda")
    x[0, 0, 1, 2] = float("nan")
    x[0, 0, 2, 9] = float("inf")
    y = rotary.fwd(rope, x)[0]
    bad = ~torch.isfinite(y[0, 0])
    want = torch.zeros((4, 12), dtype=torch.bool)
    want[1, 2] = want[1, 6] = want[2, 9] = True
    assert torch.equal(bad.cpu(), want)


def test_given_stream_and_graph():
    Q, K = fused(4, 33, 8, 2, 64, 19)
    rope = rotary.Rope(64)
    pos = torch.tensor([0, 5, 9, 100], dtype=torch.int32, device="cuda")
    want = rotary.fwd(rope, Q, K, pos=pos)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = rotary.fwd(rope, Q, K, pos=pos, stream=side.cuda_stream)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = rotary.fwd(rope, Q, K, pos=pos)
        back = rotary.bwd(rope, *out, pos=pos, out_dtype=F32)
    for step in range(3):
        pos.add_(1)           # places are read when the graph runs
        g.replay()
        want = rotary.fwd(rope, Q, K, pos=pos)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))
        assert all(torch.equal(a, b) for a, b in zip(back, rotary.bwd(rope, *want, pos=pos, out_dtype=F32)))


def test_refused_from_torch():
    Q, K = fused(2, 3, 4, 2, 16, 21)
    rope = rotary.Rope(16)
    with pytest.raises(ValueError):
        rotary.fwd(rope, Q, K, pos=torch.zeros(2, dtype=torch.int64, device="cuda"))
    with pytest.raises(ValueError):
        rotary.fwd(rope, Q, K, pos=torch.zeros((2, 4), dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError):
        rotary.fwd(rope, Q.cpu(), K)
    with pytest.raises(sbp.SbpError) as e:
        rotary.fwd(rotary.Rope(18), Q, K)
    assert e.value.code == sbp.SBP_ERR_SHAPE


def test_positions_with_any_strides():
    """Positions shared by all sequences (a stride of 0), and a column of a wider tensor."""
    Q, K = fused(3, 20, 4, 2, 64, 23)
    rope = rotary.Rope(64)
    row = torch.randint(0, 9000, (20,), dtype=torch.int32, device="cuda")
    want = rotary.fwd(rope, Q, K, pos=row.expand(3, 20).contiguous())
    got = rotary.fwd(rope, Q, K, pos=row.expand(3, 20))
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    wide = torch.randint(0, 9000, (3, 7), dtype=torch.int32, device="cuda")
    want = rotary.fwd(rope, Q, K, pos=wide[:, 4].contiguous())
    got = rotary.fwd(rope, Q, K, pos=wide[:, 4])
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_copied_columns_keep_their_bits():
    g = torch.Generator(device="cuda").manual_seed(25)
    x = torch.randint(-(1 << 15), 1 << 15, (2, 3, 5, 40), generator=g, device="cuda", dtype=torch.int16)
    x[..., ::3] |= 0x7f80
    y, _ = rotary.fwd(rotary.Rope(12), x.view(BF))
    assert torch.equal(y[..., 12:].contiguous().view(torch.int16), x[..., 12:])
