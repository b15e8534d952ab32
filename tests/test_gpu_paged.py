"""GPU tests of the paged cache against plain forms (paged_ref.py): appending with and without
rotation, attention of chunks and of single tokens; padded and packed rows; lengths from none
to long, pages that end inside a tile, bad pages, freed pages before a window, what is not finite
where nobody looks, strides, offsets past 32 bits, head splits, workspaces, streams, graphs."""
import math

import pytest
import torch

import paged_ref as pref
import rope_ref
from paper_2301_06813_amd import paged, rotary, sbp
from paper_2301_06813_amd.attention import rank_heads

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def rn(shape, seed, dtype=BF):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def i32(v):
    return None if v is None else torch.tensor(v, dtype=torch.int32, device="cuda")


def pool(pages, Hk, P, D, seed, layout="token"):
    """Keys and values [pages][Hk][P][D] of one of the memory layouts."""
    if layout == "token":
        return [rn((pages, P, Hk, D), seed + i).permute(0, 2, 1, 3) for i in range(2)]
    if layout == "head":
        return [rn((pages, Hk, P, D), seed + i) for i in range(2)]
    if layout == "both":        # keys and values of a page side by side
        t = rn((pages, 2, P, Hk, D), seed)
        return [t[:, i].permute(0, 2, 1, 3) for i in range(2)]
    if layout == "odd":         # rows at odd elements, odd strides
        return [rn((pages, Hk, P, D + 3), seed + i)[..., 1:1 + D] for i in range(2)]
    raise ValueError(layout)


def deal_pages(n, width, spare, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randperm(n * width + spare, generator=g)[:n * width].view(n, width).tolist()


class Batch:
    """Sequences with `new` new tokens each, packed or padded."""

    def __init__(self, new, lens, heads, D, P, layout="token", packed=False, pad=0, extra=1, gap=0,
                 seed=1):
        H, Hk = heads
        n = len(new)
        self.n, self.new, self.len, self.P, self.D = n, list(new), list(lens), P, D
        width = (max(list(lens) + [1]) + P - 1) // P + extra
        self.table = deal_pages(n, width, 2, seed)
        self.kc, self.vc = pool(n * width + 2, Hk, P, D, seed + 10, layout)
        self.len_q = self.row_q = None
        if packed:
            self.row_q = [gap]
            for x in new:
                self.row_q.append(self.row_q[-1] + x)
            B, S = 1, self.row_q[-1] + pad
        else:
            B, S = n, max(list(new) + [0]) + pad
            if any(x != S for x in new):
                self.len_q = list(new)
        act = rn((B, S, H + 2 * Hk, D), seed + 20).permute(0, 2, 1, 3)
        self.Q, self.K, self.V = act[:, :H], act[:, H:H + Hk], act[:, H + Hk:]
        self.seqs = pref.lengths(n, S, self.len_q, self.row_q)
        self.cache = paged.Cache(self.kc, self.vc)

    def args(self):
        return i32(self.table), i32(self.len)

    def rows(self):
        return dict(len_q=i32(self.len_q), row_q=i32(self.row_q))


def check_attn(b, causal=True, window=0, scale=None, **kw):
    s = 1 / math.sqrt(b.D) if scale is None else scale
    O, lse = b.cache.attend(b.Q, *b.args(), scale=s, causal=causal, window=window, **b.rows(), **kw)
    torch.cuda.synchronize()
    want, bound, wl, used = pref.attend(b.Q, b.kc, b.vc, b.table, b.len, b.seqs, s, causal, window)
    live = used if b.row_q is not None else torch.ones_like(used)
    sel = live[:, None, :].expand(lse.shape)
    pref.check("O", O[sel], want[sel], bound[sel])
    empty = (wl == -math.inf) & sel
    assert torch.equal((lse == -math.inf)[sel], empty[sel])
    off = (lse.double() - wl)[sel & ~empty].abs()
    # scores below 2^5 in fp32, one logarithm: 2^-14 as in the bounds' F
    assert off.numel() == 0 or float(off.max()) <= 2.0 ** -14
    assert float(O[empty].abs().sum()) == 0.0
    return O, lse


# ---------------------------------------------------------------- attention
ATTN = [
    # new tokens, lengths, (H, Hk), D, page, packed
    ([1], [1], (1, 1), 64, 16, False),
    ([1, 1, 1], [1, 17, 300], (8, 2), 64, 16, False),
    ([1] * 5, [31, 32, 33, 127, 129], (4, 4), 128, 16, False),
    ([1] * 3, [1000, 65, 2049], (14, 2), 80, 24, False),
    ([1, 1], [4097, 3], (64, 8), 128, 64, False),
    ([7, 7], [7, 400], (4, 1), 64, 1, False),
    ([5, 0, 3, 8], [70, 9, 3, 8], (6, 3), 40, 7, False),
    ([64, 64], [64, 640], (2, 2), 64, 128, False),
    ([200], [777], (16, 4), 128, 16, False),
    ([130, 90, 130], [1030, 500, 130], (8, 2), 128, 33, False),
    ([33, 1, 1, 70, 1, 0, 129], [900, 5, 1500, 70, 64, 10, 1300], (8, 2), 128, 16, True),
    ([1, 1, 1, 300], [2000, 1, 77, 300], (14, 2), 80, 24, True),
    ([3, 257], [3, 2500], (3, 1), 96, 50, True),
    ([1] * 70, list(range(1, 71)), (4, 2), 64, 16, True),
    ([2, 2], [600, 40], (128, 1), 64, 16, False),
    ([9], [50], (2, 1), 3, 5, False),
    ([520], [520], (7, 1), 128, 10, False),
]


@pytest.mark.parametrize("layout", ["token", "head", "odd"])
@pytest.mark.parametrize("case", ATTN, ids=lambda c: "%dx%d-%s-%d-%d-%s" % (
    len(c[0]), max(c[0]), c[2], c[3], c[4], "packed" if c[5] else "padded"))
def test_attention(case, layout):
    new, lens, heads, D, P, packed = case
    b = Batch(new, lens, heads, D, P, layout, packed)
    check_attn(b)
    check_attn(b, window=37)


@pytest.mark.parametrize("kw", [dict(causal=False), dict(causal=False, window=90), dict(window=1),
                                dict(window=64), dict(out_dtype=F32), dict(scale=1.7)], ids=str)
@pytest.mark.parametrize("packed", [False, True])
def test_masks_types_and_scales(packed, kw):
    b = Batch([1, 40, 130], [500, 333, 190], (6, 2), 64, 16, packed=packed, pad=3)
    O, lse = check_attn(b, **kw)
    assert O.dtype == kw.get("out_dtype", BF)


def test_rows_without_keys_and_rows_of_no_sequence():
    # sequences with no tokens, with fewer tokens than new ones, with no new ones
    b = Batch([4, 4, 0, 2], [0, 2, 50, -3], (4, 2), 64, 16, pad=2)
    O, lse = check_attn(b)
    assert (lse[0] == -math.inf).all() and (lse[2] == -math.inf).all()
    b = Batch([4, 4, 0, 2], [0, 2, 50, -3], (4, 2), 64, 16, packed=True, pad=5, gap=3)
    out = torch.full((1, 4, b.Q.shape[2], 64), 7.0, dtype=BF, device="cuda")
    check_attn(b, out=out)
    assert float((out[:, :, :3] - 7).abs().max()) == 0 and float((out[:, :, -5:] - 7).abs().max()) == 0
    # a table of no entries, no sequences
    b = Batch([2, 2], [5, 5], (4, 2), 64, 16)
    b.table = [[], []]
    O, lse = b.cache.attend(b.Q, torch.empty((2, 0), dtype=torch.int32, device="cuda"), i32([5, 5]))
    assert float(O.abs().max()) == 0 and (lse == -math.inf).all()
    O, lse = b.cache.attend(b.Q[:0], torch.empty((0, 3), dtype=torch.int32, device="cuda"),
                            i32([]))
    assert O.shape == (0, 4, 2, 64)


def test_lengths_past_the_table_and_rows_that_descend():
    b = Batch([3, 3], [40, 20], (4, 2), 64, 8, extra=0)
    b.len = [1000, 41]                      # the table has room for 40
    check_attn(b)
    b = Batch([3, 5, 4], [40, 20, 30], (4, 2), 64, 8, packed=True)
    for rows in ([0, 9, 4, 8], [-5, 2, 2, 1000], [12, 12, 12, 12], [100, 200, -7, 3]):
        b.row_q = rows
        b.seqs = pref.lengths(3, b.Q.shape[2], None, rows)
        if rows[0] == 0:                    # rows of two sequences hold either's
            b.cache.attend(b.Q, *b.args(), **b.rows())
        else:
            check_attn(b)


@pytest.mark.parametrize("new", [1, 150])
def test_pages_that_do_not_exist_are_not_seen(new):
    b = Batch([new] * 4, [400, 300, 200, 170], (4, 2), 64, 16)
    b.table[0][3] = -1
    b.table[0][20] = 1 << 30
    b.table[1][0] = b.kc.shape[0]
    b.table[2] = [-1] * len(b.table[2])     # none at all
    b.table[3][:5] = [-(1 << 31)] * 5
    O, lse = check_attn(b)
    assert (lse[2] == -math.inf).all() and float(O[2].abs().max()) == 0


@pytest.mark.parametrize("new", [1, 9, 140])
def test_what_nobody_sees_is_not_read(new):
    """NaN and infinities behind the sequences' ends, on pages of others, in front of every
    window and in rows of no sequence."""
    for packed in (False, True):
        b = Batch([new] * 3, [300, 150, 411], (8, 2), 128, 16, packed=packed, pad=4)
        window = 100
        keep = torch.zeros((b.kc.shape[0], 16), dtype=torch.bool, device="cuda")
        for row, n, x in zip(b.table, b.len, b.new):
            for j in range(max(0, n - x + 1 - window), n):
                keep[row[j // 16], j % 16] = True
            for k in range(max(0, n - x + 1 - window) // 16):
                row[k] = (1 << 20) if k % 2 else -1     # freed, or taken over by others
        for c, bad in ((b.kc, math.nan), (b.vc, math.inf)):
            c.permute(0, 2, 1, 3)[~keep] = bad
        for x, first, n in b.seqs:
            b.Q[x, :, first + n:] = math.nan if not packed else b.Q[x, :, first + n:]
        if packed:
            b.Q[0, :, b.row_q[-1]:] = math.nan
        O, lse = check_attn(b, window=window)


def test_masked_scores_of_any_size():
    """Scores of +-10^4 and a mask: the largest seen key has the weight, hidden ones none."""
    b = Batch([3, 1], [200, 90], (2, 1), 64, 16)
    b.kc.mul_(100.0)
    b.Q.mul_(100.0)
    s = 1 / 8
    O, lse = b.cache.attend(b.Q, *b.args(), scale=s, **b.rows())
    want, bound, wl, used = pref.attend(b.Q, b.kc, b.vc, b.table, b.len, b.seqs, s, True, 0)
    # a score up to 2^17 carries 2^-24 of its terms' sum: 2^-24 2^19 = 2^-5 in the exponent
    lim = 2.0 ** -4
    live = used[:, None, :].expand(lse.shape)
    assert torch.isfinite(O).all()
    size = b.vc.abs().max().double()
    assert float((O[live].double() - want[live]).abs().max()) <= lim * float(size) * 2
    assert float((lse.double() - wl)[live].abs().max()) <= lim + 2.0 ** -22 * float(wl[live].abs().max())


def test_rows_alike_give_results_alike():
    """The same call twice, and with a workspace of any size: bit for bit where the size is
    the same, within the bounds else."""
    b = Batch([1] * 9, [5000, 1, 700, 2500, 64, 65, 1300, 4100, 9], (8, 2), 128, 16, extra=40)
    a = check_attn(b)
    c = check_attn(b)
    assert torch.equal(a[0], c[0]) and torch.equal(a[1], c[1])
    for ws in (sbp.NO_WORKSPACE, torch.empty(1 << 12, dtype=torch.uint8, device="cuda"),
               torch.empty(1 << 19, dtype=torch.uint8, device="cuda"),
               torch.full((1 << 24,), 255, dtype=torch.uint8, device="cuda")):
        x = check_attn(b, ws=ws)
        y = check_attn(b, ws=ws)
        assert torch.equal(x[0], y[0]) and torch.equal(x[1], y[1])


def test_shared_pages():
    """Two sequences with a common beginning on the same pages, and one page twice in a row."""
    b = Batch([2, 2, 1], [100, 130, 64], (4, 2), 64, 16)
    b.table[1][:5] = b.table[0][:5]
    b.table[2][1] = b.table[2][0]
    check_attn(b)


@pytest.mark.parametrize("p", [2, 5])
def test_head_split(p):
    b = Batch([1, 1, 60], [300, 7, 200], (15, 5), 64, 16, packed=True)
    wO, wl = b.cache.attend(b.Q, *b.args(), **b.rows(), ws=sbp.NO_WORKSPACE)
    for r in range(p):
        h0, h, k0, hk = rank_heads(15, 5, p, r)
        O, lse = b.cache.attend(b.Q, *b.args(), p, r, **b.rows(), ws=sbp.NO_WORKSPACE)
        assert torch.equal(O, wO[:, h0:h0 + h]) and torch.equal(lse, wl[:, h0:h0 + h])
        local = paged.Cache(b.kc[:, k0:k0 + hk], b.vc[:, k0:k0 + hk], sbp.SBP_LOCAL)
        O, lse = local.attend(b.Q[:, h0:h0 + h], *b.args(), p, r, **b.rows(), ws=sbp.NO_WORKSPACE)
        assert torch.equal(O, wO[:, h0:h0 + h]) and torch.equal(lse, wl[:, h0:h0 + h])


@pytest.mark.parametrize("new", [1, 40])
def test_offsets_past_32_bits(new):
    """Pages whose strides pass 2^31 elements, in append and in attention."""
    P, Hk, D, stride = 16, 2, 64, (1 << 31) + 64
    big = [torch.empty(2 * stride + P * Hk * D, dtype=BF, device="cuda") for _ in range(2)]
    kc, vc = (t.as_strided((3, Hk, P, D), (stride, D, Hk * D, 1)) for t in big)
    b = Batch([new], [44], (4, Hk), D, P, extra=0)
    b.table = [[2, 0, 1]]
    kc.copy_(b.kc[:3])
    vc.copy_(b.vc[:3])
    b.kc, b.vc = kc, vc
    b.cache = paged.Cache(kc, vc)
    check_attn(b)
    b.cache.append(b.K, b.V, *b.args())
    for x, i, page, slot, t in pref.places(b.seqs, b.len, b.table, 3, P):
        assert torch.equal(kc[page, :, slot], b.K[x, :, i]) and torch.equal(vc[page, :, slot], b.V[x, :, i])


def test_long_cache():
    """More tokens than 2^17, in pages of 256."""
    b = Batch([2], [(1 << 17) + 77], (4, 1), 128, 256, "head")
    check_attn(b)


def test_attention_streams_graphs_and_shared_workspace():
    b = Batch([1] * 6, [900, 40, 3, 256, 511, 2000], (8, 2), 64, 16)
    table, lens = b.args()
    want = b.cache.attend(b.Q, table, lens)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = b.cache.attend(b.Q, table, lens, stream=side.cuda_stream)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    ws = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
    graphs, outs = [], []
    for window in (0, 100):         # two graphs over one workspace
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(b.cache.attend(b.Q, table, lens, window=window, ws=ws))
        graphs.append(g)
    for step in range(3):
        lens.add_(1)                # lengths are read when the graphs run
        b.len = [n + 1 for n in b.len]
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for window, out in zip((0, 100), outs):
            want = b.cache.attend(b.Q, table, lens, window=window,
                                  ws=torch.empty(1 << 22, dtype=torch.uint8, device="cuda"))
            assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])
    check_attn(b)


# ------------------------------------------------------------------- append
def plain_append(b, rot, order, mul=1.0, table=None):
    """(keys, bounds, values, rotated Q, its bounds) after the call, on the host."""
    f = rope_ref.freqs(rot) if rot else None
    kc, vc = b.kc.cpu().double(), b.vc.cpu().double()
    kb = torch.zeros_like(kc)
    Q, K, V = b.Q.cpu(), b.K.cpu(), b.V.cpu()
    q, qb = Q.double(), torch.zeros(Q.shape, dtype=torch.float64)
    for x, i, page, slot, t in pref.places(b.seqs, b.len, b.table, kc.shape[0], b.P):
        at = torch.tensor([[t]])
        turn = lambda y: rope_ref.rotate(y[x:x + 1, :, i:i + 1], at, f, rot, order, mul)
        if rot:
            y, e = turn(Q)
            q[x, :, i], qb[x, :, i] = y[0, :, 0], e[0, :, 0]
        if page is not None:
            y, e = turn(K) if rot else (K[x:x + 1, :, i:i + 1].double(), torch.zeros(1, K.shape[1], 1, b.D))
            kc[page, :, slot], kb[page, :, slot] = y[0, :, 0], e[0, :, 0]
            vc[page, :, slot] = V[x, :, i].double()
    return kc, kb, vc, q, qb


APPEND = [
    ([1], [1], (1, 1), 64, 16, False, 64),
    ([1] * 16, [5 + 3 * i for i in range(16)], (16, 4), 64, 16, False, 64),
    ([9, 0, 4], [9, 5, 100], (6, 2), 80, 7, False, 40),
    ([33, 1, 1, 70, 1, 0, 129], [900, 5, 150, 70, 64, 10, 300], (8, 2), 128, 16, True, 128),
    ([1, 1, 1, 100], [200, 1, 77, 333], (7, 1), 33, 24, True, 10),
    ([1] * 300, [1 + i % 50 for i in range(300)], (2, 1), 16, 4, True, 16),
    ([65], [65], (3, 3), 111, 1, False, 110),
]


@pytest.mark.parametrize("order", ["halves", "pairs"])
@pytest.mark.parametrize("layout", ["token", "head", "both", "odd"])
@pytest.mark.parametrize("case", APPEND, ids=lambda c: "%dx%d-%s-%d-%d-%s" % (
    len(c[0]), max(c[0]), c[2], c[3], c[4], "packed" if c[5] else "padded"))
def test_append(case, layout, order):
    new, lens, heads, D, P, packed, rot = case
    b = Batch(new, lens, heads, D, P, layout, packed, pad=2)
    kc, kb, vc, q, qb = plain_append(b, rot, order, 1.5)
    out = b.cache.append(b.K, b.V, *b.args(), Q=b.Q, rope=rotary.Rope(rot, order=order, mul=1.5),
                         **b.rows())
    torch.cuda.synchronize()
    rope_ref.check("keys", b.kc, kc, kb)
    assert torch.equal(b.kc.cpu().double()[kb == 0], kc[kb == 0])    # others stay
    assert torch.equal(b.vc.cpu().double(), vc)
    for x, first, n in b.seqs:
        s = slice(first, first + n)
        rope_ref.check("Q", out[x, :, s], q[x, :, s], qb[x, :, s])


@pytest.mark.parametrize("layout", ["token", "odd"])
def test_append_without_rotation(layout):
    b = Batch([3, 1, 20], [50, 1, 31], (4, 2), 48, 16, layout)
    kc, _, vc, _, _ = plain_append(b, 0, "halves")
    assert b.cache.append(b.K, b.V, *b.args(), **b.rows()) is None
    assert torch.equal(b.kc.cpu().double(), kc) and torch.equal(b.vc.cpu().double(), vc)


def test_append_q_in_place_and_rows_of_no_sequence():
    for packed in (False, True):
        b = Batch([3, 1, 20], [50, 1, 31], (4, 2), 64, 16, packed=packed, pad=3)
        rope = rotary.Rope(64)
        kc, kb, vc, q, qb = plain_append(b, 64, "halves")
        keep, v = b.Q.clone(), b.V.clone()
        out = b.cache.append(b.K, b.V, *b.args(), Q=b.Q, rope=rope, out=b.Q, **b.rows())
        assert out.data_ptr() == b.Q.data_ptr() and torch.equal(b.V, v)
        used = torch.zeros(b.Q.shape[0], b.Q.shape[2], dtype=torch.bool)
        for x, first, n in b.seqs:
            s = slice(first, first + n)
            used[x, s] = True
            rope_ref.check("Q", out[x, :, s], q[x, :, s], qb[x, :, s])
        idle = ~used[:, None, :].expand(b.Q.shape[:3]).cuda()
        assert torch.equal(out[idle], keep[idle])
        rope_ref.check("keys", b.kc, kc, kb)


def test_tokens_without_a_place_are_not_stored():
    """Places past the table, before the beginning, pages that do not exist."""
    b = Batch([4, 6, 3, 2], [40, 3, 30, 20], (2, 2), 32, 8, extra=0)
    b.len = [42, 3, 30, -1]
    b.table[2] = [-1, 1 << 30, b.kc.shape[0], b.table[2][3], 0]
    kc, kb, vc, q, qb = plain_append(b, 32, "pairs")
    out = b.cache.append(b.K, b.V, *b.args(), Q=b.Q, rope=rotary.Rope(32, order="pairs"), **b.rows())
    rope_ref.check("keys", b.kc, kc, kb)
    assert torch.equal(b.vc.cpu().double(), vc)
    for x, first, n in b.seqs:
        rope_ref.check("Q", out[x, :, :n], q[x, :, :n], qb[x, :, :n])


@pytest.mark.parametrize("p", [2, 3])
def test_append_head_split(p):
    """Every rank's share into a global cache, and into one of its own."""
    b = Batch([2, 30], [40, 30], (10, 5), 64, 16, packed=True)
    rope = rotary.Rope(64)
    kc, vc = b.kc.clone(), b.vc.clone()
    wq = paged.Cache(kc, vc).append(b.K, b.V, *b.args(), Q=b.Q, rope=rope, **b.rows())
    for r in range(p):
        h0, h, k0, hk = rank_heads(10, 5, p, r)
        mine = b.kc[:, k0:k0 + hk].clone(), b.vc[:, k0:k0 + hk].clone()
        q = b.cache.append(b.K, b.V, *b.args(), p, r, Q=b.Q, rope=rope, **b.rows())
        assert torch.equal(q, wq[:, h0:h0 + h])
        local = paged.Cache(*mine, sbp.SBP_LOCAL)
        q = local.append(b.K, b.V, *b.args(), p, r, Q=b.Q, rope=rope, **b.rows())
        assert torch.equal(q, wq[:, h0:h0 + h])
        q = local.append(b.K[:, k0:k0 + hk], b.V[:, k0:k0 + hk], *b.args(), p, r, Q=b.Q[:, h0:h0 + h],
                         rope=rope, scope=sbp.SBP_LOCAL, **b.rows())
        assert torch.equal(q, wq[:, h0:h0 + h])
        assert torch.equal(mine[0], kc[:, k0:k0 + hk]) and torch.equal(mine[1], vc[:, k0:k0 + hk])
    assert torch.equal(b.kc, kc) and torch.equal(b.vc, vc)


def test_refused_from_torch():
    b = Batch([1, 1], [5, 5], (4, 2), 64, 16)
    table, lens = b.args()
    with pytest.raises(ValueError):
        b.cache.attend(b.Q, table.long(), lens)
    with pytest.raises(ValueError):
        b.cache.attend(b.Q, table, lens[:1])
    with pytest.raises(ValueError):
        b.cache.attend(b.Q, table, lens.cpu())
    with pytest.raises(ValueError):
        b.cache.append(b.K, b.V, table, lens, out=b.Q)
    with pytest.raises(sbp.SbpError) as e:
        b.cache.append(b.K, b.V, table, lens, Q=b.Q)
    assert e.value.code == sbp.SBP_ERR_NULL
    with pytest.raises(sbp.SbpError) as e:
        b.cache.attend(b.Q, table, lens, len_q=i32([1, 1]), row_q=i32([0, 1, 2]))
    assert e.value.code == sbp.SBP_ERR_SHAPE


# ------------------------------------------------------- many shapes, edges
def draw(seed):
    """A batch of sizes that meet the tiles', pages' and parts' edges in ever other ways."""
    import random
    r = random.Random(seed)
    Hk = r.choice((1, 2, 3, 8))
    group = r.choice((1, 2, 4, 5, 8, 16))
    D = r.choice((8, 16, 40, 64, 64, 96, 128, 128, r.randrange(1, 129)))
    P = r.choice((4, 8, 16, 16, 32, 100, 257, r.randrange(1, 64)))
    n = r.choice((1, 2, 5, 33, 130))
    most = {1: 700, 2: 400, 5: 150, 33: 30, 130: 5}[n]
    new = [r.choice((0, 1, 1, 1, r.randrange(1, most + 1))) for _ in range(n)]
    lens = [r.choice((x, x + r.randrange(0, 40), x + r.randrange(0, 3000 // n + 200))) for x in new]
    return dict(new=new, lens=lens, heads=(Hk * group, Hk), D=D, P=P,
                layout=r.choice(("token", "head", "both", "odd")), packed=r.random() < 0.6,
                pad=r.randrange(0, 3), gap=r.randrange(0, 2), seed=seed), dict(
                    causal=r.random() < 0.8, window=r.choice((0, 0, 0, 1, 50, 700)),
                    out_dtype=r.choice((BF, F32)))


@pytest.mark.parametrize("seed", range(60))
def test_attention_of_drawn_shapes(seed):
    shape, kw = draw(1000 + seed)
    if max(shape["new"]) == 0:
        shape["new"][0] = 1
        shape["lens"][0] += 1
    check_attn(Batch(**shape), **kw)


@pytest.mark.parametrize("seed", range(24))
def test_append_of_drawn_shapes(seed):
    shape, _ = draw(2000 + seed)
    if max(shape["new"]) == 0:
        shape["new"][0] = 1
        shape["lens"][0] += 1
    b = Batch(**shape)
    rot, order = b.D // 2 * 2, ("halves", "pairs")[seed % 2]
    kc, kb, vc, q, qb = plain_append(b, rot, order)
    kw = dict(Q=b.Q, rope=rotary.Rope(rot, order=order), out_dtype=(BF, F32)[seed // 2 % 2]) if rot else {}
    out = b.cache.append(b.K, b.V, *b.args(), **kw, **b.rows())
    torch.cuda.synchronize()
    rope_ref.check("keys", b.kc, kc, kb)
    assert torch.equal(b.kc.cpu().double()[kb == 0], kc[kb == 0])
    assert torch.equal(b.vc.cpu().double(), vc)
    for x, first, n in b.seqs if rot else ():
        s = slice(first, first + n)
        rope_ref.check("Q", out[x, :, s], q[x, :, s], qb[x, :, s])


def test_copied_columns_and_values_keep_their_bits():
    """Not-a-numbers of any payload, infinities, subnormal numbers, -0."""
    b = Batch([70, 3], [90, 3], (2, 2), 48, 16, packed=True)
    g = torch.Generator(device="cuda").manual_seed(3)
    bits = torch.randint(-(1 << 15), 1 << 15, b.V.shape, generator=g, device="cuda", dtype=torch.int16)
    bits[..., ::3] |= 0x7f80                       # every exponent bit
    b.V.copy_(bits.view(BF))
    b.K[..., 16:] = bits.view(BF)[..., 16:]
    b.cache.append(b.K, b.V, *b.args(), rope=rotary.Rope(16), **b.rows())
    raw = lambda t: t.contiguous().view(torch.int16)
    for x, i, page, slot, t in pref.places(b.seqs, b.len, b.table, b.kc.shape[0], b.P):
        assert torch.equal(raw(b.vc[page, :, slot]), raw(b.V[x, :, i]))
        assert torch.equal(raw(b.kc[page, :, slot, 16:]), raw(b.K[x, :, i, 16:]))


@pytest.mark.parametrize("new", [1, 3])
def test_room_for_more_steps_than_31_bits_count(new):
    """A table whose rows have room for 2^29 tokens: the units of the items, at most, pass 2^31
    and are taken coarser; results as with a table of their size."""
    B, H, Hk, D, P = 64, 16, 16, 64, 512
    lens = [1 + 53 * i for i in range(B)]
    b = Batch([new] * B, [max(new, n) for n in lens], (H, Hk), D, P, "head")
    wide = torch.full((B, 1 << 20), -1, dtype=torch.int32, device="cuda")
    table = i32(b.table)
    wide[:, :table.shape[1]] = table
    s = 1 / 8
    want, bound, wl, _ = pref.attend(b.Q, b.kc, b.vc, b.table, b.len, b.seqs, s, True, 0)
    for ws in (None, sbp.NO_WORKSPACE):
        O, lse = b.cache.attend(b.Q, wide, i32(b.len), scale=s, ws=ws)
        pref.check("O", O, want, bound)
        assert float((lse.double() - wl).abs().max()) <= 2.0 ** -14


@pytest.mark.parametrize("packed", [False, True])
def test_many_sequences(packed):
    """More sequences than the lanes of a wave count at once, among them many without tokens."""
    n = 700
    new = [(0, 1, 1, 2, 5)[i * i % 5] for i in range(n)]
    lens = [x + (i * 37) % 90 for i, x in enumerate(new)]
    b = Batch(new, lens, (4, 2), 64, 16, packed=packed)
    check_attn(b)
    kc, kb, vc, q, qb = plain_append(b, 64, "halves")
    b.cache.append(b.K, b.V, *b.args(), rope=rotary.Rope(64), **b.rows())
    rope_ref.check("keys", b.kc, kc, kb)
    assert torch.equal(b.vc.cpu().double(), vc)


def test_no_pages_no_lse_strided_output():
    b = Batch([2, 3], [20, 30], (4, 2), 64, 16)
    out = torch.full((2, 4, 3, 70), 7.0, dtype=F32, device="cuda")
    want, _ = b.cache.attend(b.Q, *b.args(), **b.rows(), out_dtype=F32)
    O, lse = b.cache.attend(b.Q, *b.args(), **b.rows(), out=out[..., 3:67], lse=False)
    assert lse is None and torch.equal(O, want)
    assert float((out[..., :3] - 7).abs().max()) == 0 and float((out[..., 67:] - 7).abs().max()) == 0
    none = paged.Cache(b.kc[:0], b.vc[:0])
    O, lse = none.attend(b.Q, *b.args(), **b.rows())
    assert float(O.abs().max()) == 0 and (lse == -math.inf).all()
    none.append(b.K, b.V, *b.args(), **b.rows())


def test_one_long_sequence_in_many_parts():
    """A single item of one key head, cut into as many parts as there are workgroups."""
    for new in (1, 2):
        check_attn(Batch([new], [40000], (8, 1), 64, 16, "head"))
        check_attn(Batch([new], [40000], (8, 1), 128, 64, "head"))


# new tokens, lengths, (H, Hk), D, page, layout, room of a table row in tokens, kernel
FORMS = [
    ([1] * 3, [200, 90, 7], (4, 2), 64, 16, "head", 0, "<64,2,32,4,1>"),
    ([1] * 3, [200, 90, 7], (4, 2), 64, 3, "head", 0, "<64,2,32,4,0>"),
    ([40] * 2, [200, 90], (16, 2), 64, 16, "token", 0, "<64,1,64,4,1>"),
    ([40] * 2, [200, 90], (16, 2), 50, 16, "token", 0, "<64,1,64,4,0>"),
    ([1] * 3, [200, 90, 7], (4, 2), 128, 16, "head", 0, "<128,1,32,4,1>"),
    ([1] * 3, [200, 90, 7], (4, 2), 128, 16, "odd", 0, "<128,1,32,4,0>"),
    ([1] * 3, [200, 90, 7], (4, 2), 128, 16, "head", 1600, "<128,2,32,8,1>"),
    ([1] * 3, [200, 90, 7], (4, 2), 80, 6, "head", 1600, "<128,2,32,8,0>"),
    ([70] * 2, [200, 90], (16, 2), 128, 16, "token", 1600, "<128,1,64,8,1>"),
    ([70] * 2, [200, 90], (16, 2), 100, 16, "token", 1600, "<128,1,64,8,0>"),
]


@pytest.mark.parametrize("case", FORMS, ids=lambda c: c[-1])
def test_every_form_of_the_kernel(case):
    new, lens, heads, D, P, layout, room, kernel = case
    b = Batch(new, lens, heads, D, P, layout, extra=max(room - max(lens), 0) // P + 1)
    check_attn(b)
    sbp.sbp_profile_begin(4)
    b.cache.attend(b.Q, *b.args(), **b.rows())
    names = [n for n, _ in sbp.sbp_profile_end(4)]
    assert names == ["paged_attn_kernel" + kernel, "paged_join_kernel"]


def test_parts_of_more_rows_than_a_wave_has():
    """Items cut in parts, of every order that partial outputs lie in, and of rows past 32."""
    for new, heads, D, lens, room in ((8, (16, 2), 128, 1500, 2000), (8, (16, 2), 64, 3000, 0),
                                      (20, (16, 2), 128, 900, 0), (60, (8, 1), 64, 5000, 0),
                                      (100, (8, 1), 128, 5000, 6000)):
        check_attn(Batch([new] * 2, [lens, lens - 77], heads, D, 16, "head", extra=1 + max(room - lens, 0) // 16))


@pytest.mark.parametrize("layout", ["head", "odd"])
@pytest.mark.parametrize("D", [65, 72, 80, 95, 96, 97])
def test_head_dimensions_about_96(D, layout):
    """Every form, items cut and whole (a sequence of more steps than the others)."""
    for new, lens, heads, room in (([1] * 5, [900, 33, 1, 64, 1200], (8, 2), 0),
                                   ([1] * 5, [900, 33, 1, 64, 1200], (8, 2), 1700),
                                   ([70, 65], [300, 1600], (8, 2), 0),
                                   ([40] * 2, [200, 90], (16, 2), 1700)):
        check_attn(Batch(new, lens, heads, D, 16, layout, extra=max(room - max(lens), 0) // 16 + 1))
    b = Batch([1, 1], [700, 650], (4, 1), D, 16, layout)
    for kw in (dict(out_dtype=torch.float32), dict(causal=False, window=40)):
        check_attn(b, **kw)


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("new", [
    [300, 1, 37, 128, 0, 260] * 7,                  # most of several tiles
    [200] * 70,                                     # more than 64 sequences, alike
    [3, 1, 900, 1, 1, 40] + [1] * 20,               # one long among tokens
    [150, 160, 170, 1500],                          # one much longer than other prompts
], ids=["several", "alike", "one", "longer"])
def test_sums_over_tiles_of_sequences(new, packed):
    check_attn(Batch(new, [n + i % 9 for i, n in enumerate(new)], (8, 2), 64, 16, "head", packed=packed))


@pytest.mark.parametrize("D", [8, 64, 96, 104, 128])
def test_output_rows_at_any_address(D):
    """Whole tiles and joined ones, to rows that start at odd elements; nothing beside them is written."""
    for new, lens in (([100, 70], [130, 70]), ([300], [900])):
        b = Batch(new, lens, (8, 2), D, 16, "head")
        room = torch.full((len(new), 8, max(new), D + 5), 7.0, dtype=torch.bfloat16, device="cuda")
        check_attn(b, out=room[..., 3:3 + D])
        assert bool((room[..., :3] == 7).all()) and bool((room[..., 3 + D:] == 7).all())


@pytest.mark.parametrize("D,groups", [(64, 512), (128, 256)])
@pytest.mark.parametrize("new", [1, 3])
def test_workspaces_of_odd_numbers_of_partial_outputs(new, D, groups):
    """Odd rows of an item, and room for an odd number of their partial outputs."""
    b = Batch([new], [6000], (1, 1), D, 16, "head")
    for slots in (groups, groups + 1, groups + 7, 2 * groups - 1, 2 * groups + 1):
        ws = torch.full((8 * groups + slots * new * (2 + D),), math.nan, dtype=F32, device="cuda")
        check_attn(b, ws=ws)


@pytest.mark.parametrize("new", [1, 5, 60])
def test_lengths_past_the_table_in_either_call(new):
    """Past the table's room attention takes the room for the length, in its masks too; append
    rotates by the length as it is and drops what has no place."""
    b = Batch([new, new], [96, 90], (4, 2), 64, 16, extra=0)
    full, past = i32([96, 96]), i32([97 + new, (1 << 31) - 1])
    table = b.args()[0]
    for kw in (dict(), dict(window=20), dict(window=(1 << 31) - 1), dict(causal=False, window=70)):
        want, got = (b.cache.attend(b.Q, table, n, **kw) for n in (full, past))
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    b.len = past.tolist()
    kc, kb, vc, q, qb = plain_append(b, 64, "halves")
    out = b.cache.append(b.K, b.V, table, past, Q=b.Q, rope=rotary.Rope(64))
    rope_ref.check("keys", b.kc, kc, kb)
    rope_ref.check("Q", out, q, qb)
    assert torch.equal(b.vc.cpu().double(), vc)
