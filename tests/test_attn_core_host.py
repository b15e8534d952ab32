"""Host-side checks of the softmax attention calls: every case has exactly one
defect, so no call reaches a kernel; fake device addresses, skipped wherever a GPU
is visible."""
import math

import pytest

from paper_2301_06813_amd import attention, sbp

BF, F32 = sbp.SBP_BF16, sbp.SBP_F32
GL, LO, ACC = sbp.SBP_GLOBAL, sbp.SBP_LOCAL, sbp.SBP_ACCUMULATE
MB = 1 << 20


def _gpu_visible():
    try:
        import torch
        return torch.cuda.is_available()
    except Exception:
        return False


pytestmark = pytest.mark.skipif(_gpu_visible(), reason="uses fake device addresses")


def v4(at, B, H, R, C, dtype=BF, scope=GL, sb=None, sh=None, ld=None):
    """A view `at` MiB into the fake device memory."""
    ld = C if ld is None else ld
    sh = R * ld if sh is None else sh
    sb = H * sh if sb is None else sb
    return sbp.sbp_view4_t(None if at is None else at * MB, B, H, R, C, sb, sh, ld, dtype, scope)


def opts(scale=0.125, causal=0, window=0, lq=None, lk=None):
    return sbp.sbp_attn_opts_t(scale, causal, window, lq, lk)


def fwd_args():
    # 10 query heads on 5 key heads over p = 2: rank 1 has key heads 3, 4, query heads 6..9
    return dict(q=v4(16, 2, 10, 64, 32), k=v4(32, 2, 5, 48, 32), v=v4(48, 2, 5, 48, 32),
                opts=opts(), o=v4(64, 2, 4, 64, 32, scope=LO), lse=v4(80, 2, 4, 64, 1, F32, LO),
                p=2, r=1, ws=sbp.NO_WORKSPACE)


def bwd_args():
    return dict(do=v4(96, 2, 4, 64, 32, scope=LO), q=v4(16, 2, 10, 64, 32), k=v4(32, 2, 5, 48, 32),
                v=v4(48, 2, 5, 48, 32), o=v4(64, 2, 4, 64, 32, scope=LO),
                lse=v4(80, 2, 4, 64, 1, F32, LO), opts=opts(), dq=v4(112, 2, 4, 64, 32, scope=LO),
                dk=v4(128, 2, 2, 48, 32, scope=LO), dv=v4(144, 2, 2, 48, 32, scope=LO), p=2, r=1,
                ws=sbp.sbp_workspace_t(160 * MB, 1 * MB))


def fwd(c):
    sbp.sbp_attn_core_fwd(c["q"], c["k"], c["v"], c["opts"], c["o"], c["lse"], c["p"], c["r"],
                          stream=0, ws=c["ws"])


def bwd(c):
    sbp.sbp_attn_core_bwd(c["do"], c["q"], c["k"], c["v"], c["o"], c["lse"], c["opts"], c["dq"],
                          c["dk"], c["dv"], c["p"], c["r"], stream=0, ws=c["ws"])


SHARED = [
    ("rank out of range", dict(r=2), sbp.SBP_ERR_LAYOUT),
    ("no devices", dict(p=0), sbp.SBP_ERR_LAYOUT),
    ("fp32 Q", dict(q=v4(16, 2, 10, 64, 32, F32)), sbp.SBP_ERR_DTYPE),
    ("unknown dtype", dict(v=v4(48, 2, 5, 48, 32, 7)), sbp.SBP_ERR_DTYPE),
    ("head dims differ", dict(k=v4(32, 2, 5, 48, 40)), sbp.SBP_ERR_SHAPE),
    ("V's head dim differs", dict(v=v4(48, 2, 5, 48, 16)), sbp.SBP_ERR_SHAPE),
    ("key lengths differ", dict(v=v4(48, 2, 5, 40, 32)), sbp.SBP_ERR_SHAPE),
    ("key head counts differ", dict(v=v4(48, 2, 10, 48, 32)), sbp.SBP_ERR_SHAPE),
    ("query heads no multiple of key heads", dict(q=v4(16, 2, 12, 64, 32)), sbp.SBP_ERR_SHAPE),
    ("scopes differ", dict(k=v4(32, 2, 5, 48, 32, scope=LO)), sbp.SBP_ERR_SHAPE),
    ("accumulating input", dict(q=v4(16, 2, 10, 64, 32, scope=ACC)), sbp.SBP_ERR_SHAPE),
    ("batches differ", dict(k=v4(32, 3, 5, 48, 32)), sbp.SBP_ERR_SHAPE),
    ("ld < cols", dict(q=v4(16, 2, 10, 64, 32, ld=16)), sbp.SBP_ERR_SHAPE),
    ("too many rows", dict(q=v4(16, 2, 10, (1 << 29) + 1, 32, sb=0, sh=0)), sbp.SBP_ERR_SHAPE),
    ("strides beyond 62 bits", dict(q=v4(16, (1 << 31) - 1, 10, 64, 32, sb=1 << 40)), sbp.SBP_ERR_SHAPE),
    ("misaligned", dict(q=sbp.sbp_view4_t(16 * MB + 1, 2, 10, 64, 32, 20480, 2048, 32, BF, GL)),
     sbp.SBP_ERR_ALIGN),
    ("null K", dict(k=v4(None, 2, 5, 48, 32)), sbp.SBP_ERR_NULL),
    ("scale 0", dict(opts=opts(0.0)), sbp.SBP_ERR_SHAPE),
    ("scale < 0", dict(opts=opts(-1.0)), sbp.SBP_ERR_SHAPE),
    ("scale NaN", dict(opts=opts(math.nan)), sbp.SBP_ERR_SHAPE),
    ("scale infinite", dict(opts=opts(math.inf)), sbp.SBP_ERR_SHAPE),
    ("scale below 2^-100", dict(opts=opts(2.0 ** -101)), sbp.SBP_ERR_SHAPE),
    ("scale above 2^100", dict(opts=opts(2.0 ** 101)), sbp.SBP_ERR_SHAPE),
    ("window < 0", dict(opts=opts(window=-1)), sbp.SBP_ERR_SHAPE),
    ("causal neither 0 nor 1", dict(opts=opts(causal=2)), sbp.SBP_ERR_SHAPE),
    ("misaligned lengths", dict(opts=opts(lk=200 * MB + 2)), sbp.SBP_ERR_ALIGN),
    ("workspace size < 0", dict(ws=sbp.sbp_workspace_t(160 * MB, -1)), sbp.SBP_ERR_SHAPE),
    ("null workspace", dict(ws=sbp.sbp_workspace_t(None, MB)), sbp.SBP_ERR_NULL),
    ("misaligned workspace", dict(ws=sbp.sbp_workspace_t(160 * MB + 8, MB)), sbp.SBP_ERR_ALIGN),
    ("workspace on Q", dict(ws=sbp.sbp_workspace_t(16 * MB, MB)), sbp.SBP_ERR_ALIAS),
    ("workspace on the lengths", dict(opts=opts(lq=160 * MB + 64), ws=sbp.sbp_workspace_t(160 * MB, MB)),
     sbp.SBP_ERR_ALIAS),
]
FWD = SHARED + [
    ("output heads", dict(o=v4(64, 2, 5, 64, 32, scope=LO)), sbp.SBP_ERR_SHAPE),
    ("output rows", dict(o=v4(64, 2, 4, 48, 32, scope=LO)), sbp.SBP_ERR_SHAPE),
    ("output rows overlap", dict(o=v4(64, 2, 4, 64, 32, scope=LO, sh=32)), sbp.SBP_ERR_SHAPE),
    ("accumulating output", dict(o=v4(64, 2, 4, 64, 32, F32, ACC)), sbp.SBP_ERR_SHAPE),
    ("lse columns", dict(lse=v4(80, 2, 4, 64, 2, F32, LO)), sbp.SBP_ERR_SHAPE),
    ("bf16 lse", dict(lse=v4(80, 2, 4, 64, 1, BF, LO)), sbp.SBP_ERR_DTYPE),
    ("output on V", dict(o=v4(48, 2, 4, 64, 32, scope=LO)), sbp.SBP_ERR_ALIAS),
    ("output on the lengths", dict(opts=opts(lk=64 * MB + 64)), sbp.SBP_ERR_ALIAS),
    ("lse on the output", dict(lse=v4(64, 2, 4, 64, 1, F32, LO)), sbp.SBP_ERR_ALIAS),
    ("workspace on the output", dict(ws=sbp.sbp_workspace_t(64 * MB, MB)), sbp.SBP_ERR_ALIAS),
    ("more rows than a launch covers",
     dict(q=v4(16, 1 << 12, 10, 1 << 15, 32, sb=0, sh=0), k=v4(32, 1 << 12, 5, 48, 32, sb=0, sh=0),
          v=v4(48, 1 << 12, 5, 48, 32, sb=0, sh=0), o=v4(64, 1 << 12, 4, 1 << 15, 32, scope=LO)),
     sbp.SBP_ERR_SHAPE),
    ("head dimension 129", dict(q=v4(16, 2, 10, 64, 129), k=v4(32, 2, 5, 48, 129),
                                v=v4(48, 2, 5, 48, 129), o=v4(64, 2, 4, 64, 129, scope=LO)),
     sbp.SBP_ERR_SHAPE),
    ("head dimension 0", dict(q=v4(16, 2, 10, 64, 0, ld=1), k=v4(32, 2, 5, 48, 0, ld=1),
                              v=v4(48, 2, 5, 48, 0, ld=1), o=v4(64, 2, 4, 64, 0, scope=LO, ld=1)),
     sbp.SBP_ERR_SHAPE),
]
BWD = SHARED + [
    ("fp32 dO", dict(do=v4(96, 2, 4, 64, 32, F32, LO)), sbp.SBP_ERR_DTYPE),
    ("bf16 lse", dict(lse=v4(80, 2, 4, 64, 1, BF, LO)), sbp.SBP_ERR_DTYPE),
    ("dO's heads", dict(do=v4(96, 2, 5, 64, 32, scope=LO)), sbp.SBP_ERR_SHAPE),
    ("GLOBAL O of local heads", dict(o=v4(64, 2, 4, 64, 32)), sbp.SBP_ERR_SHAPE),
    ("dK's heads", dict(dk=v4(128, 2, 4, 48, 32, scope=LO)), sbp.SBP_ERR_SHAPE),
    ("dV's rows", dict(dv=v4(144, 2, 2, 64, 32, scope=LO)), sbp.SBP_ERR_SHAPE),
    ("accumulating bf16", dict(dq=v4(112, 2, 4, 64, 32, BF, ACC)), sbp.SBP_ERR_DTYPE),
    ("dQ on dK", dict(dk=v4(112, 2, 2, 48, 32, scope=LO)), sbp.SBP_ERR_ALIAS),
    ("dV on O", dict(dv=v4(64, 2, 2, 48, 32, scope=LO)), sbp.SBP_ERR_ALIAS),
    ("workspace on dQ", dict(ws=sbp.sbp_workspace_t(112 * MB, MB)), sbp.SBP_ERR_ALIAS),
    ("workspace on dO", dict(ws=sbp.sbp_workspace_t(96 * MB, MB)), sbp.SBP_ERR_ALIAS),
    ("no workspace", dict(ws=sbp.NO_WORKSPACE), sbp.SBP_ERR_WORKSPACE),
    ("small workspace", dict(ws=sbp.sbp_workspace_t(160 * MB, 8 * 2 * 4 * 64 - 16)),
     sbp.SBP_ERR_WORKSPACE),
]


@pytest.mark.parametrize("name,change,code", FWD, ids=[c[0] for c in FWD])
def test_forward_refusals(name, change, code):
    with pytest.raises(sbp.SbpError) as ei:
        fwd({**fwd_args(), **change})
    assert ei.value.code == code


@pytest.mark.parametrize("name,change,code", BWD, ids=[c[0] for c in BWD])
def test_backward_refusals(name, change, code):
    with pytest.raises(sbp.SbpError) as ei:
        bwd({**bwd_args(), **change})
    assert ei.value.code == code


def test_gradients_in_one_buffer():
    # dQ, dK and dV as column blocks of one [batch][rows][...] buffer pass the overlap
    # check (the call then fails for want of a workspace); with columns that meet, other
    # strides or another row count they do not
    def part(first, heads, rows=64, cols=32, ld=8 * 32, sb=64 * 8 * 32):
        return sbp.sbp_view4_t(112 * MB + first * 32 * 2, 2, heads, rows, cols, sb, 32, ld, BF, LO)

    base = {**bwd_args(), "k": v4(32, 2, 5, 64, 32), "v": v4(48, 2, 5, 64, 32), "ws": sbp.NO_WORKSPACE}
    cases = [(part(0, 4), part(4, 2), part(6, 2), sbp.SBP_ERR_WORKSPACE),
             (part(4, 4), part(0, 2), part(2, 2), sbp.SBP_ERR_WORKSPACE),
             (part(0, 4), part(3, 2), part(6, 2), sbp.SBP_ERR_ALIAS),
             (part(0, 4), part(4, 2), part(7, 2), sbp.SBP_ERR_ALIAS),
             (part(0, 4), part(4, 2, ld=9 * 32, sb=64 * 9 * 32), part(6, 2), sbp.SBP_ERR_ALIAS),
             (part(0, 4), part(4, 2, sb=2 * 64 * 8 * 32), part(6, 2), sbp.SBP_ERR_ALIAS)]
    for dq, dk, dv, code in cases:
        with pytest.raises(sbp.SbpError) as ei:
            bwd({**base, "dq": dq, "dk": dk, "dv": dv})
        assert ei.value.code == code


def test_rank_heads():
    for H, Hk, p in ((16, 16, 8), (10, 5, 2), (14, 2, 3), (6, 3, 7)):
        q = k = 0
        for r in range(p):
            q0, hq, k0, hk = attention.rank_heads(H, Hk, p, r)
            assert (q0, k0) == (q, k) and hq == hk * (H // Hk)
            q, k = q + hq, k + hk
        assert (q, k) == (H, Hk)


def test_lengths_are_int32():
    import torch
    with pytest.raises(ValueError):
        sbp.attn_opts(1.0, len_q=torch.zeros(3, dtype=torch.int64))
    with pytest.raises(ValueError):
        sbp.attn_opts(1.0, len_k=torch.zeros(6, dtype=torch.int32)[::2])


TB = 1 << 20   # MiB


@pytest.mark.parametrize("heads,rows,keys,fits", [
    ((1 << 23) - 1, 8, 8, True), (1 << 23, 8, 8, False), ((1 << 23) - 1, 32, 32, True),
    (1 << 23, 1, 32, False), (1 << 23, 8, 0, True), ((1 << 24) - 1, 0, 32, True)])
def test_backward_workgroups(heads, rows, keys, fits):
    # dK's and dV's workgroups and dQ's are of one launch; what fits is then refused for its
    # workspace, which lies on Q. The forward call takes all of these
    q, k, v, do, o, lse, dq, dk, dv = (
        v4(i * TB, heads, 1, r, c, t, s, sh=max(r, 1) * c) for i, (r, c, t, s) in enumerate(
            [(rows, 32, BF, GL), (keys, 32, BF, GL), (keys, 32, BF, GL), (rows, 32, BF, LO),
             (rows, 32, BF, LO), (rows, 1, F32, LO), (rows, 32, BF, LO), (keys, 32, BF, LO),
             (keys, 32, BF, LO)], 1))
    on = q if rows else k
    call = dict(do=do, q=q, k=k, v=v, o=o, lse=lse, opts=opts(), dq=dq, dk=dk, dv=dv, p=1, r=0,
                ws=sbp.sbp_workspace_t(on.data, MB))
    with pytest.raises(sbp.SbpError) as ei:
        bwd(call)
    assert ei.value.code == (sbp.SBP_ERR_ALIAS if fits else sbp.SBP_ERR_SHAPE)
    with pytest.raises(sbp.SbpError) as ei:
        fwd(call)
    assert ei.value.code == sbp.SBP_ERR_ALIAS
