"""Host-side checks of the paged cache's calls: every case has exactly one defect, so no call
reaches a kernel; fake device addresses, skipped wherever a GPU is visible."""
import math

import pytest

from paper_2301_06813_amd import sbp

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
    ld = C if ld is None else ld
    sh = R * ld if sh is None else sh
    sb = H * sh if sb is None else sb
    return sbp.sbp_view4_t(None if at is None else int(at * MB), B, H, R, C, sb, sh, ld, dtype, scope)


def pages(table=200 * MB, ld=12, seqs=2, width=12, k=201 * MB, q=None, rows=None):
    return sbp.sbp_pages_t(table, ld, seqs, width, k, q, rows)


def append_args():
    # 10 query heads on 5 key heads over p = 2: rank 1 has key heads 3, 4, query heads 6..9
    return dict(k=v4(16, 2, 5, 64, 32), v=v4(32, 2, 5, 64, 32), pages=pages(),
                rope=sbp.sbp_rope_t(202 * MB, 32, 0, 1.0), kc=v4(48, 30, 5, 16, 32),
                vc=v4(64, 30, 5, 16, 32), q=v4(80, 2, 10, 64, 32), qo=v4(96, 2, 4, 64, 32, scope=LO),
                p=2, r=1)


def attn_args():
    return dict(q=v4(80, 2, 10, 64, 32), kc=v4(48, 30, 5, 16, 32), vc=v4(64, 30, 5, 16, 32),
                pages=pages(), scale=0.125, causal=1, window=0, o=v4(96, 2, 4, 64, 32, scope=LO),
                lse=v4(112, 2, 4, 64, 1, F32, LO), p=2, r=1, ws=sbp.NO_WORKSPACE)


def append(c):
    sbp.sbp_paged_append(c["k"], c["v"], c["pages"], c["rope"], c["kc"], c["vc"], c["q"], c["qo"],
                         c["p"], c["r"], stream=0)


def attn(c):
    sbp.sbp_paged_attn(c["q"], c["kc"], c["vc"], c["pages"], c["scale"], c["causal"], c["window"],
                       c["o"], c["lse"], c["p"], c["r"], stream=0, ws=c["ws"])


S, A, D_, N = sbp.SBP_ERR_SHAPE, sbp.SBP_ERR_ALIAS, sbp.SBP_ERR_DTYPE, sbp.SBP_ERR_NULL
AL, LA = sbp.SBP_ERR_ALIGN, sbp.SBP_ERR_LAYOUT
BOTH = [
    ("no pages", dict(pages=None), N),
    ("no cache", dict(kc=None), N),
    ("null table", dict(pages=pages(table=None)), N),
    ("null lengths", dict(pages=pages(k=None)), N),
    ("misaligned table", dict(pages=pages(table=200 * MB + 2)), AL),
    ("misaligned lengths", dict(pages=pages(k=201 * MB + 1)), AL),
    ("misaligned first rows", dict(pages=pages(q=201 * MB + 66)), AL),
    ("table rows overlap", dict(pages=pages(ld=11)), S),
    ("negative width", dict(pages=pages(width=-1)), S),
    ("negative sequences", dict(pages=pages(seqs=-1)), S),
    ("sequences for batches", dict(pages=pages(seqs=3)), S),
    ("first rows in a padded batch", dict(pages=pages(rows=201 * MB + 64)), S),
    ("too many tokens", dict(pages=pages(ld=1 << 26, width=1 << 26)), S),
    ("rank out of range", dict(r=2), LA),
    ("no devices", dict(p=0), LA),
    ("fp32 cache", dict(kc=v4(48, 30, 5, 16, 32, F32)), D_),
    ("values of another type", dict(vc=v4(64, 30, 5, 16, 32, F32)), D_),
    ("cache scopes differ", dict(vc=v4(64, 30, 5, 16, 32, scope=LO)), S),
    ("cache head dims differ", dict(kc=v4(48, 30, 5, 16, 16), vc=v4(64, 30, 5, 16, 16)), S),
    ("pages differ", dict(vc=v4(64, 29, 5, 16, 32)), S),
    ("page tokens differ", dict(vc=v4(64, 30, 5, 15, 32)), S),
    ("no tokens a page", dict(kc=v4(48, 30, 5, 0, 32), vc=v4(64, 30, 5, 0, 32)), S),
    ("query heads no multiple of key heads", dict(q=v4(80, 2, 12, 64, 32)), S),
    ("fp32 Q", dict(q=v4(80, 2, 10, 64, 32, F32)), D_),
]
APPEND = BOTH + [
    ("no K", dict(k=None), N),
    ("Q without Qo", dict(qo=None), N),
    ("Qo without Q", dict(q=None), N),
    ("Q without rotation", dict(rope=None), N),
    ("rows of V", dict(v=v4(32, 2, 5, 63, 32)), S),
    ("batches of Q", dict(q=v4(80, 1, 10, 64, 32)), S),
    ("heads of V", dict(v=v4(32, 2, 10, 64, 32)), S),
    ("scope of V", dict(v=v4(32, 2, 5, 64, 32, scope=LO)), S),
    ("heads of the cache", dict(kc=v4(48, 30, 6, 16, 32), vc=v4(64, 30, 6, 16, 32)), S),
    ("heads of a local cache", dict(kc=v4(48, 30, 5, 16, 32, scope=LO), vc=v4(64, 30, 5, 16, 32, scope=LO)), S),
    ("dim past the head", dict(rope=sbp.sbp_rope_t(202 * MB, 34, 0, 1.0)), S),
    ("fp32 K", dict(k=v4(16, 2, 5, 64, 32, F32)), D_),
    ("accumulating Qo", dict(qo=v4(96, 2, 4, 64, 32, F32, ACC)), S),
    ("heads of Qo", dict(qo=v4(96, 2, 5, 64, 32, scope=LO)), S),
    ("cache rows overlap", dict(kc=v4(48, 30, 5, 16, 32, sh=32)), A),
    ("cache pages overlap", dict(vc=v4(64, 30, 5, 16, 32, sb=64)), A),
    ("values on keys", dict(vc=v4(48, 30, 5, 16, 32)), A),
    ("cache on K", dict(kc=v4(16, 30, 5, 16, 32)), A),
    ("cache on Q", dict(vc=v4(80, 30, 5, 16, 32)), A),
    ("cache on Qo", dict(qo=v4(48, 2, 4, 64, 32, scope=LO)), A),
    ("cache on the table", dict(pages=pages(table=48 * MB + 64 * 1024)), A),
    ("cache on the frequencies", dict(rope=sbp.sbp_rope_t(64 * MB + 64 * 1024, 32, 0, 1.0)), A),
    ("Qo on V", dict(qo=v4(32, 2, 4, 64, 32, scope=LO)), A),
    ("Qo on other heads of Q", dict(qo=v4(80, 2, 4, 64, 32, scope=LO)), A),
    ("Qo on the lengths", dict(pages=pages(k=96 * MB + 4096)), A),
    ("more rows than a launch covers", dict(
        k=v4(16, 2, 5, 1 << 28, 32, sb=0, sh=0), v=v4(32, 2, 5, 1 << 28, 32, sb=0, sh=0),
        q=v4(80, 2, 10, 1 << 28, 32, sb=0, sh=0), qo=v4(1 << 20, 2, 4, 1 << 28, 32, scope=LO),
        kc=v4(1 << 30, 30, 5, 16, 32), vc=v4((1 << 30) + 16, 30, 5, 16, 32),
        pages=pages(1 << 55, 12, 2, 12, 1 << 56), rope=sbp.sbp_rope_t(1 << 57, 32, 0, 1.0)), S),
]
ATTN = BOTH + [
    ("no output", dict(o=None), N),
    ("cache of another scope", dict(kc=v4(48, 30, 5, 16, 32, scope=LO), vc=v4(64, 30, 5, 16, 32, scope=LO)), S),
    ("scale 0", dict(scale=0.0), S),
    ("scale NaN", dict(scale=math.nan), S),
    ("scale too large", dict(scale=2.0 ** 101), S),
    ("window < 0", dict(window=-1), S),
    ("causal neither 0 nor 1", dict(causal=2), S),
    ("accumulating output", dict(o=v4(96, 2, 4, 64, 32, F32, ACC)), S),
    ("output heads", dict(o=v4(96, 2, 5, 64, 32, scope=LO)), S),
    ("output rows overlap", dict(o=v4(96, 2, 4, 64, 32, scope=LO, sh=32)), S),
    ("bf16 lse", dict(lse=v4(112, 2, 4, 64, 1, BF, LO)), D_),
    ("lse columns", dict(lse=v4(112, 2, 4, 64, 2, F32, LO)), S),
    ("output on the cache", dict(o=v4(48, 2, 4, 64, 32, scope=LO)), A),
    ("output on Q", dict(o=v4(80, 2, 4, 64, 32, scope=LO)), A),
    ("output on the table", dict(pages=pages(table=96 * MB + 64)), A),
    ("lse on the output", dict(lse=v4(96, 2, 4, 64, 1, F32, LO)), A),
    ("workspace size < 0", dict(ws=sbp.sbp_workspace_t(160 * MB, -1)), S),
    ("null workspace", dict(ws=sbp.sbp_workspace_t(None, MB)), N),
    ("misaligned workspace", dict(ws=sbp.sbp_workspace_t(160 * MB + 8, MB)), AL),
    ("workspace on the cache", dict(ws=sbp.sbp_workspace_t(64 * MB, MB)), A),
    ("workspace on the lengths", dict(ws=sbp.sbp_workspace_t(201 * MB, MB)), A),
    ("workspace on lse", dict(ws=sbp.sbp_workspace_t(112 * MB, MB)), A),
    ("more rows than a launch covers", dict(
        q=v4(80, 2, 10, 1 << 29, 32, sb=0, sh=0), o=v4(1 << 20, 2, 4, 1 << 29, 32, scope=LO),
        lse=None, pages=pages(1 << 55, 12, 2, 12, 1 << 56)), S),
]


@pytest.mark.parametrize("name,change,code", APPEND, ids=[c[0] for c in APPEND])
def test_append_refusals(name, change, code):
    with pytest.raises(sbp.SbpError) as e:
        append({**append_args(), **change})
    assert e.value.code == code


@pytest.mark.parametrize("name,change,code", ATTN, ids=[c[0] for c in ATTN])
def test_attention_refusals(name, change, code):
    with pytest.raises(sbp.SbpError) as e:
        attn({**attn_args(), **change})
    assert e.value.code == code


def test_packed_needs_one_batch():
    for args, call in ((append_args(), append), (attn_args(), attn)):
        with pytest.raises(sbp.SbpError) as e:
            call({**args, "pages": pages(q=201 * MB + 64, rows=201 * MB + 128)})
        assert e.value.code == S


def test_empty_calls_return():
    kw = dict(sh=2048, sb=20480)
    none = pages(None, 0, 0, 0, None)
    append({**append_args(), "k": v4(16, 0, 5, 64, 32, **kw), "v": v4(32, 0, 5, 64, 32, **kw),
            "q": v4(80, 0, 10, 64, 32, **kw), "qo": v4(96, 0, 4, 64, 32, scope=LO, **kw), "pages": none})
    attn({**attn_args(), "q": v4(80, 0, 10, 64, 32, **kw), "o": v4(96, 0, 4, 64, 32, scope=LO, **kw),
          "lse": None, "pages": none})
    # rows of no extent
    append({**append_args(), "k": v4(16, 2, 5, 0, 32, **kw), "v": v4(32, 2, 5, 0, 32, **kw),
            "q": v4(80, 2, 10, 0, 32, **kw), "qo": v4(96, 2, 4, 0, 32, scope=LO, **kw)})


# Parts of one tensor that share a span but no element are let through: the last defect of each of
# these calls is its number of rows, found after the operands' places.
def _too_many(c):
    c["pages"] = pages(1 << 55, 12, 2, 12, 1 << 56)
    return c


@pytest.mark.parametrize("vc", [
    v4(1 << 30, 30, 5, 16, 32),                                                    # apart
    v4(1024 + 16 * 5 * 32 * 2 / MB, 30, 5, 16, 32, sb=2 * 16 * 5 * 32, sh=32, ld=160),  # [2] in a page
], ids=["apart", "side by side"])
def test_keys_and_values_of_one_tensor(vc):
    kc = v4(1024, 30, 5, 16, 32, sb=2 * 16 * 5 * 32, sh=32, ld=160)
    c = _too_many({**append_args(), "k": v4(16, 2, 5, 1 << 28, 32, sb=0, sh=0),
                   "v": v4(32, 2, 5, 1 << 28, 32, sb=0, sh=0), "q": None, "qo": None, "rope": None,
                   "kc": kc, "vc": vc})
    # K and V of 2^28 rows reach over the caches' addresses here unless these lie past them
    kc.data, vc.data = kc.data + (1 << 45), vc.data + (1 << 45)
    c["p"], c["r"] = 1, 0
    with pytest.raises(sbp.SbpError) as e:
        append(c)
    assert e.value.code == S
