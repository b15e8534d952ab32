"""Host-side checks of rotary positions: the table of frequencies against long double, and
refusals. Every refused case has exactly one defect, so no call reaches a kernel; fake device
addresses, those tests are skipped wherever a GPU is visible."""
import math

import numpy as np
import pytest

import rope_ref as ref
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


fake = pytest.mark.skipif(_gpu_visible(), reason="uses fake device addresses")

TABLES = [(64, dict()), (128, dict(base=500000.0)), (2, dict()), (40, dict(scaling="linear", factor=4.0)),
          (128, dict(scaling="base", factor=8.0)), (2, dict(scaling="base", factor=8.0)),
          (128, dict(scaling="turns", factor=8.0, low=1.0, high=4.0, context=8192.0)),
          (64, dict(scaling="pairs", factor=32.0, low=1.0, high=32.0, context=4096.0)),
          (6, dict(scaling="pairs", factor=2.0, low=5.0, high=6.0, context=64.0)),
          (80, dict(scaling="turns", factor=0.5, low=0.25, high=100.0, context=100.0))]


@pytest.mark.parametrize("dim,kw", TABLES)
def test_table_of_frequencies(dim, kw):
    c = {k: v for k, v in kw.items() if k != "scaling"}
    got = sbp.sbp_rope_turns(dim, scaling=sbp.ROPE_SCALINGS[kw.get("scaling")], **c)
    want = ref.freqs(dim, **kw) / ref.TAU
    assert len(got) == dim // 2
    for g, w in zip(got, want):
        # two long double computations of a number below 1: powers of 63 bits each
        off = np.longdouble(g) / np.longdouble(2) ** 64 - (w - np.floor(w))
        assert abs(off) <= 2.0 ** -61, (g, w)


def test_frequencies_fall():
    for dim, kw in TABLES:
        c = {k: v for k, v in kw.items() if k != "scaling"}
        t = sbp.sbp_rope_turns(dim, scaling=sbp.ROPE_SCALINGS[kw.get("scaling")], **c)
        assert all(a > b for a, b in zip(t, t[1:]))


BAD_TABLES = [dict(dim=0), dict(dim=3), dict(dim=130), dict(dim=-2), dict(base=1.0), dict(base=math.nan),
              dict(base=math.inf), dict(scaling=5), dict(scaling=-1), dict(scaling=1, factor=0.0),
              dict(scaling=2, factor=math.inf), dict(scaling=3, factor=math.nan),
              dict(scaling=3, factor=2.0, low=0.0), dict(scaling=3, factor=2.0, low=2.0, high=2.0),
              dict(scaling=4, factor=2.0, context=0.0), dict(scaling=4, factor=2.0, high=math.inf),
              dict(scaling=4, factor=2.0, low=math.nan), dict(scaling=3, factor=2.0, context=math.inf)]


@pytest.mark.parametrize("kw", BAD_TABLES, ids=str)
def test_refused_tables(kw):
    with pytest.raises(sbp.SbpError) as e:
        sbp.sbp_rope_turns(**{"dim": 64, **kw})
    assert e.value.code == sbp.SBP_ERR_SHAPE


def v4(at, B, H, R, C, dtype=BF, scope=GL, sb=None, sh=None, ld=None):
    ld = C if ld is None else ld
    sh = R * ld if sh is None else sh
    sb = H * sh if sb is None else sb
    return sbp.sbp_view4_t(None if at is None else int(at * MB), B, H, R, C, sb, sh, ld, dtype, scope)


def args():
    # 10 query heads on 5 key heads over p = 2: rank 1 has key heads 3, 4, query heads 6..9
    return dict(q=v4(16, 2, 10, 64, 32), k=v4(32, 2, 5, 64, 32),
                rope=sbp.sbp_rope_t(200 * MB, 32, 0, 1.0),
                at=sbp.sbp_places_t(201 * MB, 64, 1), qo=v4(64, 2, 4, 64, 32, scope=LO),
                ko=v4(80, 2, 2, 64, 32, scope=LO), p=2, r=1)


S, A, D_, N = sbp.SBP_ERR_SHAPE, sbp.SBP_ERR_ALIAS, sbp.SBP_ERR_DTYPE, sbp.SBP_ERR_NULL
CASES = [
    ("no rotation", dict(rope=None), N),
    ("no output", dict(qo=None), N),
    ("Ko without K", dict(k=None), N),
    ("K without Ko", dict(ko=None), N),
    ("null table", dict(rope=sbp.sbp_rope_t(None, 32, 0, 1.0)), N),
    ("misaligned table", dict(rope=sbp.sbp_rope_t(200 * MB + 4, 32, 0, 1.0)), sbp.SBP_ERR_ALIGN),
    ("odd dim", dict(rope=sbp.sbp_rope_t(200 * MB, 31, 0, 1.0)), S),
    ("dim 0", dict(rope=sbp.sbp_rope_t(200 * MB, 0, 0, 1.0)), S),
    ("dim past the head", dict(rope=sbp.sbp_rope_t(200 * MB, 34, 0, 1.0)), S),
    ("unknown order", dict(rope=sbp.sbp_rope_t(200 * MB, 32, 2, 1.0)), S),
    ("factor NaN", dict(rope=sbp.sbp_rope_t(200 * MB, 32, 0, math.nan)), S),
    ("rank out of range", dict(r=2), sbp.SBP_ERR_LAYOUT),
    ("no devices", dict(p=0), sbp.SBP_ERR_LAYOUT),
    ("scopes differ", dict(k=v4(32, 2, 5, 64, 32, scope=LO)), S),
    ("accumulating input", dict(q=v4(16, 2, 10, 64, 32, scope=ACC)), S),
    ("batches differ", dict(k=v4(32, 3, 5, 64, 32)), S),
    ("rows differ", dict(k=v4(32, 2, 5, 63, 32)), S),
    ("head dims differ", dict(k=v4(32, 2, 5, 64, 48)), S),
    ("query heads no multiple of key heads", dict(q=v4(16, 2, 12, 64, 32)), S),
    ("head dim 129", dict(q=v4(16, 2, 10, 64, 129), k=v4(32, 2, 5, 64, 129),
                          qo=v4(64, 2, 4, 64, 129, scope=LO), ko=v4(80, 2, 2, 64, 129, scope=LO)), S),
    ("input types differ", dict(k=v4(32, 2, 5, 64, 32, F32)), D_),
    ("output types differ", dict(ko=v4(80, 2, 2, 64, 32, F32, LO)), D_),
    ("bf16 outputs of fp32", dict(q=v4(16, 2, 10, 64, 32, F32), k=v4(32, 2, 5, 64, 32, F32)), D_),
    ("accumulating output", dict(qo=v4(64, 2, 4, 64, 32, F32, ACC), ko=v4(80, 2, 2, 64, 32, F32, LO)), S),
    ("output heads", dict(qo=v4(64, 2, 5, 64, 32, scope=LO)), S),
    ("output rows", dict(ko=v4(80, 2, 2, 60, 32, scope=LO)), S),
    ("output rows overlap", dict(qo=v4(64, 2, 4, 64, 32, scope=LO, ld=32, sh=32)), S),
    ("places: flag", dict(at=sbp.sbp_places_t(201 * MB, 64, 2)), S),
    ("places beyond 62 bits", dict(at=sbp.sbp_places_t(201 * MB, 1 << 60, 1)), S),
    ("places: negative ld", dict(at=sbp.sbp_places_t(201 * MB, -1, 0)), S),
    ("places: null", dict(at=sbp.sbp_places_t(None, 64, 1)), N),
    ("places: misaligned", dict(at=sbp.sbp_places_t(201 * MB + 2, 64, 1)), sbp.SBP_ERR_ALIGN),
    ("output on Q, other heads", dict(qo=v4(16, 2, 4, 64, 32, scope=LO)), A),
    ("output on K", dict(qo=v4(32, 2, 4, 64, 32, scope=LO)), A),
    ("outputs overlap", dict(ko=v4(64, 2, 2, 64, 32, scope=LO)), A),
    ("output on the positions", dict(at=sbp.sbp_places_t(64 * MB + 4096, 64, 1)), A),
    ("output on the table", dict(rope=sbp.sbp_rope_t(80 * MB, 32, 0, 1.0)), A),
    ("rank's part of Q, of another type", dict(
        q=v4(16, 2, 10, 64, 32), qo=v4(16 + 6 * 64 * 32 * 2 / MB, 2, 4, 64, 32, F32, LO, sb=10 * 64 * 32),
        ko=v4(80, 2, 2, 64, 32, F32, LO)), A),
    ("more rows than a launch covers", dict(
        q=v4(16, 1 << 8, 10, 1 << 22, 32, sb=0, sh=0, ld=32), k=v4(32, 1 << 8, 5, 1 << 22, 32, sb=0, sh=0),
        qo=v4(1 << 20, 1 << 8, 4, 1 << 22, 32, scope=LO), ko=v4(1 << 22, 1 << 8, 2, 1 << 22, 32, scope=LO),
        at=None), S),
]


@fake
@pytest.mark.parametrize("call", [sbp.sbp_rope_fwd, sbp.sbp_rope_bwd])
@pytest.mark.parametrize("name,change,code", CASES, ids=[c[0] for c in CASES])
def test_refusals(call, name, change, code):
    c = {**args(), **change}
    with pytest.raises(sbp.SbpError) as e:
        call(c["q"], c["k"], c["rope"], c["at"], c["qo"], c["ko"], c["p"], c["r"], stream=0)
    assert e.value.code == code


@fake
@pytest.mark.parametrize("call", [sbp.sbp_rope_fwd, sbp.sbp_rope_bwd])
def test_empty_calls_return(call):
    c = args()
    for rows, batch, heads in ((0, 2, 10), (64, 0, 10), (64, 2, 0)):
        n = 4 if heads else 0
        kw = dict(sh=2048, sb=20480)
        call(v4(16, batch, heads, rows, 32, **kw), v4(32, batch, heads // 2, rows, 32, **kw),
             c["rope"], None, v4(64, batch, n, rows, 32, scope=LO, **kw),
             v4(80, batch, n // 2, rows, 32, scope=LO, **kw), 2, 1, stream=0)


def _exact_turns(dim, base, scaling, factor, low, high, context):
    """The frequencies in turns a position, to 60 digits."""
    from decimal import Decimal as D, ROUND_CEILING, ROUND_FLOOR, localcontext
    with localcontext() as c:
        c.prec = 80
        tau = 2 * D("3.14159265358979323846264338327950288419716939937510582097494459230781640628620899862803")
        base, factor, low, high, context = (D(x) for x in (base, factor, low, high, context))
        b = base * factor ** (D(dim) / (dim - 2)) if scaling == "base" and dim > 2 else base
        f = [b ** (D(-2 * i) / dim) for i in range(dim // 2)]
        limited = lambda w: min(D(1), max(D(0), w))
        at = lambda n: dim * (context / (tau * n)).ln() / (2 * base.ln())
        first = max(D(0), at(high).to_integral_value(ROUND_FLOOR))
        last = min(D(dim - 1), at(low).to_integral_value(ROUND_CEILING))
        w = {"linear": lambda i: D(0), "turns": lambda i: limited((context * f[i] / tau - low) / (high - low)),
             "pairs": lambda i: 1 - limited((i - first) / max(last - first, D("0.001")))}.get(scaling, lambda i: D(1))
        return [(f[i] * w(i) + f[i] / factor * (1 - w(i))) / tau for i in range(dim // 2)]


EXACT = [dict(), dict(base=1.5), dict(base=1e12), dict(low=0.5, high=1.0, context=1e6)] + [
    dict(scaling=s, factor=x) for s in ("linear", "base", "turns", "pairs")
    for x in (1e6, 40.0, 2.0, 0.9, 0.25, 0.01, 1e-4, 2.0 ** -32)]


@pytest.mark.parametrize("dim", [2, 4, 22, 64, 128])
@pytest.mark.parametrize("kw", EXACT, ids=str)
def test_frequencies_keep_the_stated_bound(dim, kw):
    """2^-62 turns a position, 1 / factor times that for factors below 1."""
    from decimal import Decimal as D, localcontext
    kw = dict(dict(base=10000.0, scaling=None, factor=1.0, low=1.0, high=32.0, context=4096.0), **kw)
    got = sbp.sbp_rope_turns(dim, **{**kw, "scaling": sbp.ROPE_SCALINGS[kw["scaling"]]})
    with localcontext() as c:
        c.prec = 80
        bound = D(2) ** -62 * max(D(1), 1 / D(kw["factor"]))
        for g, w in zip(got, _exact_turns(dim, **kw)):
            off = (D(g) / D(2) ** 64 - w) % 1
            assert min(abs(off), 1 - abs(off)) <= bound, (g, w)


@fake
@pytest.mark.parametrize("call", [sbp.sbp_rope_fwd, sbp.sbp_rope_bwd])
@pytest.mark.parametrize("order", [sbp.SBP_ROPE_HALVES, sbp.SBP_ROPE_PAIRS])
@pytest.mark.parametrize("dim", [0, 1, 2])
@pytest.mark.parametrize("dtype,out", [(BF, BF), (BF, F32), (F32, F32)])
def test_a_head_of_one_column_has_no_pair(call, order, dim, dtype, out):
    c = {**args(), "q": v4(16, 1, 4, 7, 1, dtype), "k": v4(32, 1, 2, 7, 1, dtype),
         "qo": v4(64, 1, 4, 7, 1, out, LO), "ko": v4(80, 1, 2, 7, 1, out, LO),
         "rope": sbp.sbp_rope_t(200 * MB, dim, order, 1.0)}
    with pytest.raises(sbp.SbpError) as e:
        call(c["q"], c["k"], c["rope"], None, c["qo"], c["ko"], 1, 0, stream=0)
    assert e.value.code == S
