"""Which stream's memory the wrappers of rotary positions and of the paged cache allocate when
they are given a stream that is not torch's current one, and tensors of another device: on the CPU,
as in test_streams_host.py. Skipped wherever a GPU is visible."""
import pytest
import torch

from paper_2301_06813_amd import paged, rotary, sbp
from test_streams_host import BF, CALLER, F32, GIVEN, Elsewhere, Record

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="replaces torch's streams")
STREAMS = pytest.mark.parametrize("stream", [None, CALLER, GIVEN, 0])


def record(monkeypatch):
    r = Record(monkeypatch)
    monkeypatch.setattr(paged, "_EMPTY", torch.empty)
    monkeypatch.setattr(sbp, "sbp_paged_attn", r.library_call)
    for name in ("sbp_rope_fwd", "sbp_rope_bwd", "sbp_paged_append"):    # no workspace
        monkeypatch.setattr(sbp, name, lambda *a: r.library_call(*a, None))
    return r


def heads(*counts, dtype=BF):
    return [torch.zeros((2, h, 6, 8), dtype=dtype) for h in counts]


def cache(scope=sbp.SBP_GLOBAL):
    return paged.Cache(*(torch.zeros((9, 2, 4, 8), dtype=BF) for _ in range(2)), scope)


def step():
    return torch.zeros((2, 4), dtype=torch.int32), torch.tensor([6, 3], dtype=torch.int32)


@STREAMS
@pytest.mark.parametrize("given", [False, True], ids=["new outputs", "given outputs"])
@pytest.mark.parametrize("call", [rotary.fwd, rotary.bwd])
@pytest.mark.parametrize("both", [True, False])
def test_rotation(monkeypatch, both, call, given, stream):
    Q, K = heads(4, 2)
    K = K if both else None
    rope = rotary.Rope(8, device="cpu")
    out = (torch.zeros_like(Q), torch.zeros_like(K) if both else None) if given else None
    r = record(monkeypatch)
    got = call(rope, Q, K, pos=torch.zeros(2, dtype=torch.int32), out=out, out_dtype=F32, stream=stream)
    ins = [t for t in (Q, K, *(out or ())) if t is not None]
    if not given:
        r.check(got, ins, CALLER if stream is None else stream)
    assert (got[1] is None) == (not both)
    assert not given or all(a is b for a, b in zip(got, out))


@STREAMS
@pytest.mark.parametrize("given", [False, True], ids=["new output", "given output"])
def test_append(monkeypatch, given, stream):
    Q, K, V = heads(4, 2, 2)
    c, (table, lens), out = cache(), step(), torch.zeros_like(Q) if given else None
    r = record(monkeypatch)
    got = c.append(K, V, table, lens, Q=Q, rope=rotary.Rope(8, device="cpu"), out=out, stream=stream)
    (ran, views), = r.calls
    assert ran == (CALLER if stream is None else stream)
    if given:
        assert got is out and not r.blocks
    else:
        r.check((got,), (Q, K, V, c.k, c.v), CALLER if stream is None else stream)
    r.calls.clear()
    assert c.append(K, V, table, lens, stream=stream) is None and len(r.calls) == 1


@STREAMS
@pytest.mark.parametrize("given", [False, True], ids=["new output", "given output"])
@pytest.mark.parametrize("lse", [True, False])
def test_attend(monkeypatch, lse, given, stream):
    Q, = heads(4)
    c, (table, lens), out = cache(), step(), torch.zeros_like(Q) if given else None
    r = record(monkeypatch)
    got = c.attend(Q, table, lens, window=3, lse=lse, out=out, stream=stream)
    if given and not lse:
        assert not r.blocks
    else:
        r.check([t for t in got if t is not out], (Q, c.k, c.v, *([out] if given else ())),
                CALLER if stream is None else stream)
    assert (got[1] is None) == (not lse) and (not given or got[0] is out)


def test_tensors_on_another_device(monkeypatch):
    Q, K, V = heads(4, 2, 2)
    (table, lens), rope = step(), rotary.Rope(8, device="cpu")
    first = torch.tensor([0, 6, 6], dtype=torch.int32)
    pos, ws = torch.zeros(2, dtype=torch.int32), torch.zeros(4096, dtype=torch.uint8)
    c = cache()
    one = lambda t: t[:1]
    calls = {
        "fwd": (lambda Q, K, pos: rotary.fwd(rope, Q, K, pos=pos), (Q, K, pos)),
        "bwd": (lambda Q, K, pos: rotary.bwd(rope, Q, K, pos=pos), (Q, K, pos)),
        "append": (lambda K, V, Q, table, lens, first: c.append(
            K, V, table, lens, Q=Q, rope=rope, row_q=first), (one(K), one(V), one(Q), table, lens, first)),
        "attend": (lambda Q, table, lens, first, ws: c.attend(Q, table, lens, row_q=first, ws=ws),
                   (one(Q), table, lens, first, ws))}
    r = record(monkeypatch)
    for call, args in calls.values():
        call(*args)
    assert len(r.calls) == 4
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.Tensor, "device", property(lambda self: torch.device("cuda:0")))
    for call, args in calls.values():
        call(*args)
        for i in range(len(args)):
            with pytest.raises(ValueError, match="cuda:1"):
                call(*args[:i], args[i].as_subclass(Elsewhere), *args[i + 1:])
    assert len(r.calls) == 8


def test_window_that_is_no_int32(monkeypatch):
    Q, = heads(4)
    c, (table, lens) = cache(), step()
    r = record(monkeypatch)
    with pytest.raises(ValueError, match="int32"):
        c.attend(Q, table, lens, window=(1 << 32) + 3)      # not a window of 3
    assert not r.calls
    c.attend(Q, table, lens, window=(1 << 31) - 1)
    assert len(r.calls) == 1


@pytest.mark.parametrize("window", [-(1 << 32) + 3, -(1 << 31) - 1, 1 << 31, (1 << 40) + 1])
def test_windows_outside_int32_are_refused(monkeypatch, window):
    Q, = heads(4)
    c, (table, lens) = cache(), step()
    r = record(monkeypatch)
    with pytest.raises(ValueError, match="int32"):
        c.attend(Q, table, lens, window=window)       # its low 32 bits may be a window
    assert not r.calls
