"""Which stream's memory the torch wrappers allocate when they are given a stream that is not
torch's current one: on the CPU, with torch's streams and the library's calls replaced by
records of what was allocated and called where. Skipped wherever a GPU is visible."""
import contextlib
import threading

import pytest
import torch

from paper_2301_06813_amd import attention, linear, sbp

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="replaces torch's streams")
CALLER, GIVEN = 7, 9
BF, F32 = torch.bfloat16, torch.float32


class Stream:
    def __init__(self, handle):
        self.cuda_stream = handle


class Record:
    """Allocations (memory range, stream), library calls (stream, pointers), recorded uses."""

    def __init__(self, monkeypatch):
        self.stream, self.blocks, self.calls, self.uses, self.kept = CALLER, [], [], [], []
        patch = monkeypatch.setattr

        @contextlib.contextmanager
        def inside(s):
            was, self.stream = self.stream, s.cuda_stream
            yield
            self.stream = was

        patch(sbp, "current_stream", lambda: self.stream)
        patch(torch.cuda, "current_stream", lambda *a: Stream(self.stream))
        patch(torch.cuda, "default_stream", lambda *a: Stream(0))
        patch(torch.cuda, "ExternalStream", Stream)
        patch(torch.cuda, "stream", inside)
        patch(torch.cuda, "current_device", lambda: None)
        patch(torch.Tensor, "new_empty", self.allocating(torch.Tensor.new_empty))
        patch(torch.Tensor, "record_stream",
              lambda t, s: self.uses.append((t.data_ptr(), s.cuda_stream)))
        empty = self.allocating(torch.empty)
        patch(torch, "empty", empty)
        patch(attention, "_EMPTY", empty)
        patch(sbp, "_default_ws", {})
        for name in ("sbp_gated_fwd", "sbp_gated_bwd", "sbp_attn_core_fwd", "sbp_attn_core_bwd",
                     "sbp_linear_fwd", "sbp_linear_bwd", "sbp_nd_linear_fwd", "sbp_nd_linear_bwd"):
            patch(sbp, name, self.library_call)

    def allocating(self, make):
        def new(*a, **kw):
            kw.pop("device", None)
            t = make(*a, **kw)
            self.kept.append(t)    # no address comes twice
            self.blocks.append((t.data_ptr(), t.numel() * t.element_size(), self.stream))
            return t
        return new

    def library_call(self, *args):
        stream, ws = args[-2:]
        views = [a.data for a in args if isinstance(a, (sbp.sbp_view_t, sbp.sbp_view4_t))]
        if isinstance(ws, torch.Tensor):
            views.append(ws.data_ptr())
        self.calls.append((self.stream if stream is None else stream, views))

    def check(self, out, inputs, stream):
        """Everything that the call wrote to is of `stream`'s memory, it ran there, and what
        it returned is recorded for the caller's stream (another one than `stream`)."""
        (ran, views), = self.calls
        assert ran == stream
        given = {t.data_ptr() for t in inputs}
        written = [v for v in views if v not in given]
        assert written
        for v in written:
            owner, = [s for at, n, s in self.blocks if at <= v < at + n]
            assert owner == stream
        for t in out:
            assert t is None or stream == CALLER or (t.data_ptr(), CALLER) in self.uses
        assert self.stream == CALLER


def gated(dtype):
    return (torch.zeros((6, 8), dtype=dtype), torch.zeros((8, 4), dtype=dtype),
            torch.zeros((8, 4), dtype=dtype))


@pytest.mark.parametrize("stream", [None, CALLER, GIVEN, 0])
@pytest.mark.parametrize("save", [True, False])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_gated_forward(monkeypatch, dtype, save, stream):
    r, T = Record(monkeypatch), gated(dtype)
    out = linear.gated_fwd("COL", 1, 0, *T, save=save, stream=stream)
    r.check(out, T, CALLER if stream is None else stream)


@pytest.mark.parametrize("stream", [None, CALLER, GIVEN, 0])
@pytest.mark.parametrize("given", [False, True], ids=["new outputs", "given outputs"])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_gated_backward(monkeypatch, dtype, given, stream):
    X, Wg, Wu = gated(dtype)
    dH, G, U = (torch.zeros((6, 4), dtype=dtype) for _ in range(3))
    out = [torch.zeros(t.shape, dtype=dtype) for t in (X, Wg, Wu)] if given else None
    r = Record(monkeypatch)
    got = linear.gated_bwd("COL", 1, 0, dH, X, Wg, Wu, G, U, out=out, stream=stream)
    r.check(got, (X, Wg, Wu, dH, G, U, *(out or ())), CALLER if stream is None else stream)
    assert not given or all(a is b for a, b in zip(got, out))


def heads(*counts):
    return [torch.zeros((2, h, 6, 8), dtype=BF) for h in counts]


@pytest.mark.parametrize("stream", [None, CALLER, GIVEN, 0])
@pytest.mark.parametrize("given", [False, True], ids=["new outputs", "given output"])
def test_attention_forward(monkeypatch, given, stream):
    Q, K, V = heads(4, 2, 2)
    out = torch.zeros_like(Q) if given else None
    lens = torch.tensor([6, 3], dtype=torch.int32)
    r = Record(monkeypatch)
    got = attention.core_fwd(Q, K, V, causal=True, window=3, len_k=lens, out=out, stream=stream)
    r.check(got, (Q, K, V, *([out] if given else ())), CALLER if stream is None else stream)
    assert not given or got[0] is out


@pytest.mark.parametrize("stream", [None, CALLER, GIVEN, 0])
@pytest.mark.parametrize("own", [False, True], ids=["kept workspace", "workspace of the call"])
def test_attention_backward(monkeypatch, own, stream):
    Q, K, V, dO, O = heads(4, 2, 2, 4, 4)
    lse = torch.zeros((2, 4, 6))
    if own:
        monkeypatch.setattr(sbp, "SBP_WORKSPACE_BYTES", 64)
    r = Record(monkeypatch)
    got = attention.core_bwd(dO, Q, K, V, O, lse, scale=0.5, stream=stream)
    r.check(got, (Q, K, V, dO, O, lse), CALLER if stream is None else stream)
    assert len(r.blocks) == 3 + own


def test_kept_workspace(monkeypatch):
    # of the stream's own memory, whichever stream is current when it is first needed
    monkeypatch.setattr(sbp, "SBP_WORKSPACE_BYTES", 4096)
    r = Record(monkeypatch)
    for stream in (GIVEN, 0, CALLER):
        ws = sbp.default_workspace(stream)
        (at, _, owner), = [b for b in r.blocks if b[0] == ws.data]
        assert owner == stream and r.stream == CALLER
        assert sbp.default_workspace(stream).data == at
    assert len(r.blocks) == 3


def test_threads_keep_workspaces_of_their_own(monkeypatch):
    # two threads that are there at once, on one stream: a call's launches may come between
    # those of the other's call
    monkeypatch.setattr(sbp, "SBP_WORKSPACE_BYTES", 4096)
    Record(monkeypatch)
    found, both = {}, threading.Barrier(2)

    def work(i):
        found[i] = [sbp.default_workspace(CALLER).data for _ in range(2)]
        both.wait(30)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join(60)
    mine = sbp.default_workspace(CALLER).data
    assert found[0][0] == found[0][1] and found[1][0] == found[1][1]
    assert len({found[0][0], found[1][0], mine}) == 3


@pytest.mark.parametrize("stream", [None, CALLER, GIVEN, 0])
@pytest.mark.parametrize("nd", [False, True], ids=["1-D", "mesh"])
def test_linear(monkeypatch, nd, stream):
    X, W, dY = torch.zeros((6, 8)), torch.zeros((8, 4)), torch.zeros((6, 4))
    at = (("COL", "DP"), (1, 1), (0, 0)) if nd else ("COL", 1, 0)
    fwd, bwd = (linear.call_nd, linear.call_bwd_nd) if nd else (linear.call, linear.call_bwd)
    for make in (lambda: fwd("fwd", *at, X, W, None, stream=stream)[:1],
                 lambda: bwd(*at, X, W, dY, stream=stream)[:2]):
        with monkeypatch.context() as m:
            r = Record(m)
            r.check(make(), (X, W, dY), CALLER if stream is None else stream)


class Elsewhere(torch.Tensor):
    """A tensor of another device."""
    device = property(lambda self: torch.device("cuda:1"))


@pytest.mark.parametrize("call", ["gated_fwd", "gated_bwd", "core_fwd", "core_bwd"])
def test_workspace_on_another_device(monkeypatch, call):
    X, Wg, Wu = gated(BF)
    dH = torch.zeros((6, 4), dtype=BF)
    Q, K, V, dO = heads(4, 2, 2, 4)
    ws = torch.zeros(4096, dtype=torch.uint8)
    r = Record(monkeypatch)
    make = {"gated_fwd": lambda w: linear.gated_fwd("COL", 1, 0, X, Wg, Wu, ws=w),
            "gated_bwd": lambda w: linear.gated_bwd("COL", 1, 0, dH, X, Wg, Wu, dH, dH, ws=w),
            "core_fwd": lambda w: attention.core_fwd(Q, K, V, ws=w),
            "core_bwd": lambda w: attention.core_bwd(dO, Q, K, V, dO, torch.zeros((2, 4, 6)), ws=w)}[call]
    for good in (None, ws, sbp.NO_WORKSPACE):
        make(good)
    assert len(r.calls) == 3
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.Tensor, "device", property(lambda self: torch.device("cuda:0")))
    make(ws)
    with pytest.raises(ValueError, match="cuda:1"):
        make(ws.as_subclass(Elsewhere))
    assert len(r.calls) == 4
