"""GPU tests of the torch wrappers' `stream` argument: calls on a stream that is not torch's
current one, with work of the current stream on both sides of them that reads and writes
blocks of the sizes that the call allocates."""
import threading

import pytest
import torch

from paper_2301_06813_amd import attention, inputs, linear, sbp

from helpers import say

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
M, K, N = 256, 512, 1024


def rn(shape, seed, dtype):
    return inputs.randn(shape, 1.0, seed, dtype, "cuda")


def gated(dtype):
    return rn((M, K), 1, dtype), rn((K, N), 2, dtype) / 16, rn((K, N), 3, dtype) / 16


def gated_fwd(dtype, save):
    T = gated(dtype)
    return (lambda **kw: linear.gated_fwd("COL", 1, 0, *T, save=save, **kw)), [(M, N)] * 3, dtype


def gated_bwd(dtype):
    T, dH = gated(dtype), rn((M, N), 4, dtype)
    _, G, U = linear.gated_fwd("COL", 1, 0, *T)
    return (lambda **kw: linear.gated_bwd("COL", 1, 0, dH, *T, G, U, **kw)), \
        [(2, M, N), (M, K), (K, N), (K, N)], dtype


def heads():
    return [rn((2, h, 300, 64), 5 + i, BF) for i, h in enumerate((8, 2, 2, 8))]


def attn_fwd():
    Q, K, V, _ = heads()
    return (lambda **kw: attention.core_fwd(Q, K, V, causal=True, **kw)), [Q.shape], BF


def attn_bwd():
    Q, K, V, dO = heads()
    O, lse = attention.core_fwd(Q, K, V, causal=True)
    return (lambda **kw: attention.core_bwd(dO, Q, K, V, O, lse, causal=True, **kw)), \
        [Q.shape, K.shape, V.shape], BF


def linear_fwd():
    X, W, _ = gated(BF)
    return (lambda **kw: linear.call("fwd", "COL", 1, 0, X, W, None, **kw)[:1]), [(M, N)], BF


def linear_bwd():
    (X, W, _), dY = gated(F32), rn((M, N), 4, F32)
    return (lambda **kw: linear.call_bwd_nd(("COL", "DP"), (1, 1), (0, 0), X, W, dY, **kw)[:2]), \
        [(M, K), (K, N)], F32


CALLS = {"gated forward, fp32": lambda: gated_fwd(F32, True),
         "gated forward, fp32, H only": lambda: gated_fwd(F32, False),
         "gated forward, bf16, H only": lambda: gated_fwd(BF, False),
         "gated backward, bf16": lambda: gated_bwd(BF),
         "gated backward, fp32": lambda: gated_bwd(F32),
         "attention forward": attn_fwd, "attention backward": attn_bwd,
         "linear forward": linear_fwd, "linear backward on a mesh, fp32": linear_bwd}


@pytest.mark.parametrize("name", CALLS)
def test_given_stream(name):
    call, blocks, dtype = CALLS[name]()
    busy = rn((4096, 4096), 9, F32)
    alloc = lambda: [torch.empty(s, dtype=dtype, device="cuda") for s in blocks]
    want = [t for t in call() if t is not None]
    side = torch.cuda.Stream()
    call(stream=side.cuda_stream)      # the stream's workspace is there
    torch.cuda.synchronize()
    for rep in range(3):
        say(name, "given stream", rep)
        # the current stream still reads blocks that it has given back when the call starts
        old = alloc()
        for i, t in enumerate(old):
            t.fill_(i + 1)
        side.wait_stream(torch.cuda.current_stream())
        for _ in range(8):
            busy @ busy
        sums = [t.clone() for t in old]
        del old, t
        got = [t for t in call(stream=side.cuda_stream) if t is not None]
        torch.cuda.synchronize()
        for i, t in enumerate(sums):
            assert bool((t == i + 1).all())
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        # the given stream is busy, and the current one fills new blocks after the call
        with torch.cuda.stream(side):
            for _ in range(8):
                busy @ busy
        got = [t for t in call(stream=side.cuda_stream) if t is not None]
        new = alloc() + alloc()
        for t in new:
            t.fill_(-3)
        torch.cuda.synchronize()
        assert len(got) == len(want) and all(torch.equal(a, b) for a, b in zip(got, want))
        assert all(bool((t == -3).all()) for t in new)
        # dropped while the current stream still uses them
        got = [t for t in call(stream=side.cuda_stream) if t is not None]
        torch.cuda.current_stream().wait_stream(side)
        for _ in range(8):
            busy @ busy
        kept = [t.clone() for t in got]
        del got, t
        call(stream=side.cuda_stream)
        with torch.cuda.stream(side):
            for s in blocks + blocks:
                torch.empty(s, dtype=dtype, device="cuda").fill_(5)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(kept, want))


def test_the_null_stream():
    # handle 0 is the null stream, also where another one is current
    T = gated(F32)
    want = linear.gated_fwd("COL", 1, 0, *T)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    say("null stream")
    with torch.cuda.stream(side):
        got = linear.gated_fwd("COL", 1, 0, *T, stream=0)
    torch.cuda.default_stream().synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_workspace_of_a_call(monkeypatch):
    # more query rows than the kept workspace holds statistics of: the call brings its own
    call, blocks, _ = attn_bwd()
    need = attention.bwd_workspace_bytes(2, 8, 300)
    want = call(ws=torch.empty(need, dtype=torch.uint8, device="cuda"))
    busy = rn((4096, 4096), 9, F32)
    side = torch.cuda.Stream()
    monkeypatch.setattr(sbp, "SBP_WORKSPACE_BYTES", need - 32)
    torch.cuda.synchronize()
    for rep in range(3):
        say("workspace of a call", rep)
        old = torch.full((need,), 7, dtype=torch.uint8, device="cuda")
        side.wait_stream(torch.cuda.current_stream())
        for _ in range(8):
            busy @ busy
        kept = old.clone()
        del old
        got = call(stream=side.cuda_stream)
        new = [torch.full((need,), 9, dtype=torch.uint8, device="cuda") for _ in range(4)]
        torch.cuda.synchronize()
        assert bool((kept == 7).all()) and all(bool((t == 9).all()) for t in new)
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_first_call_on_a_stream():
    # the workspace that is kept for a stream is allocated by its first call: not from a
    # block that the current stream has given back and still reads
    T = rn((16, 8192), 1, BF), rn((8192, 64), 2, BF), rn((8192, 64), 3, BF)   # a split reduction
    want = linear.gated_fwd("COL", 1, 0, *T)
    busy = rn((4096, 4096), 9, F32)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    say("first call")
    old = torch.full((sbp.SBP_WORKSPACE_BYTES,), 7, dtype=torch.uint8, device="cuda")
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(8):
        busy @ busy
    kept = old.clone()
    del old
    got = linear.gated_fwd("COL", 1, 0, *T, stream=side.cuda_stream)
    L = linear.layouts("COL", 1, 0)
    H = torch.empty((16, 64), dtype=BF, device="cuda")
    torch.cuda.synchronize()
    other = torch.cuda.Stream()
    old = torch.full((sbp.SBP_WORKSPACE_BYTES,), 7, dtype=torch.uint8, device="cuda")
    other.wait_stream(torch.cuda.current_stream())
    for _ in range(8):
        busy @ busy
    kept2 = old.clone()
    del old
    sbp.sbp_gated_fwd(sbp.view(T[0]), L["x"], sbp.view(T[1]), sbp.view(T[2]), L["w"],
                      sbp.SBP_ACT_SILU, sbp.view(H, sbp.SBP_LOCAL), stream=other.cuda_stream)
    torch.cuda.synchronize()
    assert bool((kept == 7).all()) and bool((kept2 == 7).all())
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and torch.equal(H, want[0])


def test_two_threads_on_one_stream():
    # calls of several launches that pass data through the kept workspace, made by two host
    # threads at once: row statistics and split partials must be the call's own
    work = []
    for seed in (20, 40):
        Q, K, V, dO = (rn((1, h, s, 64), seed + i, BF) for i, (h, s) in
                       enumerate(((8, 40), (2, 3000), (2, 3000), (8, 40))))
        X, Wg, Wu, dH = (rn(s, seed + 5 + i, BF) for i, s in
                         enumerate(((16, 4096), (4096, 96), (4096, 96), (16, 96))))

        def calls(Q=Q, K=K, V=V, dO=dO, X=X, Wg=Wg, Wu=Wu, dH=dH):
            O, lse = attention.core_fwd(Q, K, V)
            H, G, U = linear.gated_fwd("COL", 1, 0, X, Wg, Wu)
            return (O, lse, *attention.core_bwd(dO, Q, K, V, O, lse), H, G, U,
                    *linear.gated_bwd("COL", 1, 0, dH, X, Wg, Wu, G, U))

        work.append(calls)
    sbp.sbp_profile_begin(64)
    want = [f() for f in work]
    names = " ".join(n for n, _ in sbp.sbp_profile_end(64))
    assert all(n in names for n in ("core_join", "core_stat", "core_sum", "gated_join"))
    torch.cuda.synchronize()
    start, got = threading.Barrier(2), [[], []]

    def run(i):
        start.wait(30)
        for _ in range(100):
            got[i].append(work[i]())

    say("two threads")
    threads = [threading.Thread(target=run, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join(100)
    torch.cuda.synchronize()
    for i in range(2):
        assert len(got[i]) == 100
        for out in got[i]:
            assert all(torch.equal(a, b) for a, b in zip(out, want[i]))
