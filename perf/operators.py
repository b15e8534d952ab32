"""The operators between the linear layers of a Transformer layer, measured on
one MI355X: softmax attention of a device's heads and the gated feed-forward
block, each forward and backward.

``run`` makes one pass. In their plain form the operators are elementary torch
operations in fp32, rounded once to the outputs' type; with ``own`` set they
are the library's calls. ``exact`` gives the same outputs in 64 bits.

Fields of an attention case (``op`` "attn_fwd", "attn_bwd"):
  batch, heads, kv_heads   global head counts; heads / kv_heads query heads
                           share a key and value head
  p, r                     devices that split the heads, and this one
  seq_q, seq_k, dim        rows of Q, of K and V, and the head dimension
  causal, window           query i of a sequence sees keys up to its own place
                           counted from the sequences' ends, and with a window
                           the last `window` of those only
  ragged                   sequence b uses 1 - ragged b / batch of its rows (a
                           padded batch); 0: every row
  fused                    Q, K and V are parts of one [batch][seq][heads][dim]
                           activation (the output of a fused projection), else
                           tensors of their own, K and V as a cache keeps them
Fields of a gated case (``op`` "gated_fwd", "gated_bwd"): H = act(X Wg) * (X Wu)
  m, k, n                  X is m x k, Wg and Wu are k x n (global extents)
  sig, p, r                signature, devices, this device
  act                      "silu", "gelu" (its tanh form) or "relu"
  save                     forward: X Wg and X Wu are kept for the backward pass
  dtype                    "bf16" or "f32"
"""
from __future__ import annotations

import math

import torch

own = False


# ------------------------------------------------------------------ cases
def _attn(name, op, batch, heads, kv_heads, seq_q, seq_k, dim, causal=True, window=0, ragged=0.0,
          fused=False, p=1, r=0):
    c = dict(op=op, batch=batch, heads=heads, kv_heads=kv_heads, seq_q=seq_q, seq_k=seq_k,
             dim=dim, causal=causal, window=window, ragged=ragged, fused=fused, p=p, r=r)
    return c if name is None else dict(name=name, **c)


def _gated(name, op, m, k, n, sig="COL", p=1, r=0, act="silu", save=True, dtype="bf16"):
    c = dict(op=op, m=m, k=k, n=n, sig=sig, p=p, r=r, act=act, save=save, dtype=dtype)
    return c if name is None else dict(name=name, **c)


def listed():
    return [
        # one new token of 16 sequences against their caches of up to 4096
        _attn("attn_fwd_token", "attn_fwd", 16, 16, 4, 1, 4096, 64, ragged=0.75),
        # the Transformer's attention: 8 sequences of 1024, 16 heads of 64 over 8 devices
        _attn("attn_fwd_layer", "attn_fwd", 8, 16, 16, 1024, 1024, 64, fused=True, p=8),
        # one long sequence, four query heads to a key head
        _attn("attn_fwd_long", "attn_fwd", 1, 16, 4, 8192, 8192, 128, fused=True),
        # a small padded batch: odd lengths, a head dimension of 80, a window
        _attn("attn_bwd_padded", "attn_bwd", 5, 6, 2, 333, 333, 80, window=100, ragged=0.7,
              fused=True),
        # gradients of the Transformer's attention
        _attn("attn_bwd_layer", "attn_bwd", 8, 16, 16, 1024, 1024, 64, fused=True, p=8),
        # gradients of one long sequence
        _attn("attn_bwd_long", "attn_bwd", 1, 16, 4, 8192, 8192, 128, fused=True),
        # one token through a feed-forward block
        _gated("gated_fwd_token", "gated_fwd", 1, 1024, 4096, save=False),
        # 8192 tokens through a device's eighth of the Transformer's block, in training
        _gated("gated_fwd_layer", "gated_fwd", 8192, 1024, 4096, p=8, r=3),
        # a wide block (hidden 8192, 32768 over 8 devices)
        _gated("gated_fwd_wide", "gated_fwd", 8192, 8192, 32768, p=8),
        # fp32 training at sizes that are no multiple of anything
        _gated("gated_bwd_f32_odd", "gated_bwd", 513, 1000, 1375, act="gelu", dtype="f32"),
        # gradients of the Transformer's block, one device's share
        _gated("gated_bwd_layer", "gated_bwd", 8192, 1024, 512),
        # gradients of the wide block, one device's share
        _gated("gated_bwd_wide", "gated_bwd", 8192, 8192, 4096),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_attn(rng):
    op = rng.choice(("attn_fwd", "attn_bwd"))
    kv_heads = rng.choice((1, 2, 3, 4, 8, 16))
    heads = kv_heads * rng.choice((1, 1, 2, 4, 7))
    dim = rng.choice((64, 64, 128, 128, rng.randrange(8, 129)))
    seq_q = _log(rng, 1, 8192)
    token = op == "attn_fwd" and rng.random() < 0.3
    fused = not token and rng.random() < 0.6
    if token:
        seq_q = rng.choice((1, 1, 2, 5))
    seq_k = seq_q if fused else _log(rng, max(1, seq_q // 2), 8192)
    causal = rng.random() < 0.7
    window = _log(rng, 16, 4096) if causal and rng.random() < 0.2 else 0
    ragged = round(rng.uniform(0.1, 0.9), 2) if rng.random() < 0.4 else 0.0
    p = rng.choice((1, 1, kv_heads))
    return _attn(None, op, _log(rng, 1, 32), heads, kv_heads, seq_q, seq_k, dim, causal, window,
                 ragged, fused, p, rng.randrange(p))


def _draw_gated(rng):
    op = rng.choice(("gated_fwd", "gated_bwd"))
    k, n = _log(rng, 64, 8192), _log(rng, 64, 8192)
    if rng.random() < 0.75:
        k, n = max(64, k // 64 * 64), max(64, n // 64 * 64)
    m = rng.randrange(1, 33) if rng.random() < 0.25 else _log(rng, 1, 8192)
    p = rng.choice((1, 2, 8)) if op == "gated_fwd" else 1
    return _gated(None, op, m, k, n, rng.choice(("COL", "DP")), p, rng.randrange(p),
                  rng.choice(("silu", "silu", "gelu", "relu")), op == "gated_bwd" or
                  rng.random() < 0.6, "f32" if rng.random() < 0.2 else "bf16")


def draw(rng):
    most = {}
    for c in listed():
        w, o = work(c), most.setdefault(c["op"], {"bytes": 0, "flops": 0})
        for f in o:
            o[f] = max(o[f], w[f])
    while True:
        c = _draw_attn(rng) if rng.random() < 0.5 else _draw_gated(rng)
        w = work(c)
        # fp32 products run at a fifteenth of the rate of bf16 ones
        cost = w["flops"] * (15 if c.get("dtype") == "f32" else 1)
        scores = 0
        if c["op"].startswith("attn"):   # the plain form holds every score
            scores = c["batch"] * (c["heads"] // c["p"]) * c["seq_q"] * c["seq_k"]
        if cost <= most[c["op"]]["flops"] and w["bytes"] <= most[c["op"]]["bytes"] and \
                scores <= 16 * 8192 * 8192:
            return c


def _split(n, p, r):
    """[offset, length) of the r-th of p balanced blocks."""
    return r * (n // p) + min(r, n % p), n // p + (r < n % p)


def _lens(c, seq):
    return [max(1, int(round(seq * (1.0 - c["ragged"] * b / c["batch"])))) for b in range(c["batch"])]


def _pairs(c):
    """Pairs of a query and a key that it sees, of one head, over the batch."""
    total = 0
    lq = _lens(c, c["seq_q"]) if c["fused"] else [c["seq_q"]] * c["batch"]
    for q, k in zip(lq, _lens(c, c["seq_k"])):
        for i in range(q):
            hi = min(k, i + 1 + k - q) if c["causal"] else k
            lo = max(0, i + 1 + k - q - c["window"]) if c["window"] else 0
            total += max(0, hi - lo)
    return total


def work(case):
    """What a pass has to read, write and compute: a product of two numbers and
    its sum are two operations; exponentials and activations are left out."""
    c = case
    if c["op"].startswith("attn"):
        hk = _split(c["kv_heads"], c["p"], c["r"])[1]
        h = hk * (c["heads"] // c["kv_heads"])
        lq = sum(_lens(c, c["seq_q"])) if c["fused"] else c["batch"] * c["seq_q"]
        lk = sum(_lens(c, c["seq_k"]))
        q, kv, st = 2 * h * lq * c["dim"], 2 * hk * lk * c["dim"], 4 * h * lq
        pairs = _pairs(c) * h
        if c["op"] == "attn_fwd":
            return {"bytes": 2 * q + 2 * kv + st, "flops": 4 * c["dim"] * pairs}
        return {"bytes": 4 * q + 4 * kv + st, "flops": 10 * c["dim"] * pairs}
    m = _split(c["m"], c["p"], c["r"])[1] if c["sig"] == "DP" else c["m"]
    n = _split(c["n"], c["p"], c["r"])[1] if c["sig"] == "COL" else c["n"]
    k, b = c["k"], 4 if c["dtype"] == "f32" else 2
    if c["op"] == "gated_fwd":
        return {"bytes": b * (m * k + 2 * k * n + (3 if c["save"] else 1) * m * n),
                "flops": 4 * m * k * n}
    return {"bytes": b * (2 * m * k + 4 * k * n + 3 * m * n), "flops": 8 * m * k * n}


# ----------------------------------------------------------------- inputs
def _randn(shape, seed, dtype, std=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)


def prepare(case, seed):
    c = dict(case)
    s = {"case": c}
    if c["op"].startswith("attn"):
        B, H, Hk, D = c["batch"], c["heads"], c["kv_heads"], c["dim"]
        if c["fused"]:
            act = _randn((B, c["seq_q"], H + 2 * Hk, D), 10 * seed + 1, torch.bfloat16)
            act = act.permute(0, 2, 1, 3)
            s["Q"], s["K"], s["V"] = act[:, :H], act[:, H:H + Hk], act[:, H + Hk:]
        else:
            s["Q"] = _randn((B, H, c["seq_q"], D), 10 * seed + 1, torch.bfloat16)
            s["K"] = _randn((B, Hk, c["seq_k"], D), 10 * seed + 2, torch.bfloat16)
            s["V"] = _randn((B, Hk, c["seq_k"], D), 10 * seed + 3, torch.bfloat16)
        i32 = dict(dtype=torch.int32, device="cuda")
        s["len_k"] = torch.tensor(_lens(c, c["seq_k"]), **i32) if c["ragged"] else None
        s["len_q"] = torch.tensor(_lens(c, c["seq_q"]), **i32) if c["ragged"] and c["fused"] else None
        s["scale"] = 1.0 / math.sqrt(D)
        if c["op"] == "attn_bwd":
            O, lse = _plain_attn_fwd(s)
            h = O.shape[1]
            dO = _randn((B, c["seq_q"], h, D), 10 * seed + 4, torch.bfloat16).permute(0, 2, 1, 3)
            s["O"], s["lse"], s["dO"] = O, lse, dO
        return s
    dt = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
    m, k, n = c["m"], c["k"], c["n"]
    s["X"] = _randn((m, k), 10 * seed + 1, dt)
    s["Wg"] = _randn((k, n), 10 * seed + 2, dt, 1.0 / math.sqrt(k))
    s["Wu"] = _randn((k, n), 10 * seed + 3, dt, 1.0 / math.sqrt(k))
    if c["op"] == "gated_bwd":
        X, Wg, Wu = s["X"].float(), s["Wg"].float(), s["Wu"].float()
        s["G"], s["U"] = (X @ Wg).to(dt), (X @ Wu).to(dt)
        s["dH"] = _randn((m, n), 10 * seed + 4, dt)
    return s


# ------------------------------------------------------------- plain forms
def _rank_heads(s):
    """This device's heads of Q, K and V (the others where they are global)."""
    c = s["case"]
    off, hk = _split(c["kv_heads"], c["p"], c["r"])
    g = c["heads"] // c["kv_heads"]
    return (s["Q"][:, off * g:(off + hk) * g], s["K"][:, off:off + hk], s["V"][:, off:off + hk],
            hk, g)


def _seen(s, sq, sk):
    """[batch or 1][1][1][sq][sk] truth values: query i sees key j."""
    c = s["case"]
    i = torch.arange(sq, device="cuda").view(1, sq, 1)
    j = torch.arange(sk, device="cuda").view(1, 1, sk)
    lq = s["len_q"].view(-1, 1, 1).long() if s["len_q"] is not None else sq
    lk = s["len_k"].view(-1, 1, 1).long() if s["len_k"] is not None else sk
    seen = (i < lq) & (j < lk)
    if c["causal"]:
        seen = seen & (j <= i + (lk - lq))
    if c["window"]:
        seen = seen & (j > i + (lk - lq) - c["window"])
    return seen[:, None, None]


def _plain_attn_fwd(s):
    Q, K, V, hk, g = _rank_heads(s)
    B, _, sq, D = Q.shape
    sk = K.shape[2]
    q = Q.float().reshape(B, hk, g * sq, D)
    k, v = K.float().contiguous(), V.float().contiguous()
    x = (q @ k.transpose(2, 3)).view(B, hk, g, sq, sk) * s["scale"]
    x = x.masked_fill(~_seen(s, sq, sk), -math.inf)
    top = x.amax(-1, keepdim=True)
    x = torch.exp(x - torch.where(top == -math.inf, 0.0, top))
    total = x.sum(-1, keepdim=True)
    lse = torch.where(total > 0, top + torch.log(total), -math.inf).view(B, hk * g, sq)
    x = x / torch.where(total > 0, total, 1.0)
    o = (x.view(B, hk, g * sq, sk) @ v).view(B, hk * g, sq, D)
    return o.to(Q.dtype), lse


def _plain_attn_bwd(s):
    Q, K, V, hk, g = _rank_heads(s)
    B, _, sq, D = Q.shape
    sk = K.shape[2]
    q = Q.float().reshape(B, hk, g * sq, D)
    k, v = K.float().contiguous(), V.float().contiguous()
    do = s["dO"].float().reshape(B, hk, g * sq, D)
    o = s["O"].float().reshape(B, hk, g * sq, D)
    lse = s["lse"].view(B, hk, g, sq, 1)
    seen = _seen(s, sq, sk)
    P = (q @ k.transpose(2, 3)).view(B, hk, g, sq, sk) * s["scale"]
    P = torch.exp(P - torch.where(lse == -math.inf, 0.0, lse)).masked_fill(~seen, 0.0)
    P = P.view(B, hk, g * sq, sk)
    dV = P.transpose(2, 3) @ do
    dS = do @ v.transpose(2, 3) - (do * o).sum(-1, keepdim=True)
    dS = dS * P
    dQ = (dS @ k) * s["scale"]
    dK = (dS.transpose(2, 3) @ q) * s["scale"]
    return dQ.view(B, hk * g, sq, D).to(Q.dtype), dK.to(K.dtype), dV.to(V.dtype)


def _act(x, act):
    """act(x) and its derivative."""
    if act == "relu":
        on = (x > 0).to(x.dtype)
        return x * on, on
    if act == "silu":
        z = torch.sigmoid(x)
        return x * z, z * (1 + x * (1 - z))
    a, b = 2 * math.sqrt(2 / math.pi), 0.044715   # x sigmoid(a (x + b x^3)): the tanh form
    z = torch.sigmoid(a * (x + b * x * x * x))
    return x * z, z + x * z * (1 - z) * a * (1 + 3 * b * x * x)


def _shares(s):
    """This device's shares of X, Wg and Wu."""
    c = s["case"]
    X, Wg, Wu = s["X"], s["Wg"], s["Wu"]
    if c["sig"] == "DP":
        off, m = _split(c["m"], c["p"], c["r"])
        return X[off:off + m], Wg, Wu
    off, n = _split(c["n"], c["p"], c["r"])
    return X, Wg[:, off:off + n], Wu[:, off:off + n]


def _plain_gated_fwd(s):
    X, Wg, Wu = _shares(s)
    dt = X.dtype
    X = X.float()
    G, U = X @ Wg.float(), X @ Wu.float()
    H = _act(G, s["case"]["act"])[0] * U
    return (H.to(dt), G.to(dt), U.to(dt)) if s["case"]["save"] else (H.to(dt),)


def _plain_gated_bwd(s):
    X, Wg, Wu = _shares(s)
    dt = X.dtype
    X, Wg, Wu = X.float(), Wg.float(), Wu.float()
    G, U, dH = s["G"].float(), s["U"].float(), s["dH"].float()
    a, da = _act(G, s["case"]["act"])
    dG, dU = dH * U * da, dH * a
    dX = dG @ Wg.t() + dU @ Wu.t()
    return dX.to(dt), (X.t() @ dG).to(dt), (X.t() @ dU).to(dt)


# -------------------------------------------------------------------- run
def run(state):
    s, c = state, state["case"]
    if own:
        from paper_2301_06813_amd import attention, linear
        if c["op"] == "attn_fwd":
            return attention.core_fwd(s["Q"], s["K"], s["V"], c["p"], c["r"], scale=s["scale"],
                                      causal=c["causal"], window=c["window"], len_q=s["len_q"],
                                      len_k=s["len_k"])
        if c["op"] == "attn_bwd":
            return attention.core_bwd(s["dO"], s["Q"], s["K"], s["V"], s["O"], s["lse"], c["p"],
                                      c["r"], scale=s["scale"], causal=c["causal"],
                                      window=c["window"], len_q=s["len_q"], len_k=s["len_k"])
        if c["op"] == "gated_fwd":
            H, G, U = linear.gated_fwd(c["sig"], c["p"], c["r"], s["X"], s["Wg"], s["Wu"],
                                       c["act"], save=c["save"])
            return (H, G, U) if c["save"] else (H,)
        return linear.gated_bwd(c["sig"], c["p"], c["r"], s["dH"], s["X"], s["Wg"], s["Wu"],
                                s["G"], s["U"], c["act"])
    return {"attn_fwd": _plain_attn_fwd, "attn_bwd": _plain_attn_bwd,
            "gated_fwd": _plain_gated_fwd, "gated_bwd": _plain_gated_bwd}[c["op"]](s)


# ------------------------------------------------------------------ exact
def _exact_attn(s):
    """One head of one sequence at a time, over the rows and keys that exist."""
    c = s["case"]
    Q, K, V, hk, g = _rank_heads(s)
    B, H, sq, D = Q.shape
    sk = K.shape[2]
    f64 = dict(dtype=torch.float64, device="cuda")
    bwd = c["op"] == "attn_bwd"
    O, lse = torch.zeros((B, H, sq, D), **f64), torch.full((B, H, sq), -math.inf, **f64)
    dQ, dK, dV = torch.zeros((B, H, sq, D), **f64), torch.zeros((B, hk, sk, D), **f64), \
        torch.zeros((B, hk, sk, D), **f64)
    lens_q = _lens(c, sq) if c["ragged"] and c["fused"] else [sq] * B
    lens_k = _lens(c, sk) if c["ragged"] else [sk] * B
    for b in range(B):
        nq, nk = lens_q[b], lens_k[b]
        last = torch.arange(nq, device="cuda") + (nk - nq)     # the last key that a row sees
        keys = torch.arange(nk, device="cuda")
        hidden = torch.zeros((nq, nk), dtype=torch.bool, device="cuda")
        if c["causal"]:
            hidden |= keys[None, :] > last[:, None]
        if c["window"]:
            hidden |= keys[None, :] <= last[:, None] - c["window"]
        for h in range(H):
            q, k, v = Q[b, h, :nq].double(), K[b, h // g, :nk].double(), V[b, h // g, :nk].double()
            x = torch.mm(q, k.t().contiguous()).mul_(s["scale"])
            x[hidden] = -math.inf
            if not bwd:
                z = torch.logsumexp(x, 1)
                w = torch.exp(x - torch.where(z == -math.inf, torch.zeros_like(z), z)[:, None])
                lse[b, h, :nq], O[b, h, :nq] = z, torch.mm(w, v)
                continue
            z, do = s["lse"][b, h, :nq].double(), s["dO"][b, h, :nq].double()
            w = torch.exp(x - torch.where(z == -math.inf, torch.zeros_like(z), z)[:, None])
            inner = torch.sum(do * s["O"][b, h, :nq].double(), 1)
            dx = w * (torch.mm(do, v.t().contiguous()) - inner[:, None]) * s["scale"]
            dQ[b, h, :nq] = torch.mm(dx, k)
            dK[b, h // g, :nk] += torch.mm(dx.t().contiguous(), q)
            dV[b, h // g, :nk] += torch.mm(w.t().contiguous(), do)
    return (dQ, dK, dV) if bwd else (O, lse)


def _exact_gated(s):
    c = s["case"]
    X, Wg, Wu = (t.double() for t in _shares(s))

    def gate(x):
        if c["act"] == "relu":
            return torch.clamp(x, min=0.0)
        if c["act"] == "silu":
            return x / (1.0 + torch.exp(-x))
        return 0.5 * x * (1.0 + torch.tanh(math.sqrt(2 / math.pi) * (x + 0.044715 * x ** 3)))

    if c["op"] == "gated_fwd":
        G, U = torch.mm(X, Wg), torch.mm(X, Wu)
        H = gate(G) * U
        return (H, G, U) if c["save"] else (H,)
    G = s["G"].double().requires_grad_(True)
    U, dH = s["U"].double(), s["dH"].double()
    with torch.enable_grad():
        a = gate(G)
        dG, = torch.autograd.grad(a, G, dH * U)
    dU = dH * a.detach()
    dX = torch.mm(dG, Wg.t().contiguous()) + torch.mm(dU, Wu.t().contiguous())
    Xt = X.t().contiguous()
    return dX, torch.mm(Xt, dG), torch.mm(Xt, dU)


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_attn(s) if case["op"].startswith("attn") else _exact_gated(s)
