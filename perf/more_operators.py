"""Rotary positions and attention over a paged cache, measured on one MI355X:
the rotation of Q and K (forward and backward), appending a step's keys and values
to the cache with the rotation applied on the way, and the attention of the new
tokens over the cache.

``run`` makes one pass. In their plain form the operators are elementary torch
operations in fp32 (angles in 64 bits), rounded once to the outputs' type; with
``own`` set they are the library's calls. ``exact`` gives the same outputs in 64 bits.

Fields of every case:
  op                       "rope_fwd", "rope_bwd", "append", "paged"
  batch, heads, kv_heads   sequences; global head counts
  p, r                     devices that split the heads, and this one
  seq, dim                 new tokens of a sequence, the head dimension
  rot, order               rotated columns of a head (0: none), and which make a pair:
                           "halves" (i, i + rot / 2) or "pairs" (2 i, 2 i + 1)
  scaling                  of the frequencies: "", "linear", "base", "turns", "pairs"
Rotations (Q and K are parts of a fused [batch][seq][heads][dim] activation):
  pos                      "none": row i is at place i; "first": from a place per
                           sequence on; "rows": a place per row
  far                      the largest place
  dtype                    "bf16" or "f32"
Append and attention over the cache (bf16):
  cached                   tokens that the longest sequence has, the new ones included
  page                     tokens of a page
  ragged                   sequence b has 1 - ragged b / batch of them
  layout                   a page's memory: "token" [row][head][dim], "head" [head][row][dim]
  chunks                   0: a padded batch, `seq` new tokens of every sequence; else packed
                           rows: the first `chunks` sequences bring up to `seq` tokens, the
                           others one each
  causal, window           as in the attention of whole sequences
"""
from __future__ import annotations

import math

import torch

own = False


# ------------------------------------------------------------------ cases
def _rope(name, op, batch, heads, kv_heads, seq, dim, rot=None, order="halves", scaling="",
          pos="none", far=0, dtype="bf16", p=1, r=0):
    c = dict(op=op, batch=batch, heads=heads, kv_heads=kv_heads, seq=seq, dim=dim,
             rot=dim if rot is None else rot, order=order, scaling=scaling, pos=pos,
             far=max(far, seq), dtype=dtype, p=p, r=r)
    return c if name is None else dict(name=name, **c)


def _paged(name, op, batch, heads, kv_heads, seq, dim, cached, page, ragged=0.0, layout="token",
           chunks=0, causal=True, window=0, rot=0, order="halves", scaling="", p=1, r=0):
    c = dict(op=op, batch=batch, heads=heads, kv_heads=kv_heads, seq=seq, dim=dim, cached=cached,
             page=page, ragged=ragged, layout=layout, chunks=chunks, causal=causal, window=window,
             rot=rot, order=order, scaling=scaling, p=p, r=r)
    return c if name is None else dict(name=name, **c)


def listed():
    return [
        # one new token of 16 sequences
        _rope("rope_fwd_token", "rope_fwd", 16, 16, 4, 1, 64, pos="first", far=4096),
        # the Transformer's Q and K: 8 sequences of 1024, 16 heads of 64
        _rope("rope_fwd_layer", "rope_fwd", 8, 16, 16, 1024, 64),
        # one long sequence of a wide model, far positions, scaled frequencies
        _rope("rope_fwd_long", "rope_fwd", 1, 64, 8, 32768, 128, scaling="turns", pos="first",
              far=1 << 20),
        # fp32 gradients of packed documents, part of an odd head
        _rope("rope_bwd_f32_odd", "rope_bwd", 5, 6, 2, 333, 80, rot=40, order="pairs",
              pos="rows", far=1000, dtype="f32"),
        # gradients of the Transformer's Q and K
        _rope("rope_bwd_layer", "rope_bwd", 8, 16, 16, 1024, 64),
        # a serving step's single tokens
        _paged("append_token", "append", 16, 16, 4, 1, 64, 4096, 16, ragged=0.75, rot=64),
        # a serving step that takes in prompts: 8 of up to 1024 tokens among 24 single tokens
        _paged("append_chunks", "append", 32, 64, 8, 1024, 128, 8192, 64, ragged=0.5,
               layout="head", chunks=8, rot=128, order="pairs", scaling="pairs"),
        # one new token of 16 sequences against their caches of up to 4096
        _paged("paged_token", "paged", 16, 16, 4, 1, 64, 4096, 16, ragged=0.75),
        # 32 long conversations of a wide model, a token each
        _paged("paged_token_long", "paged", 32, 64, 8, 1, 128, 32768, 64, ragged=0.75,
               layout="head"),
        # a chunk of each of 4 prompts, whose earlier chunks are in the cache
        _paged("paged_chunk", "paged", 4, 16, 4, 512, 128, 8192, 16, ragged=0.4),
        # prompts among single tokens, odd sizes throughout, a window
        _paged("paged_mixed_odd", "paged", 30, 14, 2, 700, 80, 5001, 24, ragged=0.9, chunks=3,
               window=1000),
        # a chunk at the end of one very long document
        _paged("paged_chunk_long", "paged", 1, 16, 4, 2048, 128, 65536, 64, layout="head"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_heads(rng):
    kv_heads = rng.choice((1, 2, 3, 4, 8, 8, 16))
    heads = kv_heads * rng.choice((1, 1, 2, 4, 7, 8))
    dim = rng.choice((64, 64, 128, 128, rng.randrange(8, 129)))
    p = rng.choice((1, 1, kv_heads))
    return dict(heads=heads, kv_heads=kv_heads, dim=dim, p=p, r=rng.randrange(p))


def _draw_rotation(rng, dim):
    return dict(rot=dim // 2 * 2 if rng.random() < 0.6 else 2 * rng.randrange(2, dim // 2 + 1),
                order=rng.choice(("halves", "pairs")),
                scaling=rng.choice(("", "", "linear", "base", "turns", "pairs")))


def _draw_rope(rng):
    h = _draw_heads(rng)
    pos = rng.choice(("none", "first", "rows"))
    return _rope(None, rng.choice(("rope_fwd", "rope_bwd")), _log(rng, 1, 32),
                 seq=rng.choice((1, _log(rng, 1, 32768))), pos=pos,
                 far=0 if pos == "none" else _log(rng, 64, 1 << 20),
                 dtype="f32" if rng.random() < 0.3 else "bf16", **h, **_draw_rotation(rng, h["dim"]))


def _draw_paged(rng, op):
    h = _draw_heads(rng)
    batch = _log(rng, 1, 64)
    seq = 1 if rng.random() < 0.35 else _log(rng, 2, 2048)
    cached = _log(rng, max(seq, 16), 65536)
    page = rng.choice((16, 16, 32, 64, 128, rng.randrange(1, 100)))
    chunks = rng.randrange(1, batch + 1) if batch > 1 and seq > 1 and rng.random() < 0.5 else 0
    more = _draw_rotation(rng, h["dim"]) if op == "append" else dict(
        causal=rng.random() < 0.9, window=_log(rng, 16, 8192) if rng.random() < 0.2 else 0)
    if not more.get("causal", True):
        more["window"] = 0
    return _paged(None, op, batch, seq=seq, cached=cached, page=page,
                  ragged=round(rng.uniform(0.1, 0.9), 2) if rng.random() < 0.6 else 0.0,
                  layout=rng.choice(("token", "head")), chunks=chunks, **h, **more)


def draw(rng):
    most = {}
    for c in listed():
        w, o = work(c), most.setdefault(c["op"], {"bytes": 0, "flops": 0})
        for f in o:
            o[f] = max(o[f], w[f])
    most["rope_bwd"] = most["rope_fwd"]
    while True:
        x = rng.random()
        c = _draw_rope(rng) if x < 0.35 else _draw_paged(rng, "append" if x < 0.55 else "paged")
        w, o = work(c), most[c["op"]]
        if w["bytes"] > o["bytes"] or w["flops"] > o["flops"]:
            continue
        if c["op"] in ("append", "paged"):
            if c["batch"] * c["cached"] * c["kv_heads"] * c["dim"] > 1 << 30:   # the cache
                continue
            # the plain form holds every score
            if not c["chunks"] and c["batch"] * c["heads"] // c["p"] * c["seq"] * c["cached"] > 1 << 31:
                continue
        return c


def _split(n, p, r):
    """[offset, length) of the r-th of p balanced blocks."""
    return r * (n // p) + min(r, n % p), n // p + (r < n % p)


def _lens(c):
    """Per sequence: new tokens, and tokens in the cache with them."""
    B = c["batch"]
    if c["chunks"]:
        new = [max(1, c["seq"] - 37 * b) if b < c["chunks"] else 1 for b in range(B)]
    else:
        new = [c["seq"]] * B
    return new, [max(n, int(round(c["cached"] * (1.0 - c["ragged"] * b / B)))) for b, n in
                 enumerate(new)]


def _pairs(c):
    """Pairs of a query and a key that it sees, of one head, over the batch."""
    total = 0
    for n, k in zip(*_lens(c)):
        for i in range(n):
            hi = i + 1 + k - n if c["causal"] else k
            lo = max(0, i + 1 + k - n - c["window"]) if c["window"] else 0
            total += hi - lo
    return total


def _seen_keys(c):
    """Keys that some query sees, of one head, over the batch."""
    return sum(min(k, n - 1 + c["window"]) if c["window"] else k for n, k in zip(*_lens(c)))


def work(case):
    """What a pass has to read, write and compute: a product of two numbers and
    its sum are two operations; exponentials, sines and cosines are left out."""
    c = case
    hk = _split(c["kv_heads"], c["p"], c["r"])[1]
    h = hk * (c["heads"] // c["kv_heads"])
    D = c["dim"]
    if c["op"].startswith("rope"):
        rows, b = c["batch"] * c["seq"], 4 if c["dtype"] == "f32" else 2
        return {"bytes": 2 * b * rows * (h + hk) * D, "flops": 3 * rows * (h + hk) * c["rot"]}
    rows = sum(_lens(c)[0])
    if c["op"] == "append":
        return {"bytes": 4 * rows * (h + 2 * hk) * D, "flops": 3 * rows * (h + hk) * c["rot"]}
    return {"bytes": 4 * rows * h * D + 4 * rows * h + 4 * _seen_keys(c) * hk * D,
            "flops": 4 * D * h * _pairs(c)}


# ----------------------------------------------------------------- inputs
_BASE, _FACTOR, _LOW, _HIGH, _CONTEXT = 10000.0, 8.0, 1.0, 32.0, 4096.0


def _randn(shape, seed, dtype):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(dtype)


def _handle(c):
    """The library's table of a case's frequencies, which a program makes once."""
    from paper_2301_06813_amd import rotary
    return rotary.Rope(c["rot"], base=_BASE, order=c["order"], scaling=c["scaling"] or None,
                       factor=_FACTOR, low=_LOW, high=_HIGH, context=_CONTEXT,
                       mul=_mul(c), device="cuda")


def _mul(c):
    """The factor of the rotated columns that goes with frequencies scaled by pairs."""
    return 0.1 * math.log(_FACTOR) + 1.0 if c["scaling"] == "pairs" else 1.0


def prepare(case, seed):
    c = dict(case)
    s = {"case": c}
    B, H, Hk, D, n = c["batch"], c["heads"], c["kv_heads"], c["dim"], c["seq"]
    cpu = torch.Generator().manual_seed(seed)
    if c["op"].startswith("rope"):
        dt = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
        act = _randn((B, n, H + 2 * Hk, D), 10 * seed + 1, dt).permute(0, 2, 1, 3)
        s["Q"], s["K"] = act[:, :H], act[:, H:H + Hk]
        s["pos"] = None
        if c["pos"] == "first":
            s["pos"] = torch.randint(0, c["far"] - n + 1, (B,), generator=cpu)
            s["pos"][0] = c["far"] - n
        elif c["pos"] == "rows":     # documents laid end to end: places start again
            at = torch.randint(1, c["far"] + 1, (B, n), generator=cpu)
            s["pos"] = (torch.arange(n)[None, :] + at[:, :1]) % at.amax(1, keepdim=True)
        if s["pos"] is not None:
            s["pos"] = s["pos"].to(torch.int32).cuda()
        if own:
            s["rope"] = _handle(c)
        return s
    new, cached = _lens(c)
    s["new"], s["cached"] = new, cached          # the scheduler knows them on the host
    if c["chunks"]:
        act = _randn((1, sum(new), H + 2 * Hk, D), 10 * seed + 1, torch.bfloat16)
        s["row_q"] = torch.tensor([sum(new[:b]) for b in range(B + 1)], dtype=torch.int32,
                                  device="cuda")
    else:
        act = _randn((B, n, H + 2 * Hk, D), 10 * seed + 1, torch.bfloat16)
        s["row_q"] = None
    act = act.permute(0, 2, 1, 3)
    s["Q"], s["K"], s["V"] = act[:, :H], act[:, H:H + Hk], act[:, H + Hk:]
    s["len_k"] = torch.tensor(cached, dtype=torch.int32, device="cuda")
    # pages lie anywhere in the pool
    P = c["page"]
    width = (max(cached) + P - 1) // P
    pages = B * width + 3
    s["table"] = torch.randperm(pages, generator=cpu)[:B * width].view(B, width).to(torch.int32).cuda()
    for i, name in enumerate(("kc", "vc")):
        shape = (pages, P, Hk, D) if c["layout"] == "token" else (pages, Hk, P, D)
        t = _randn(shape, 10 * seed + 2 + i, torch.bfloat16)
        s[name] = t.permute(0, 2, 1, 3) if c["layout"] == "token" else t
    s["scale"] = 1.0 / math.sqrt(D)
    if own:
        from paper_2301_06813_amd import paged
        s["cache"] = paged.Cache(s["kc"], s["vc"])
        s["rope"] = _handle(c) if c["rot"] else None
    return s


# ------------------------------------------------------------- plain forms
def _heads_of(s):
    """This device's query heads and key heads, as slices of the global ones."""
    c = s["case"]
    off, hk = _split(c["kv_heads"], c["p"], c["r"])
    g = c["heads"] // c["kv_heads"]
    return slice(off * g, (off + hk) * g), slice(off, off + hk)


def _freqs(c):
    rot = c["rot"]
    i = torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot
    base = _BASE
    if c["scaling"] == "base" and rot > 2:
        base = _BASE * _FACTOR ** (rot / (rot - 2))
    f = base ** -i
    if c["scaling"] == "linear":
        return f / _FACTOR
    if c["scaling"] == "turns":
        w = ((_CONTEXT * f / (2 * math.pi) - _LOW) / (_HIGH - _LOW)).clamp(0.0, 1.0)
        return f * w + f / _FACTOR * (1 - w)
    if c["scaling"] == "pairs":
        def place(turns):
            return rot * math.log(_CONTEXT / (2 * math.pi * turns)) / (2 * math.log(_BASE))
        lo, hi = max(0, math.floor(place(_HIGH))), min(rot - 1, math.ceil(place(_LOW)))
        w = ((i * rot / 2 - lo) / max(hi - lo, 0.001)).clamp(0.0, 1.0)
        return f * (1 - w) + f / _FACTOR * w
    return f


def _plain_rotate(x, pos, c, sign):
    """x [batch][heads][rows][dim], rotated by sign times the angles of pos [batch][rows]."""
    rot = c["rot"]
    a = pos.double()[:, None, :, None] * _freqs(c)
    cos, sin = (torch.cos(a) * _mul(c)).float(), (torch.sin(a) * (sign * _mul(c))).float()
    x = x.float()
    y = x.clone()
    one, two = (slice(0, rot // 2), slice(rot // 2, rot)) if c["order"] == "halves" else \
        (slice(0, rot, 2), slice(1, rot, 2))
    u, v = x[..., one], x[..., two]
    y[..., one] = u * cos - v * sin
    y[..., two] = v * cos + u * sin
    return y


def _places(s):
    c = s["case"]
    at = torch.arange(c["seq"], device="cuda")[None, :]
    if c["pos"] == "none":
        return at
    return s["pos"].long()[:, None] + at if c["pos"] == "first" else s["pos"].long()


def _plain_rope(s, sign):
    hq, hk = _heads_of(s)
    pos = _places(s)
    return tuple(_plain_rotate(x, pos, s["case"], sign).to(x.dtype)
                 for x in (s["Q"][:, hq], s["K"][:, hk]))


def _plain_append(s):
    c = s["case"]
    hq, hk = _heads_of(s)
    B, P = c["batch"], c["page"]
    if s["row_q"] is not None:      # sequence and place of every packed row
        first = s["row_q"].long()
        row = torch.arange(s["Q"].shape[2], device="cuda")
        seq = (row[:, None] >= first[None, 1:]).sum(1)
        t = s["len_k"].long()[seq] - first[seq + 1] + row
    else:
        seq = torch.arange(B, device="cuda").repeat_interleave(c["seq"])
        t = (s["len_k"].long()[:, None] - c["seq"] + torch.arange(c["seq"], device="cuda")).view(-1)
    pos = t.view(s["Q"].shape[0], -1)
    rows = lambda x: x.transpose(1, 2).reshape(-1, x.shape[1], x.shape[3])
    k, q = (_plain_rotate(x, pos, c, 1) for x in (s["K"][:, hk], s["Q"][:, hq]))
    page, slot = s["table"].long()[seq, t // P], t % P
    s["kc"][page, hk, slot] = rows(k).to(s["kc"].dtype)
    s["vc"][page, hk, slot] = rows(s["V"][:, hk])
    return q.to(s["Q"].dtype), s["kc"], s["vc"]


def _plain_softmax_product(x, v):
    """exp(x - lse) v and lse, of rows of masked scores."""
    top = x.amax(-1, keepdim=True)
    x = torch.exp(x - torch.where(top == -math.inf, 0.0, top))
    total = x.sum(-1, keepdim=True)
    lse = torch.where(total > 0, top + torch.log(total), -math.inf)
    return (x / torch.where(total > 0, total, 1.0)) @ v, lse


def _plain_seen(c, n, keys, device="cuda"):
    """[..., n, keys.max] truth values: query i of n sees key j, keys long each."""
    lk = torch.as_tensor(keys, device=device).view(-1, 1, 1)
    i = torch.arange(n, device=device).view(1, n, 1)
    j = torch.arange(int(max(keys)), device=device).view(1, 1, -1)
    seen = j < lk
    if c["causal"]:
        seen = seen & (j <= i + lk - n)
    if c["window"]:
        seen = seen & (j > i + lk - n - c["window"])
    return seen


def _plain_paged(s):
    c = s["case"]
    hq, hk = _heads_of(s)
    Q, kc, vc = s["Q"][:, hq], s["kc"][:, hk], s["vc"][:, hk]
    Hq, Hk, D, P = Q.shape[1], kc.shape[1], c["dim"], c["page"]
    g = Hq // Hk

    def gather(pool, table, n):     # [sequences][heads][n][dim]
        t = pool[table.long()].transpose(1, 2)
        return t.reshape(t.shape[0], Hk, -1, D)[:, :, :n].float()

    def attend(q, table, keys):     # q [sequences][heads][n][dim]
        b, n, top = q.shape[0], q.shape[2], max(keys)
        k, v = gather(kc, table, top), gather(vc, table, top)
        x = q.float().reshape(b, Hk, g * n, D) @ k.transpose(2, 3)
        x = (x * s["scale"]).view(b, Hk, g, n, top)
        x = x.masked_fill_(~_plain_seen(c, n, keys)[:, None, None], -math.inf)
        o, lse = _plain_softmax_product(x.view(b, Hk, g * n, top), v)
        return o.view(b, Hq, n, D), lse.view(b, Hq, n)

    if not c["chunks"]:
        O, lse = attend(Q, s["table"], s["cached"])
        return O.to(Q.dtype), lse
    parts, at = [], 0
    for b, (n, keys) in enumerate(zip(s["new"], s["cached"])):
        parts.append(attend(Q[:, :, at:at + n], s["table"][b:b + 1, :(keys + P - 1) // P], [keys]))
        at += n
    return torch.cat([o for o, _ in parts], 2).to(Q.dtype), torch.cat([z for _, z in parts], 2)


# -------------------------------------------------------------------- run
def run(state):
    s, c = state, state["case"]
    if own:
        if c["op"].startswith("rope"):
            from paper_2301_06813_amd import rotary
            turn = rotary.fwd if c["op"] == "rope_fwd" else rotary.bwd
            return turn(s["rope"], s["Q"], s["K"], c["p"], c["r"], pos=s["pos"])
        if c["op"] == "append":
            Q = s["cache"].append(s["K"], s["V"], s["table"], s["len_k"], c["p"], c["r"], Q=s["Q"],
                                  rope=s["rope"], row_q=s["row_q"])
            return Q, s["kc"], s["vc"]
        return s["cache"].attend(s["Q"], s["table"], s["len_k"], c["p"], c["r"], scale=s["scale"],
                                 causal=c["causal"], window=c["window"], row_q=s["row_q"])
    if c["op"].startswith("rope"):
        return _plain_rope(s, 1 if c["op"] == "rope_fwd" else -1)
    return _plain_append(s) if c["op"] == "append" else _plain_paged(s)


# ------------------------------------------------------------------ exact
def _exact_angles(c, pos):
    """cos and sin, times the factor, of places pos (a flat tensor), a column for a pair."""
    rot, f = c["rot"], []
    for i in range(rot // 2):
        x = math.exp(-2.0 * i / rot * math.log(_BASE))
        if c["scaling"] == "linear":
            x = x / _FACTOR
        elif c["scaling"] == "base" and rot > 2:
            x = x * math.exp(-2.0 * i / (rot - 2) * math.log(_FACTOR))
        elif c["scaling"] == "turns":
            turns = _CONTEXT * x / (2.0 * math.pi)
            kept = min(1.0, max(0.0, (turns - _LOW) / (_HIGH - _LOW)))
            x = x * (kept + (1.0 - kept) / _FACTOR)
        elif c["scaling"] == "pairs":
            per = rot / (2.0 * math.log(_BASE))
            lo = max(0, math.floor(per * math.log(_CONTEXT / (2.0 * math.pi * _HIGH))))
            hi = min(rot - 1, math.ceil(per * math.log(_CONTEXT / (2.0 * math.pi * _LOW))))
            part = min(1.0, max(0.0, (i - lo) / max(hi - lo, 0.001)))
            x = x * (1.0 - part + part / _FACTOR)
        f.append(x)
    a = torch.outer(pos.double(), torch.tensor(f, dtype=torch.float64, device="cuda"))
    m = 0.1 * math.log(_FACTOR) + 1.0 if c["scaling"] == "pairs" else 1.0
    return m * torch.cos(a), m * torch.sin(a)


def _exact_turn(x, cos, sin, c, back=False):
    """x [rows][heads][dim] in 64 bits, as complex numbers times cos + i sin."""
    rot = c["rot"]
    z = x[..., :rot]
    z = z.unflatten(-1, (2, rot // 2)).transpose(-1, -2) if c["order"] == "halves" else \
        z.unflatten(-1, (rot // 2, 2))
    w = torch.complex(cos, -sin if back else sin)[:, None, :]
    z = torch.view_as_real(torch.view_as_complex(z.contiguous()) * w)
    z = z.transpose(-1, -2) if c["order"] == "halves" else z
    return torch.cat([z.flatten(-2), x[..., rot:]], -1)


def _exact_rope(s):
    c = s["case"]
    hq, hk = _heads_of(s)
    outs = []
    for x in (s["Q"][:, hq], s["K"][:, hk]):
        y = torch.empty(x.shape, dtype=torch.float64, device="cuda")
        for b in range(c["batch"]):
            pos = torch.arange(c["seq"], device="cuda")
            if c["pos"] == "first":
                pos = pos + s["pos"][b].item()
            elif c["pos"] == "rows":
                pos = s["pos"][b]
            cos, sin = _exact_angles(c, pos)
            y[b] = _exact_turn(x[b].transpose(0, 1).double(), cos, sin, c,
                               c["op"] == "rope_bwd").transpose(0, 1)
        outs.append(y)
    return tuple(outs)


def _rows_of(s, b):
    """(index of Q's batch, first row) of sequence b."""
    return (0, sum(s["new"][:b])) if s["row_q"] is not None else (b, 0)


def _exact_append(s):
    c = s["case"]
    hq, hk = _heads_of(s)
    kc, vc = s["kc"].double(), s["vc"].double()
    q = torch.empty(s["Q"][:, hq].shape, dtype=torch.float64, device="cuda")
    table = s["table"].tolist()
    for b, (n, keys) in enumerate(zip(s["new"], s["cached"])):
        x, at = _rows_of(s, b)
        cos, sin = _exact_angles(c, torch.arange(keys - n, keys, device="cuda"))
        turn = lambda t: _exact_turn(t[x, :, at:at + n].transpose(0, 1).double(), cos, sin,
                                     c).transpose(0, 1)
        q[x, :, at:at + n] = turn(s["Q"][:, hq])
        k, v = turn(s["K"][:, hk]), s["V"][x, hk, at:at + n].double()
        i = 0
        while i < n:                 # a page at a time
            page, slot = divmod(keys - n + i, c["page"])
            m = min(n - i, c["page"] - slot)
            kc[table[b][page], hk, slot:slot + m] = k[:, i:i + m]
            vc[table[b][page], hk, slot:slot + m] = v[:, i:i + m]
            i += m
    return q, kc, vc


def _exact_paged(s):
    """One key head of one sequence at a time, a query head after the other."""
    c = s["case"]
    hq, hk = _heads_of(s)
    Q, kc, vc = s["Q"][:, hq], s["kc"][:, hk], s["vc"][:, hk]
    g, D = Q.shape[1] // kc.shape[1], c["dim"]
    O = torch.zeros(Q.shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(Q.shape[:3], dtype=torch.float64, device="cuda")
    for b, (n, keys) in enumerate(zip(s["new"], s["cached"])):
        x, at = _rows_of(s, b)
        pages = s["table"][b, :(keys + c["page"] - 1) // c["page"]].long()
        last = torch.arange(keys - n, keys, device="cuda")[:, None]
        key = torch.arange(keys, device="cuda")[None, :]
        hidden = key > last if c["causal"] else torch.zeros((n, keys), dtype=torch.bool,
                                                            device="cuda")
        if c["window"]:
            hidden = hidden | (key <= last - c["window"])
        for h in range(kc.shape[1]):
            k = kc[pages, h].reshape(-1, D)[:keys].double()
            v = vc[pages, h].reshape(-1, D)[:keys].double()
            kt = k.t().contiguous()
            for e in range(h * g, h * g + g):
                w = torch.mm(Q[x, e, at:at + n].double(), kt).mul_(s["scale"])
                w[hidden] = -math.inf
                z = torch.logsumexp(w, 1)
                w = w.sub_(z[:, None]).exp_()
                lse[x, e, at:at + n], O[x, e, at:at + n] = z, torch.mm(w, v)
    return O, lse


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"].startswith("rope"):
        return _exact_rope(s)
    return _exact_append(s) if case["op"] == "append" else _exact_paged(s)
