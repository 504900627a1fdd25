"""Workloads of the 8-bit language-model operators, in plain torch and through this library.

A case is a plain dict.  `listed` names twelve, `draw` gives others of the same ranges, `prepare` makes
what a program holds before the call, `run` is one pass, `work` the bytes and operations that a pass
cannot do without, and `exact` the same results from the definitions in 64 bits.

Operators
  linear   y = (codes(x) . w^T) * sx[token] * sw[channel] + bias: rows of activations quantized to 8 bits
           with a scale for each token, multiplied with 8-bit weights that have a scale for each output
           channel;
  append   new keys and values written to a paged cache of 8-bit codes, queries and keys rotated by their
           positions on the way.  A page of one head is a block with one scale, the smallest power of two
           that keeps its largest value within 127 codes; where new tokens raise it, the block's older
           codes are rounded again.  The pages are read back as values;
  attend   softmax attention of new queries over such a cache, grouped heads, causal or not, for single
           tokens, chunks and whole prompts.

`own` False: elementary torch operations in 32 bits, rounded once at the end.  `own` True: the calls that
a user makes of the library.
"""
from __future__ import annotations

import math
import random

import torch

own = False

FL_LO, FL_HI = -32, 40  # fractional lengths that a block's scale 2^-FL may take
_FT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


# ------------------------------------------------------------------------------ cases
def listed():
    return [
        # one token through a 4096 x 4096 FC layer: decoding alone, the weights' read and the launches
        _linear("linear_token", M=1, N=4096, K=4096, dtype="bf16", bias=0),
        # a decoding batch through the largest FC layer of the library's networks (25088 inputs)
        _linear("linear_batch", M=64, N=4096, K=25088, dtype="f16", bias=1),
        # a short prompt, odd in tokens, channels and inputs, into 1000 logits kept in 32 bits
        _linear("linear_odd", M=251, N=1001, K=4090, dtype="bf16", out="f32", bias=1),
        # prompts packed into one matrix, the widest layer: tensor-core bound
        _linear("linear_prompt", M=8192, N=16384, K=4096, dtype="bf16", bias=0),
        # one sequence decoding a token, as many key heads as query heads
        _append("append_token", B=1, n=1, ragged=0, ctx=200, Hq=8, Hkv=8, D=64, page=16, rot=64, inter=0, dtype="f16"),
        # a serving batch decoding: one token each, grouped heads, blocks of every fill
        _append("append_batch", B=256, n=1, ragged=0, ctx=250, Hq=32, Hkv=8, D=128, page=64, rot=128, inter=0, dtype="bf16"),
        # chunks of unequal length (one of them empty) behind short contexts, half of each head rotated
        _append("append_ragged", B=23, n=700, ragged=1, ctx=90, Hq=16, Hkv=4, D=64, page=32, rot=32, inter=1, dtype="bf16"),
        # whole prompts into an empty cache
        _append("append_prompt", B=4, n=8192, ragged=0, ctx=0, Hq=32, Hkv=8, D=128, page=128, rot=128, inter=0, dtype="bf16"),
        # one sequence decoding over a short cache: latency
        _attend("attend_token", B=1, n=1, ragged=0, ctx=999, Hq=8, Hkv=8, D=64, page=16, causal=1, dtype="f16"),
        # a serving batch decoding over caches of unequal length: the cache's read
        _attend("attend_batch", B=64, n=1, ragged=1, ctx=16000, Hq=32, Hkv=8, D=128, page=64, causal=1, dtype="bf16"),
        # few tokens of two sequences over a very long cache (a draft being verified): work split over the cache
        _attend("attend_long", B=2, n=4, ragged=0, ctx=200001, Hq=32, Hkv=8, D=128, page=128, causal=1, dtype="bf16"),
        # whole prompts: tensor-core bound
        _attend("attend_prompt", B=2, n=8192, ragged=0, ctx=0, Hq=32, Hkv=8, D=128, page=64, causal=1, dtype="bf16"),
    ]


def _linear(name, **kw):
    return _named(name, {"kind": "linear", "out": kw.get("dtype"), **kw})


def _append(name, **kw):
    return _named(name, {"kind": "append", "shape": 1, **kw})


def _attend(name, **kw):
    return _named(name, {"kind": "attend", "shape": 1, "lse": 0, **kw})


def _named(name, d):
    if name:
        d["name"] = name
    return d


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _heads(rng):
    Hkv = rng.choice([1, 2, 4, 8])
    return Hkv * rng.choice([1, 1, 2, 4, 4, 5, 8]), Hkv


def draw(rng: random.Random):
    kind = rng.choice(["linear", "append", "attend", "attend"])
    if kind == "linear":
        while True:
            c = _linear(None, M=_log(rng, 1, 8192), N=_log(rng, 64, 16384), K=_log(rng, 64, 25088),
                        dtype=rng.choice(["bf16", "f16"]), bias=rng.randint(0, 1))
            if rng.random() < 0.5:  # layers are mostly multiples of 64; the rest are odd
                c["N"], c["K"] = (c["N"] + 63) // 64 * 64, (c["K"] + 63) // 64 * 64
            if rng.random() < 0.2:
                c["out"] = "f32"
            if c["M"] * c["N"] * c["K"] <= 8192 * 16384 * 4096 and c["N"] <= 16384 and c["K"] <= 25088:
                return c
    Hq, Hkv = _heads(rng)
    D, page, ragged = rng.choice([64, 128, 128]), rng.choice([16, 32, 64, 128]), rng.randint(0, 1)
    shape, dtype = rng.randrange(1000), rng.choice(["bf16", "bf16", "f16"])
    if kind == "append":
        while True:
            one = rng.random() < 0.5
            c = _append(None, B=_log(rng, 1, 256 if one else 32), n=rng.choice([1, 1, 2, 4]) if one else _log(rng, 2, 8192),
                        ragged=ragged, ctx=_log(rng, 1, 300) - 1, Hq=Hq, Hkv=Hkv, D=D, page=page,
                        rot=rng.choice([D, D, D // 2]), inter=rng.randint(0, 1), dtype=dtype, shape=shape)
            if work(c)["bytes"] <= work(_append(None, B=4, n=8192, ragged=0, ctx=0, Hq=32, Hkv=8, D=128, page=128, rot=128))["bytes"]:
                return c
    while True:
        what = rng.choice(["token", "token", "chunk", "prompt"])
        B = _log(rng, 1, 64 if what == "token" else 8)
        n = rng.choice([1, 1, 1, 2, 4, 7]) if what == "token" else _log(rng, 8, 1000) if what == "chunk" else _log(rng, 100, 8192)
        ctx = _log(rng, 1, 200000) if what == "token" else _log(rng, 1, 20000) if what == "chunk" else 0
        c = _attend(None, B=B, n=n, ragged=ragged, ctx=ctx, Hq=Hq, Hkv=Hkv, D=D, page=page, causal=int(rng.random() < 0.8),
                    dtype=dtype, lse=rng.randint(0, 1), shape=shape)
        w = work(c)
        scores = B * Hq * n * (n + ctx)  # of the plain form, in 32 bits
        if w["bytes"] <= 1.3e9 and w["flops"] <= 1.1e12 and scores <= 2 * 32 * 8192 * 8192 and B * (n + ctx) * Hkv * D <= 1.1e9:
            return c


def _lengths(c):
    """New tokens and tokens before them of each sequence, by the case alone."""
    B, n, ctx = c["B"], c["n"], c["ctx"]
    if not c["ragged"]:
        if c["kind"] == "append":  # (blocks of every fill)
            r = random.Random(c.get("shape", 1))
            return [n] * B, [r.randint(0, ctx) for _ in range(B)]
        return [n] * B, [ctx] * B
    r = random.Random(c.get("shape", 1))
    news = [n if n == 1 else r.randint(1, n) for _ in range(B)]
    ctxs = [r.randint(ctx // 16, ctx) for _ in range(B)]
    if B > 2 and n > 1:
        news[B // 2] = 0
    if B > 3 and c["kind"] == "attend" and c["causal"] and n == 1:
        ctxs[1] = 0
    return news, ctxs


def work(case):
    c = case
    if c["kind"] == "linear":
        M, N, K = c["M"], c["N"], c["K"]
        out = 4 if c["out"] == "f32" else 2
        return {"bytes": 2 * M * K + N * K + 4 * N * (1 + c["bias"]) + out * M * N, "flops": 2 * M * N * K}
    news, ctxs = _lengths(c)
    T = sum(news)
    if c["kind"] == "append":
        # queries and keys and values in, queries and codes out, and the pages read back as 16-bit values
        pages = sum(-(-(a + b) // c["page"]) for a, b in zip(news, ctxs))
        pool = pages * c["page"] * c["Hkv"] * c["D"] * 2
        return {"bytes": T * c["D"] * (4 * c["Hq"] + 6 * c["Hkv"]) + 3 * pool, "flops": 6 * T * c["rot"] * (c["Hq"] + c["Hkv"])}
    keys = sum(a + b for a, b in zip(news, ctxs) if a)
    pairs = sum(a * b + (a * (a + 1) // 2 if c["causal"] else a * a) for a, b in zip(news, ctxs))
    return {"bytes": 2 * keys * c["Hkv"] * c["D"] + 4 * T * c["Hq"] * c["D"], "flops": 4 * pairs * c["Hq"] * c["D"]}


# ------------------------------------------------------------------------------ inputs
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _codes(shape, g, spread):
    """8-bit codes of a normal tensor, in pieces so that large ones need no large scratch."""
    out = torch.empty(shape, dtype=torch.int8, device="cuda")
    flat = out.view(-1)
    for i in range(0, flat.numel(), 1 << 28):
        part = flat[i:i + (1 << 28)]
        part.copy_((torch.randn(part.numel(), device="cuda", generator=g) * spread).round_().clamp_(-127, 127))
    return out


def _batch(c, seed):
    """The page table and lengths of a batch: pages scattered over the pool, unused entries -1."""
    news, ctxs = _lengths(c)
    lens = [a + b for a, b in zip(news, ctxs)]
    need = [-(-n // c["page"]) for n in lens]
    total = max(1, sum(need))
    order = torch.randperm(total, generator=torch.Generator().manual_seed(int(seed) + 1)).int()
    table = torch.full((c["B"], max(1, max(need))), -1, dtype=torch.int32)
    at = 0
    for b, k in enumerate(need):
        table[b, :k] = order[at:at + k]
        at += k
    starts = torch.tensor([sum(news[:b]) for b in range(c["B"] + 1)], dtype=torch.int32)
    return {"pages": table.cuda(), "lens": torch.tensor(lens, dtype=torch.int32).cuda(), "n_pages": total,
            "starts": starts.cuda() if c["ragged"] else None, "T": sum(news), "max_len": max(1, max(lens)), "most": max(news)}


def prepare(case, seed):
    c, g = case, _gen(seed)
    if c["kind"] == "linear":
        M, N, K, dt = c["M"], c["N"], c["K"], _FT[c["dtype"]]
        # activations of tokens of unequal size, a few inputs larger than the rest
        x = torch.randn(M, K, device="cuda", generator=g) * torch.exp(0.5 * torch.randn(M, 1, device="cuda", generator=g))
        x *= torch.where(torch.rand(K, device="cuda", generator=g) < 0.01, 8.0, 1.0)
        return {"c": c, "x": x.to(dt), "w": _codes((N, K), g, 32.0), "out": _FT[c["out"]],
                "sw": torch.exp(0.3 * torch.randn(N, device="cuda", generator=g)) * (1.0 / (32 * math.sqrt(K))),
                "bias": torch.randn(N, device="cuda", generator=g) * 0.1 if c["bias"] else None}
    s = {"c": c, **_batch(c, seed)}
    P, Hq, Hkv, D, dt, T = s["n_pages"], c["Hq"], c["Hkv"], c["D"], _FT[c["dtype"]], s["T"]
    s["k"], s["v"] = _codes((P, Hkv, c["page"], D), g, 24.0), _codes((P, Hkv, c["page"], D), g, 24.0)
    # blocks' scales: powers of two as appending leaves them, for every other seed any calibrated ones
    for name in ("k_scale", "v_scale"):
        e = torch.randint(4, 7, (P, Hkv), device="cuda", generator=g).float()
        if c["kind"] == "attend" and int(seed) % 2:
            e = e + torch.rand(P, Hkv, device="cuda", generator=g)
        s[name] = torch.exp2(-e)
    if c["kind"] == "attend":
        s["q"] = torch.randn(T, Hq, D, device="cuda", generator=g).to(dt)
        s["scale"] = 1.0 / math.sqrt(D)
        return s
    # queries, keys and values as a fused projection leaves them, side by side in one row per token
    qkv = torch.randn(T, (Hq + 2 * Hkv) * D, device="cuda", generator=g).to(dt).view(T, Hq + 2 * Hkv, D)
    s["q"], s["new_k"], s["new_v"] = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    half = c["rot"] // 2
    angle = torch.arange(s["max_len"], device="cuda").double()[:, None] * 10000.0 ** (-torch.arange(half, device="cuda").double() / half)
    s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
    s["all"] = torch.arange(P, dtype=torch.int32, device="cuda")
    return s


# ------------------------------------------------------------------------------ one pass
_library = None


def _ops():
    global _library
    if _library is None:
        from paper_2203_12091_gb300 import llm
        _library = llm
    return _library


def run(state):
    s = state
    kind = s["c"]["kind"]
    if not own:
        return _PLAIN[kind](s)
    ops = _ops()
    if kind == "linear":
        if "layer" not in s:  # the layer that a program keeps: its weights' rows padded where they are not whole 16 bytes
            s["layer"] = ops.Linear8(s["w"], s["sw"], s["bias"])
        return s["layer"](s["x"], s["out"])
    if "cache" not in s:  # the handle that a program keeps
        s["cache"] = ops.KVCache(s["k"], s["v"], s["k_scale"], s["v_scale"])
    cache, c = s["cache"], s["c"]
    if kind == "append":
        q = ops.kv_append(cache, s["pages"], s["lens"], s["new_k"], s["new_v"], q=s["q"], starts=s["starts"], cos=s["cos"],
                          sin=s["sin"], interleaved=bool(c["inter"]))
        k, v = ops.kv_values(cache, s["all"], torch.bfloat16)
        return q, k, v, s["k_scale"], s["v_scale"]
    return ops.kv_attention(cache, s["pages"], s["lens"], s["q"], starts=s["starts"], scale=s["scale"], causal=bool(c["causal"]),
                            return_lse=bool(c["lse"]))


def _plain_linear(s):
    x = s["x"].float()
    amax = x.abs().amax(1, keepdim=True)
    codes = (x * torch.where(amax > 0, 127.0 / amax, 0.0)).round().clamp(-127, 127)
    y = (codes @ s["w"].float().t()) * (amax / 127.0) * s["sw"]
    if s["bias"] is not None:
        y = y + s["bias"]
    return y.to(s["out"])


def _tokens(s, T, device):
    """Sequence, place among its new tokens, and position of every new token."""
    lens = s["lens"].long()
    B = lens.numel()
    t = torch.arange(T, device=device)
    starts = s["starts"].long() if s["starts"] is not None else torch.arange(B + 1, device=device) * (T // B)
    b = torch.searchsorted(starts, t, right=True) - 1
    place = t - starts[b]
    return b, place, lens[b] - (starts[b + 1] - starts[b]) + place


def _rotate(x, cos, sin, rot, inter):
    half = rot // 2
    if inter:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
    else:
        a, b = x[..., :half], x[..., half:rot]
    ra, rb = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack((ra, rb), -1).flatten(-2) if inter else torch.cat((ra, rb), -1)
    return torch.cat((turned, x[..., rot:]), -1)


def _block_scale(amax):
    """The smallest 2^-FL, FL in [FL_LO, FL_HI], with amax <= 127 * 2^-FL."""
    m, e = torch.frexp(amax)
    fl = torch.where(m <= 127.0 / 128.0, 7 - e, 6 - e).clamp(FL_LO, FL_HI)
    fl = torch.where(amax > 0, fl, FL_HI)
    return torch.ldexp(torch.ones_like(amax), -fl)


def _store(codes, scale, x, page, slot):
    """Rows x [T, H, D] into the blocks `page` at `slot`, scales raised and older codes rounded again as needed."""
    P, H, S, D = codes.shape
    new = torch.zeros_like(scale, dtype=x.dtype).scatter_reduce_(0, page[:, None].expand(-1, H), x.abs().amax(-1), "amax")
    first = torch.full((P,), S, device=x.device).scatter_reduce_(0, page, slot, "amin")
    touched = (first < S)[:, None]
    before = torch.where((first > 0)[:, None], scale.to(x.dtype), 0.0)
    after = torch.where(touched, torch.maximum(before, _block_scale(new)), scale.to(x.dtype))
    older = touched & (torch.arange(S, device=x.device)[None, :] < first[:, None])
    again = (codes.to(x.dtype) * (scale.to(x.dtype) / after)[:, :, None, None]).round().clamp(-128, 127)
    codes.copy_(torch.where(older[:, None, :, None], again, codes.to(x.dtype)))
    scale.copy_(after)
    codes[page, :, slot] = (x / after[page][:, :, None]).round().clamp(-128, 127).to(torch.int8)


def _plain_append(s):
    c = s["c"]
    b, _, pos = _tokens(s, s["T"], s["q"].device)
    page, slot = s["pages"].long()[b, pos // c["page"]], pos % c["page"]
    cos, sin = s["cos"][pos][:, None], s["sin"][pos][:, None]
    q = _rotate(s["q"].float(), cos, sin, c["rot"], c["inter"]).to(s["q"].dtype)
    _store(s["k"], s["k_scale"], _rotate(s["new_k"].float(), cos, sin, c["rot"], c["inter"]), page, slot)
    _store(s["v"], s["v_scale"], s["new_v"].float(), page, slot)
    k, v = (s[n].float() * s[n + "_scale"][:, :, None, None] for n in ("k", "v"))
    return q, k.to(torch.bfloat16), v.to(torch.bfloat16), s["k_scale"], s["v_scale"]


def _gathered(s, name, B, dtype):
    """Values [B, Hkv, tokens, D] of a batch's pages, one after the other."""
    table = s["pages"].long().clamp(min=0)
    x = s[name][table].to(dtype) * s[name + "_scale"][table].to(dtype)[..., None, None]
    return x.transpose(1, 2).flatten(2, 3)


def _plain_attend(s):
    c, T = s["c"], s["T"]
    B, Hq, Hkv, D, n = c["B"], c["Hq"], c["Hkv"], c["D"], s["most"]
    dev = s["q"].device
    b, place, pos = _tokens(s, T, dev)
    q = torch.zeros(B, n, Hq, D, device=dev)
    q[b, place] = s["q"].float()
    at = torch.full((B, n), -1, device=dev)  # positions; rows that no token fills see nothing
    at[b, place] = pos
    q = q.view(B, n, Hkv, Hq // Hkv, D).permute(0, 2, 3, 1, 4).flatten(2, 3)
    k = _gathered(s, "k", B, torch.float32)
    key = torch.arange(k.shape[2], device=dev)
    seen = key < s["lens"].long()[:, None, None]
    seen = seen & (key <= at[:, :, None] if c["causal"] else at[:, :, None] >= 0)  # [B, n, keys]
    seen = seen[:, None, None]
    w = ((q @ k.transpose(2, 3)) * s["scale"]).view(B, Hkv, Hq // Hkv, n, -1).masked_fill_(~seen, -math.inf)
    del k
    top = w.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    w = w.sub_(top).exp_()
    total = w.sum(-1, keepdim=True)
    out = w.flatten(2, 3) @ _gathered(s, "v", B, torch.float32)
    out = out.view(B, Hkv, Hq // Hkv, n, D) / torch.where(total > 0, total, 1.0)
    out = out.permute(0, 3, 1, 2, 4).reshape(B, n, Hq, D)[b, place].to(s["q"].dtype)
    if not c["lse"]:
        return out
    return out, (top + total.log()).permute(0, 3, 1, 2, 4).reshape(B, n, Hq)[b, place]


_PLAIN = {"linear": _plain_linear, "append": _plain_append, "attend": _plain_attend}


# ------------------------------------------------------------------------------ the definitions in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return {"linear": _exact_linear, "append": _exact_append, "attend": _exact_attend}[case["kind"]](s)


def _exact_linear(s):
    rows, x, w = [], s["x"], s["w"].double()
    for i in range(0, x.shape[0], 1024):
        part = x[i:i + 1024].double()
        sx = part.abs().amax(1) / 127
        codes = torch.where(sx[:, None] > 0, part / sx[:, None], 0.0).round()
        y = (codes @ w.t()) * sx[:, None] * s["sw"].double()
        rows.append(y + s["bias"].double() if s["bias"] is not None else y)
    return torch.cat(rows)


def _exact_append(s):
    c = s["c"]
    lens, table = s["lens"].tolist(), s["pages"].tolist()
    starts = s["starts"].tolist() if s["starts"] is not None else [i * (s["T"] // c["B"]) for i in range(c["B"] + 1)]
    S, rot, half = c["page"], c["rot"], c["rot"] // 2

    def turn(x, pos):
        cos, sin = s["cos"][pos].double()[:, None], s["sin"][pos].double()[:, None]
        y = x.clone()
        i, j = (slice(0, rot, 2), slice(1, rot, 2)) if c["inter"] else (slice(0, half), slice(half, rot))
        y[..., i] = x[..., i] * cos - x[..., j] * sin
        y[..., j] = x[..., j] * cos + x[..., i] * sin
        return y

    q, k, v = s["q"].double(), s["new_k"].double(), s["new_v"].double()
    where, pos = [], torch.empty(s["T"], dtype=torch.long, device=q.device)
    for b in range(c["B"]):
        n = starts[b + 1] - starts[b]
        pos[starts[b]:starts[b + 1]] = torch.arange(lens[b] - n, lens[b], device=q.device)
        p = lens[b] - n
        while p < lens[b]:  # the new tokens of one page
            e = min(lens[b], (p // S + 1) * S)
            where.append((table[b][p // S], p % S, e - p, starts[b] + p - (lens[b] - n)))
            p = e
    q, k = turn(q, pos), turn(k, pos)
    out = []
    idx = torch.tensor([w[0] for w in where], device=q.device)
    first = torch.tensor([w[1] for w in where], device=q.device)
    count = torch.tensor([w[2] for w in where], device=q.device)
    token = torch.tensor([w[3] for w in where], device=q.device)
    slots = torch.arange(S, device=q.device)
    fresh = (slots >= first[:, None]) & (slots < (first + count)[:, None])
    src = (token[:, None] + slots - first[:, None]).clamp(0, s["T"] - 1)
    for codes, scale, x in ((s["k"], s["k_scale"], k), (s["v"], s["v_scale"], v)):
        old, held = codes.double(), scale.double()
        after = held.clone()
        for i in range(0, len(where), 512):
            at, new = idx[i:i + 512], x[src[i:i + 512]].transpose(1, 2)  # [pages, heads, slots, D]
            f, o = fresh[i:i + 512][:, None, :, None], (slots < first[i:i + 512][:, None])[:, None, :, None]
            amax = torch.where(f, new.abs(), 0.0).amax((2, 3))
            fl = torch.floor(torch.log2(127.0 / amax.clamp(min=1e-300))).clamp(FL_LO, FL_HI)
            fl = torch.where(amax * torch.exp2(fl) > 127, fl - 1, fl)
            fl = torch.where(amax * torch.exp2(fl + 1) <= 127, fl + 1, fl).clamp(FL_LO, FL_HI)
            sc = torch.maximum(torch.exp2(-fl), torch.where(first[i:i + 512][:, None] > 0, held[at], 0.0))
            after[at] = sc
            sc = sc[:, :, None, None]
            page = torch.where(o, (old[at] * (held[at][:, :, None, None] / sc)).round(), old[at])
            old[at] = torch.where(f, (new / sc).round().clamp(-128, 127), page)
        out += [old * after[:, :, None, None], after]
    return q, out[0], out[2], out[1], out[3]


def _exact_attend(s):
    c = s["c"]
    if work(c)["flops"] > 3e12:
        return None
    lens = s["lens"].tolist()
    starts = s["starts"].tolist() if s["starts"] is not None else [i * (s["T"] // c["B"]) for i in range(c["B"] + 1)]
    Hq, Hkv, D, S = c["Hq"], c["Hkv"], c["D"], c["page"]
    out = torch.zeros(s["T"], Hq, D, dtype=torch.float64, device=s["q"].device)
    lse = torch.full((s["T"], Hq), -math.inf, dtype=torch.float64, device=s["q"].device)
    for b in range(c["B"]):
        n, L = starts[b + 1] - starts[b], lens[b]
        if not n or not L:
            continue
        at = s["pages"][b, :-(-L // S)].long()
        pos = torch.arange(L - n, L, device=out.device)
        for h in range(Hkv):
            k = (s["k"][at, h].double() * s["k_scale"][at, h].double()[:, None, None]).flatten(0, 1)[:L]
            v = (s["v"][at, h].double() * s["v_scale"][at, h].double()[:, None, None]).flatten(0, 1)[:L]
            for g in range(h * (Hq // Hkv), (h + 1) * (Hq // Hkv)):
                w = s["q"][starts[b]:starts[b] + n, g].double() @ k.t() * s["scale"]
                if c["causal"]:
                    w = w.masked_fill(torch.arange(L, device=out.device) > pos[:, None], -math.inf)
                lse[starts[b]:starts[b] + n, g] = torch.logsumexp(w, 1)
                out[starts[b]:starts[b] + n, g] = torch.softmax(w, 1) @ v
    return (out, lse) if c["lse"] else out
