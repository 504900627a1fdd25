"""Workloads of the 8-bit layers with their norm, epilogue and gate inside, and of their gradients, in plain torch and
through this library.

A case is a plain dict.  `listed` names twelve, `draw` gives others of the same ranges, `prepare` makes
what a program holds before the call, `run` is one pass, `work` the bytes and operations that a pass
cannot do without, and `exact` the same results from the definitions in 64 bits.

Operators, with z = (codes(n(x)) . w^T) * sx[token] * sw[channel] + bias, codes(n(x)) the rows quantized to 8 bits with a
scale each, and n(x) = x, or x / sqrt(mean(x^2) + eps) * weight
  layer       y = act(z) + residual;
  gated       y = act(z_gate) * z_up, both products of the same rows;
  layer_grad, gated_grad   a training pass: y as above and, for dy, the gradient dx of the layer whose weights are frozen,
              dx = dz . (w * sw), dz = dy * act'(z), or dz_gate = dy * z_up * act'(z_gate) and dz_up = dy * act(z_gate);
              the rounding to codes counts as the identity.

`own` False: elementary torch operations in 32 bits, rounded once at the end.  `own` True: the calls that
a user makes of the library.
"""
from __future__ import annotations

import math
import random

import torch

own = False

EPS = 1e-5
_FT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
_BYTES = {"bf16": 2, "f16": 2, "f32": 4}


# ------------------------------------------------------------------------------ cases
def listed():
    return [
        # one token through the layer that ends an attention block, added to its input: decoding alone, the weights' read
        _case("layer_token", "layer", M=1, N=4096, K=4096, dtype="bf16", res=1),
        # a batch through the largest FC layer of the library's networks (25088 inputs) and its ReLU
        _case("layer_batch", "layer", M=64, N=4096, K=25088, dtype="f16", bias=1, act="relu"),
        # a short prompt, odd in tokens, channels and inputs, with everything around the product, kept in 32 bits
        _case("layer_odd", "layer", M=251, N=1001, K=4090, dtype="f16", out="f32", bias=1, act="gelu", res=1, norm=1),
        # prompts packed into one matrix through the layer that ends a feed-forward block, added to its input: tensor-core bound
        _case("layer_prompt", "layer", M=8192, N=4096, K=16384, dtype="bf16", res=1),
        # one token through the feed-forward block of the library's decoder
        _case("gated_token", "gated", M=1, N=5632, K=2048, dtype="bf16", norm=1),
        # a serving batch decoding through a large feed-forward block
        _case("gated_batch", "gated", M=64, N=16384, K=4096, dtype="f16", norm=1),
        # a prompt of some hundred tokens, nothing a multiple of anything, biases
        _case("gated_odd", "gated", M=777, N=1365, K=2050, dtype="bf16", act="gelu_tanh", bias=1),
        # prompts packed into one matrix: tensor-core bound
        _case("gated_prompt", "gated", M=8192, N=16384, K=4096, dtype="bf16", norm=1),
        # training what lies below a frozen classifier: a small batch, odd in tokens
        _case("layer_grad_small", "layer_grad", M=50, N=1000, K=4096, dtype="f16", bias=1, act="gelu"),
        # training below the layer that ends a large feed-forward block
        _case("layer_grad_large", "layer_grad", M=4096, N=4096, K=16384, dtype="bf16", res=1),
        # training below a feed-forward block of odd sizes, activations and gradients in 32 bits
        _case("gated_grad_odd", "gated_grad", M=517, N=2749, K=1030, dtype="f32", act="gelu", bias=1),
        # training below the feed-forward block of the library's decoder, packed sequences
        _case("gated_grad_large", "gated_grad", M=8192, N=5632, K=2048, dtype="bf16"),
    ]


def _case(name, kind, dtype, **kw):
    c = {"kind": kind, "dtype": dtype, "out": dtype, "bias": 0, "res": 0, "norm": 0, "act": "silu" if "gated" in kind else "none", **kw}
    if name:
        c["name"] = name
    return c


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


_LARGEST = 2 * 8192 * 2 * 16384 * 4096  # operations of gated_prompt


def draw(rng: random.Random):
    kind = rng.choice(["layer", "layer", "gated", "gated", "layer_grad", "gated_grad"])
    gated, grad = "gated" in kind, "grad" in kind
    while True:
        c = _case(None, kind, rng.choice(["bf16", "bf16", "bf16", "f16", "f16", "f32"]), M=_log(rng, 1, 8192), N=_log(rng, 64, 16384),
                  K=_log(rng, 64, 8192 if gated else 25088), bias=rng.randint(0, 1), res=0 if gated else rng.randint(0, 1),
                  norm=0 if grad else rng.randint(0, 1))
        # (ReLU's derivative jumps: a code that rounds the other way turns whole terms of a gradient on or off)
        smooth = ["silu", "gelu", "gelu_tanh"] + ([] if grad else ["relu"])
        c["act"] = rng.choice(smooth if gated else ["none", "none"] + smooth)
        if rng.random() < 0.15:
            c["out"] = "f32"
        if rng.random() < 0.5:  # layers are mostly multiples of 64; the rest are odd
            c["N"], c["K"] = (c["N"] + 63) // 64 * 64, (c["K"] + 63) // 64 * 64
        if work(c)["flops"] <= _LARGEST and work(c)["bytes"] <= 1.2e9:
            return c


def work(case):
    c = case
    M, N, K = c["M"], c["N"], c["K"]
    sides = 2 if "gated" in c["kind"] else 1
    xb, yb, grad = _BYTES[c["dtype"]], _BYTES[c["out"]], "grad" in c["kind"]
    constants = sides * N * (K + 4 * (1 + c["bias"])) + 4 * K * c["norm"]
    rows = xb * M * K * (2 if grad else 1) + yb * M * N * (1 + c["res"] + (1 if grad else 0))
    return {"bytes": constants + rows, "flops": 2 * sides * M * N * K * (2 if grad else 1)}


# ------------------------------------------------------------------------------ inputs
def _codes(shape, g, spread):
    """8-bit codes of a normal tensor, in pieces so that large ones need no large scratch."""
    out = torch.empty(shape, dtype=torch.int8, device="cuda")
    flat = out.view(-1)
    for i in range(0, flat.numel(), 1 << 28):
        part = flat[i:i + (1 << 28)]
        part.copy_((torch.randn(part.numel(), device="cuda", generator=g) * spread).round_().clamp_(-127, 127))
    return out


def prepare(case, seed):
    c, g = case, torch.Generator(device="cuda").manual_seed(int(seed))
    M, N, K = c["M"], c["N"], c["K"]

    def normal(*shape):
        return torch.randn(*shape, device="cuda", generator=g)
    # activations of tokens of unequal size, a few inputs larger than the rest
    x = normal(M, K) * torch.exp(0.5 * normal(M, 1))
    x *= torch.where(torch.rand(K, device="cuda", generator=g) < 0.01, 8.0, 1.0)
    s = {"c": c, "x": x.to(_FT[c["dtype"]]), "out": _FT[c["out"]], "act": None if c["act"] == "none" else c["act"],
         "norm": torch.exp(0.2 * normal(K)) if c["norm"] else None, "res": normal(M, N).to(_FT[c["out"]]) if c["res"] else None}
    s["w"], s["sw"], s["bias"] = [], [], []
    for _ in range(2 if "gated" in c["kind"] else 1):
        s["w"].append(_codes((N, K), g, 32.0))
        s["sw"].append(torch.exp(0.3 * normal(N)) * (1.0 / (32 * math.sqrt(K))))
        s["bias"].append(normal(N) * 0.1 if c["bias"] else None)
    if "grad" in c["kind"]:
        # gradients of tokens of unequal weight, some of which the loss leaves out
        live = torch.rand(M, 1, device="cuda", generator=g) >= 0.1
        s["dy"] = (normal(M, N) * torch.exp(0.5 * normal(M, 1)) * 0.02 * live).to(s["out"])
        s["x"].requires_grad_()
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
    if not own:
        with torch.no_grad():
            return _plain(state)
    s = state
    kind, ops = s["c"]["kind"], _ops()
    if "layer" not in s:  # the layer that a program keeps: its weights in the order that the kernels read, for gradients transposed too
        if "gated" in kind:
            s["layer"] = ops.GatedLinear8(s["w"][0], s["sw"][0], s["w"][1], s["sw"][1], gate_bias=s["bias"][0], up_bias=s["bias"][1],
                                          activation=s["act"])
        else:
            s["layer"] = ops.Linear8(s["w"][0], s["sw"][0], s["bias"][0])
        if "grad" in kind:
            s["layer"].with_gradient()
    if kind == "gated":
        return s["layer"](s["x"], s["out"], norm=s["norm"], eps=EPS)
    if kind == "layer":
        return s["layer"](s["x"], s["out"], norm=s["norm"], eps=EPS, activation=s["act"], residual=s["res"])
    with torch.enable_grad():
        if kind == "gated_grad":
            y = s["layer"](s["x"], s["out"])
        else:
            y = s["layer"](s["x"], s["out"], activation=s["act"], residual=s["res"])
        dx, = torch.autograd.grad(y, s["x"], s["dy"])
    return y.detach(), dx


def _act(z, name):
    """act(z) and act'(z)"""
    if name is None:
        return z, torch.ones_like(z)
    if name == "relu":
        return z.clamp(min=0), (z > 0).to(z.dtype)
    if name == "silu":
        p = torch.sigmoid(z)
        return z * p, p + z * p * (1 - p)
    if name == "gelu":
        p = 0.5 * (1 + torch.erf(z * math.sqrt(0.5)))
        return z * p, p + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    a = math.sqrt(2 / math.pi)  # gelu_tanh
    t = torch.tanh(a * (z + 0.044715 * z ** 3))
    return 0.5 * z * (1 + t), 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * a * (1 + 3 * 0.044715 * z * z)


def _plain(s):
    x = s["x"].float()
    n = x if s["norm"] is None else x * s["norm"]
    amax = n.abs().amax(1, keepdim=True)
    codes = (n * torch.where(amax > 0, (1.0 / amax) * 127.0, 0.0)).round().clamp(-127, 127)
    sx = amax * (1.0 / 127.0)
    if s["norm"] is not None:
        sx = sx * torch.rsqrt(x.square().mean(1, keepdim=True) + EPS)
    z = []
    for w, sw, bias in zip(s["w"], s["sw"], s["bias"]):
        z.append((codes @ w.float().t()).mul_(sx).mul_(sw))
        if bias is not None:
            z[-1] += bias
    f, df = _act(z[0], s["act"])
    y = f * z[1] if len(z) > 1 else f if s["res"] is None else f + s["res"].float()
    y = y.to(s["out"])
    if "grad" not in s["c"]["kind"]:
        return y
    dy = s["dy"].float()
    dz = [dy * z[1] * df, dy * f] if len(z) > 1 else [dy * df]
    dx = sum((d * sw) @ w.float() for d, w, sw in zip(dz, s["w"], s["sw"]))
    return y, dx.to(s["x"].dtype)


# ------------------------------------------------------------------------------ the definitions in 64 bits
def exact(case, seed):
    with torch.no_grad():
        s = prepare(case, seed)
        parts = [_exact_rows(s, i, min(i + 1024, case["M"])) for i in range(0, case["M"], 1024)]
        if "grad" not in case["kind"]:
            return torch.cat(parts)
        return torch.cat([p[0] for p in parts]), torch.cat([p[1] for p in parts])


def _exact_rows(s, lo, hi):
    v = s["x"][lo:hi].double()
    if s["norm"] is not None:
        v = v / (v.pow(2).sum(1, keepdim=True) / v.shape[1] + EPS).sqrt() * s["norm"].double()
    step = v.abs().max(1, keepdim=True).values / 127
    rows = torch.where(step > 0, v / step, 0.0).round() * step  # the values that the codes stand for
    weights = [w.double() * sw.double()[:, None] for w, sw in zip(s["w"], s["sw"])]
    z = [rows @ w.t() if b is None else rows @ w.t() + b.double() for w, b in zip(weights, s["bias"])]
    g, name = z[0], s["act"]
    if name is None:
        f, slope = g, torch.ones_like(g)
    elif name == "relu":
        f, slope = torch.where(g > 0, g, 0.0), torch.where(g > 0, 1.0, 0.0)
    elif name == "gelu":
        cdf = 0.5 * torch.erfc(-g / math.sqrt(2))
        f, slope = g * cdf, cdf + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    else:  # silu, and gelu_tanh as g / (1 + exp(-2 u))
        u, du = (g, 1.0) if name == "silu" else (2 * math.sqrt(2 / math.pi) * (g + 0.044715 * g.pow(3)),
                                                2 * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * g.pow(2)))
        p = 1 / (1 + torch.exp(-u))
        f, slope = g * p, p + g * p * (1 / (1 + torch.exp(u))) * du
    y = f * z[1] if len(z) > 1 else f
    if s["res"] is not None:
        y = y + s["res"][lo:hi].double()
    if "grad" not in s["c"]["kind"]:
        return y
    dy = s["dy"][lo:hi].double()
    dx = (dy * slope * (z[1] if len(z) > 1 else 1.0)) @ weights[0]
    if len(z) > 1:
        dx = dx + (dy * f) @ weights[1]
    return y, dx
