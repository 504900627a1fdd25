"""CPU oracle of the 8-bit language-model operators (numpy), written from their definitions.

Codes, scales and rotations follow the definitions' own fp32 steps, so integer outputs compare bit for
bit; products and attention are in 64 bits.
"""
from __future__ import annotations

import math

import numpy as np

FL_LO, FL_HI = -32, 40
f32 = np.float32


def quantize_tokens(x):
    """Rows [M, K] of fp32 values -> (codes int8, scales fp32)."""
    x = np.asarray(x, dtype=f32)
    a = np.max(np.where(np.isfinite(x), np.abs(x), f32(0)), axis=1, initial=0).astype(f32)
    live = a >= f32(2.0 ** -100)
    inv = np.where(live, (f32(1) / np.where(live, a, f32(1))) * f32(127), f32(0)).astype(f32)
    scale = np.where(live, a * (f32(1) / f32(127)), f32(0)).astype(f32)
    v = np.where(np.isfinite(x), x, f32(0)) * inv[:, None]
    return np.clip(np.rint(v), -127, 127).astype(np.int8), scale


def linear(codes, scale, w, w_scale, bias=None):
    """(y in 64 bits, sum of |products| scaled alike)."""
    c, ww = codes.astype(np.int64), w.astype(np.int64)
    s = scale.astype(np.float64)[:, None] * w_scale.astype(np.float64)
    y = (c @ ww.T) * s
    b = 0.0 if bias is None else bias.astype(np.float64)
    return y + b, (np.abs(c) @ np.abs(ww).T) * s + np.abs(b)


def block_scale(a):
    """The smallest 2^-FL, FL in [FL_LO, FL_HI], with a <= 127 * 2^-FL."""
    for fl in range(FL_HI, FL_LO - 1, -1):
        if float(a) <= 127.0 * 2.0 ** -fl:
            return 2.0 ** -fl
    return 2.0 ** -FL_LO


def rotate(x, pos, cos, sin, rot, interleaved):
    """x [..., D] fp32 at position pos; every product and sum rounded to fp32."""
    y = np.array(x, dtype=f32)
    i, j = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    a, b, c, s = y[..., i].copy(), y[..., j].copy(), cos[pos], sin[pos]
    y[..., i] = a * c - b * s
    y[..., j] = b * c + a * s
    return y


class Cache:
    def __init__(self, k, v, k_scale, v_scale):
        self.k, self.v, self.k_scale, self.v_scale = (np.array(t) for t in (k, v, k_scale, v_scale))

    def values(self, b_pages, n, head, which):
        """The first n tokens of a page list in 64 bits."""
        codes, scale = (self.k, self.k_scale) if which == "k" else (self.v, self.v_scale)
        page = codes.shape[2]
        out = [codes[b_pages[p // page], head, p % page].astype(np.float64) * float(scale[b_pages[p // page], head]) for p in range(n)]
        return np.array(out).reshape(n, codes.shape[3])


def _append_rows(codes, scale, page_id, head, slot0, x):
    """Rows x [n, D] (fp32) into slots slot0 .. of one block."""
    fin = np.isfinite(x)
    x = np.where(fin, x, f32(0))
    before = f32(scale[page_id, head]) if slot0 > 0 else f32(0)
    after = max(before, f32(block_scale(np.max(np.abs(x)))))
    if slot0 > 0 and after != before:
        old = codes[page_id, head, :slot0].astype(f32) * f32(before / after)
        codes[page_id, head, :slot0] = np.clip(np.rint(old), -128, 127).astype(np.int8)
    scale[page_id, head] = after
    codes[page_id, head, slot0:slot0 + len(x)] = np.clip(np.rint((x / after).astype(f32)), -128, 127).astype(np.int8)


def append(cache, pages, lens, starts, k, v, q=None, cos=None, sin=None, interleaved=False):
    """k, v, q: fp32 [T, heads, D].  Updates the cache; returns the rotated queries (fp32, not rounded further)."""
    page, rot = cache.k.shape[2], 0 if cos is None else 2 * cos.shape[1]
    out = None if q is None else np.zeros(q.shape, dtype=f32)
    for b in range(len(lens)):
        t0, n = starts[b], starts[b + 1] - starts[b]
        p = lens[b] - n
        if p < 0:
            t0, n, p = t0 - p, n + p, 0
        while n > 0:
            m = min(n, page - p % page)
            live = m if rot == 0 else max(0, min(m, len(cos) - p))
            for i in range(live if out is not None else 0):
                out[t0 + i] = rotate(q[t0 + i], p + i, cos, sin, rot, interleaved) if rot else q[t0 + i]
            pid = pages[b][p // page] if p // page < len(pages[b]) else -1
            if 0 <= pid < len(cache.k) and live:
                for h in range(cache.k.shape[1]):
                    kk = np.stack([rotate(k[t0 + i, h], p + i, cos, sin, rot, interleaved) if rot else k[t0 + i, h] for i in range(live)])
                    _append_rows(cache.k, cache.k_scale, pid, h, p % page, kk.astype(f32))
                    _append_rows(cache.v, cache.v_scale, pid, h, p % page, v[t0:t0 + live, h].astype(f32))
            t0, n, p = t0 + m, n - m, p + m
    return out


def attention(cache, pages, lens, starts, q, scale, causal):
    """(out, lse, spread, slack) in 64 bits for q [T, Hq, D]: spread = sum_p softmax |value|, and slack = the largest
    sum_i |q_i key_i| * scale of a row (what bounds the rounding of its scores)."""
    T, Hq, D = q.shape
    G = Hq // cache.k.shape[1]
    out, spread = np.zeros((T, Hq, D)), np.zeros((T, Hq, D))
    lse, slack = np.full((T, Hq), -np.inf), np.zeros((T, Hq))
    for b in range(len(lens)):
        n = starts[b + 1] - starts[b]
        if n == 0 or lens[b] == 0:
            continue
        for h in range(cache.k.shape[1]):
            k, v = (cache.values(pages[b], lens[b], h, w) for w in "kv")
            for i in range(n):
                pos = lens[b] - n + i
                end = 0 if pos < 0 else pos + 1 if causal else lens[b]
                if end == 0:
                    continue
                qq = q[starts[b] + i, h * G:(h + 1) * G].astype(np.float64)
                s = qq @ k[:end].T * scale
                m = s.max(1, keepdims=True)
                w = np.exp(s - m)
                l = w.sum(1, keepdims=True)
                t, g = starts[b] + i, slice(h * G, (h + 1) * G)
                out[t, g], spread[t, g] = (w / l) @ v[:end], (w / l) @ np.abs(v[:end])
                lse[t, g] = (m + np.log(l))[:, 0]
                slack[t, g] = (np.abs(qq) @ np.abs(k[:end]).T).max(1) * scale
    return out, lse, spread, slack


def paged(rng, lens, page, heads, dim, spare=2, arbitrary=False):
    """A random cache for sequences of the given lengths: (Cache, table [B, pages] with -1 past each sequence)."""
    need = [-(-n // page) for n in lens]
    total = sum(need) + spare
    order = rng.permutation(total)
    table = np.full((len(lens), max(1, max(need, default=1))), -1, dtype=np.int32)
    at = 0
    for b, m in enumerate(need):
        table[b, :m] = order[at:at + m]
        at += m
    codes = [np.clip(np.rint(rng.normal(0, 30, (total, heads, page, dim))), -127, 127).astype(np.int8) for _ in range(2)]
    e = [rng.integers(4, 7, (total, heads)) + (rng.random((total, heads)) if arbitrary else 0.0) for _ in range(2)]
    return Cache(*codes, *[np.exp2(-x).astype(f32) for x in e]), table


def rope_tables(n, rot):
    a = np.arange(n)[:, None] * 10000.0 ** (-np.arange(rot // 2) / (rot / 2))
    return np.cos(a).astype(f32), np.sin(a).astype(f32)


def default_scale(dim):
    return 1.0 / math.sqrt(dim)
