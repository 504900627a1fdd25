"""Decoder layers of language models in 8 bits: rows quantized with a scale each, products of 8-bit rows,
and a paged cache of 8-bit keys and values with attention over it.

Torch tensors in, torch tensors out; every step runs in the library's kernels on the current stream, which
is also the stream that the results belong to.  Shapes and types are checked here, sizes, strides and
alignment in the library (``_lib.FxpqError``).  What a kernel finds wrong with the data (non-finite values,
page ids outside the cache, positions past the rotation tables) is latched and read by
``fxpq.fxpq_get_device_status``.
"""
from __future__ import annotations

import math

import torch

from . import _lib as L
from . import fxpq as F

_FT = {torch.float32: L.FT_F32, torch.float16: L.FT_F16, torch.bfloat16: L.FT_BF16}


def _ftype(name, dtype, types=_FT):
    if dtype not in types:
        raise TypeError(f"{name}: {dtype} is none of {', '.join(str(t) for t in types)}")
    return types[dtype]


def _want(name, t, dtype, dims):
    if not t.is_cuda or t.dtype != dtype or t.dim() != dims or not t.is_contiguous():
        raise ValueError(f"{name}: a contiguous {dims}-dimensional CUDA tensor of {dtype} is needed, "
                         f"got {tuple(t.shape)} of {t.dtype} on {t.device}, strides {t.stride()}")


def quantize_tokens(x):
    """Rows x [..., K] (float32, float16 or bfloat16) -> (codes int8 [..., K], scales float32 [...]), value =
    code * scale.  The codes' rows lie a multiple of 16 bytes apart, as `linear_i8` needs them."""
    ft = _ftype("quantize_tokens", x.dtype)
    if not x.is_cuda or x.dim() < 1:
        raise ValueError(f"quantize_tokens: rows on a CUDA device are needed, got {tuple(x.shape)} on {x.device}")
    K, lead = x.shape[-1], x.shape[:-1]
    rows = x if x.dim() == 2 else x.reshape(math.prod(lead), K)
    if K > 1 and rows.stride(1) != 1:
        rows = rows.contiguous()
    M, pitch = rows.shape[0], (K + 15) // 16 * 16
    codes = torch.empty((M, pitch), dtype=torch.int8, device=x.device)
    scale = torch.empty(M, dtype=torch.float32, device=x.device)
    F.fxpq_quantize_tokens(rows, ft, M, K, rows.stride(0), codes, pitch, scale)
    if pitch != K:
        codes = codes[:, :K]
    return (codes, scale) if x.dim() == 2 else (codes.unflatten(0, lead) if lead else codes[0], scale.view(lead))


def linear_i8(codes, scale, w, w_scale, bias=None, out_dtype=torch.bfloat16):
    """y [M, N] = (codes [M, K] . w [N, K]^T) * scale[:, None] * w_scale + bias.  Both code tensors: rows a multiple of
    16 bytes apart (`quantize_tokens` makes such rows)."""
    ft = _ftype("linear_i8", out_dtype)
    M, K = codes.shape
    N = w.shape[0]
    if codes.dtype != torch.int8 or w.dtype != torch.int8 or w.dim() != 2 or w.shape[1] != K:
        raise ValueError(f"linear_i8: int8 rows of one length are needed, got {tuple(codes.shape)} of {codes.dtype} and "
                         f"{tuple(w.shape)} of {w.dtype}")
    if (K > 1 and (codes.stride(1) != 1 or w.stride(1) != 1)) or not codes.is_cuda or not w.is_cuda:
        raise ValueError("linear_i8: the codes of a row must be contiguous and on a CUDA device")
    _want("linear_i8: scale", scale, torch.float32, 1)
    _want("linear_i8: w_scale", w_scale, torch.float32, 1)
    if bias is not None:
        _want("linear_i8: bias", bias, torch.float32, 1)
    if scale.shape[0] != M or w_scale.shape[0] != N or (bias is not None and bias.shape[0] != N):
        raise ValueError("linear_i8: one scale for each token, one scale and bias for each channel are needed")
    y = torch.empty((M, N), dtype=out_dtype, device=codes.device)
    need = F.fxpq_linear_i8_workspace(M, N, K)
    ws = torch.empty(need, dtype=torch.uint8, device=codes.device) if need else None
    F.fxpq_linear_i8(codes, _pitch(codes, K), scale, w, _pitch(w, K), w_scale, bias, M, N, K, ft, y, N, ws)
    return y


def _pitch(t, K):  # (a single row, or rows of nothing, may have any stride)
    return t.stride(0) if t.shape[0] > 1 and K else (K + 15) // 16 * 16


class Linear8:
    """A layer with 8-bit weights w int8 [N, K], one scale for each output channel: rows that are not whole 16 bytes
    are padded once."""

    def __init__(self, w, w_scale, bias=None):
        _want("Linear8: w", w, torch.int8, 2)
        N, K = w.shape
        if K % 16 or w.data_ptr() % 16:
            padded = torch.zeros((N, (K + 15) // 16 * 16), dtype=torch.int8, device=w.device)
            padded[:, :K] = w
            w = padded[:, :K]
        self.w, self.w_scale, self.bias = w, w_scale, bias

    @classmethod
    def from_float(cls, w, bias=None):
        """Quantizes float weights [N, K]."""
        codes, scale = quantize_tokens(w)
        layer = cls.__new__(cls)
        layer.w, layer.w_scale, layer.bias = codes, scale, None if bias is None else bias.float().contiguous()
        return layer

    def __call__(self, x, out_dtype=None):
        """x [..., K] in a float type -> [..., N] in out_dtype (x's own by default)."""
        rows = x if x.dim() == 2 else x.reshape(-1, x.shape[-1])
        codes, scale = quantize_tokens(rows)
        y = linear_i8(codes, scale, self.w, self.w_scale, self.bias, out_dtype or x.dtype)
        return y if x.dim() == 2 else y.view(*x.shape[:-1], y.shape[-1])


class KVCache:
    """A paged cache: int8 codes k, v [n_pages, heads, page, dim] and float32 scales [n_pages, heads], one for each
    block (a page of one head).  page is 16, 32, 64 or 128, dim 64 or 128."""

    def __init__(self, k, v, k_scale, v_scale):
        _want("KVCache: k", k, torch.int8, 4)
        _want("KVCache: v", v, torch.int8, 4)
        _want("KVCache: k_scale", k_scale, torch.float32, 2)
        _want("KVCache: v_scale", v_scale, torch.float32, 2)
        if v.shape != k.shape or k_scale.shape != k.shape[:2] or v_scale.shape != k.shape[:2]:
            raise ValueError("KVCache: k and v of one shape and a scale for each page and head are needed")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.n_pages, self.heads, self.page, self.dim = k.shape
        self.desc = L.KVCacheDesc(k.data_ptr(), v.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(), self.n_pages, self.page,
                                  self.heads, self.dim)

    @classmethod
    def empty(cls, n_pages, heads, page, dim, device="cuda"):
        codes = [torch.zeros((n_pages, heads, page, dim), dtype=torch.int8, device=device) for _ in range(2)]
        return cls(*codes, *[torch.ones((n_pages, heads), dtype=torch.float32, device=device) for _ in range(2)])


def _batch(name, pages, lens, starts, T):
    if pages.dtype != torch.int32 or pages.dim() != 2 or (pages.shape[1] > 1 and pages.stride(1) != 1) or not pages.is_cuda:
        raise ValueError(f"{name}: pages must be int32 [sequences, pages] on a CUDA device")
    _want(f"{name}: lens", lens, torch.int32, 1)
    B = lens.shape[0]
    if pages.shape[0] != B:
        raise ValueError(f"{name}: {pages.shape[0]} rows of pages and {B} lengths")
    if starts is not None:
        _want(f"{name}: starts", starts, torch.int32, 1)
        if starts.shape[0] != B + 1:
            raise ValueError(f"{name}: starts must have {B + 1} entries")
    elif B and T % B:
        raise ValueError(f"{name}: {T} new tokens are not the same number for each of {B} sequences (give starts)")
    wide = pages.shape[1]
    return L.KVBatchDesc(pages.data_ptr(), lens.data_ptr(), None if starts is None else starts.data_ptr(), B, wide, T, 0,
                         pages.stride(0) if B > 1 else max(wide, 1))


def _rows(name, x, T, heads, dim):
    if x.dim() != 3 or tuple(x.shape) != (T, heads, dim) or not x.is_cuda or x.stride(2) != 1:
        raise ValueError(f"{name}: rows [{T}, {heads}, {dim}] with contiguous heads are needed, got {tuple(x.shape)} with "
                         f"strides {x.stride()}")
    return L.KVRows(x.data_ptr(), x.stride(0), x.stride(1))


def kv_append(cache, pages, lens, k, v, q=None, starts=None, cos=None, sin=None, interleaved=False):
    """Appends new keys and values k, v [T, heads, dim] to the cache; returns the rotated queries [T, q_heads, dim]
    (None without q).

    pages int32 [B, n]: each sequence's pages; lens int32 [B]: tokens of each sequence, the new ones included; starts
    int32 [B + 1]: where each sequence's new tokens begin among the T rows (None: T / B each).
    cos, sin float32 [positions, rot / 2]: keys and queries turn by their positions in their first rot values, pairs
    (i, i + rot / 2) or with interleaved (2 i, 2 i + 1).  k, v and q may be views with any token and head strides."""
    if k.dim() != 3:
        raise ValueError(f"kv_append: k must be [tokens, heads, dim], got {tuple(k.shape)}")
    T = k.shape[0]
    ft = _ftype("kv_append", k.dtype)
    if v.dtype != k.dtype or (q is not None and q.dtype != k.dtype):
        raise TypeError("kv_append: k, v and q must have one type")
    batch = _batch("kv_append", pages, lens, starts, T)
    rk, rv = _rows("kv_append: k", k, T, cache.heads, cache.dim), _rows("kv_append: v", v, T, cache.heads, cache.dim)
    rq = out = None
    heads = 0
    if q is not None:
        heads = q.shape[1] if q.dim() == 3 else 0
        rq = _rows("kv_append: q", q, T, heads, cache.dim)
        out = torch.empty((T, heads, cache.dim), dtype=q.dtype, device=q.device)
    n_pos = rot = 0
    if (cos is None) != (sin is None):
        raise ValueError("kv_append: cos and sin go together")
    if cos is not None:
        _want("kv_append: cos", cos, torch.float32, 2)
        _want("kv_append: sin", sin, torch.float32, 2)
        if cos.shape != sin.shape:
            raise ValueError("kv_append: cos and sin must have one shape")
        n_pos, rot = cos.shape[0], 2 * cos.shape[1]
    F.fxpq_kv_append(cache.desc, batch, ft, rk, rv, rq, heads, out, cos, sin, n_pos, rot, int(interleaved))
    return out


def kv_values(cache, pages, dtype=torch.bfloat16):
    """The values code * scale of the pages int32 [n]: keys and values [n, heads, page, dim]."""
    _want("kv_values: pages", pages, torch.int32, 1)
    n = pages.shape[0]
    k, v = (torch.empty((n, cache.heads, cache.page, cache.dim), dtype=dtype, device=pages.device) for _ in range(2))
    F.fxpq_kv_values(cache.desc, pages, n, _ftype("kv_values", dtype), k, v)
    return k, v


_Q_TYPES = {torch.float16: L.FT_F16, torch.bfloat16: L.FT_BF16}


def kv_attention(cache, pages, lens, q, starts=None, scale=None, causal=True, return_lse=False):
    """Softmax attention of the queries q [T, q_heads, dim] (float16 or bfloat16, any token and head strides) of the
    last tokens of each sequence over the cache, which already holds those tokens; q_heads is a multiple of the
    cache's heads.  scale: 1 / sqrt(dim) by default.  Returns [T, q_heads, dim], and with return_lse the logarithms
    float32 [T, q_heads] of the sums of exponentials; rows that see no key are zeros and -inf."""
    ft = _ftype("kv_attention", q.dtype, _Q_TYPES)
    if q.dim() != 3:
        raise ValueError(f"kv_attention: q must be [tokens, heads, dim], got {tuple(q.shape)}")
    T, heads = q.shape[0], q.shape[1]
    if heads == 0 or heads % cache.heads:
        raise ValueError(f"kv_attention: {heads} query heads are no multiple of {cache.heads}")
    batch = _batch("kv_attention", pages, lens, starts, T)
    rq = _rows("kv_attention: q", q, T, heads, cache.dim)
    out = torch.empty((T, heads, cache.dim), dtype=q.dtype, device=q.device)
    lse = torch.empty((T, heads), dtype=torch.float32, device=q.device) if return_lse else None
    need = F.fxpq_kv_attention_workspace(cache.desc, batch, heads)
    ws = torch.empty(need, dtype=torch.uint8, device=q.device) if need else None
    F.fxpq_kv_attention(cache.desc, batch, ft, rq, heads, 1.0 / math.sqrt(cache.dim) if scale is None else float(scale),
                        int(bool(causal)), out, lse, ws)
    return (out, lse) if return_lse else out
