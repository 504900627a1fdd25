"""Decoder layers of language models in 8 bits: rows quantized with a scale each, products of 8-bit rows,
and a paged cache of 8-bit keys and values with attention over it.

Torch tensors in, torch tensors out; every step runs in the library's kernels on the current stream, which
is also the stream that the results belong to.  Shapes and types are checked here, sizes, strides and
alignment in the library (``_lib.FxpqError``).  What a kernel finds wrong with the data (non-finite values,
page ids outside the cache, positions past the rotation tables) is latched and read by
``fxpq.fxpq_get_device_status``.

The operators are for inference and have no gradient: tensors that require one are refused while gradients are
recorded (RuntimeError).
"""
from __future__ import annotations

import math
import struct

import torch

from . import _lib as L
from . import fxpq as F

# Small calls are bound by the host, so arguments are marshalled by hand here: descriptors packed as bytes (0.3 us, a
# ctypes structure 1.1), no views, one allocation where there were two.  One token through a 4096 x 4096 layer took 25.8 us
# on the host with two wrapped calls; 8.8 on the GPU.
_FT = {torch.float32: L.FT_F32, torch.float16: L.FT_F16, torch.bfloat16: L.FT_BF16}
_BATCH = struct.Struct("PPPiiiiq").pack  # fxpq_kv_batch
_ROWS = struct.Struct("Pqq").pack        # fxpq_kv_rows
_empty, _i8, _i32, _u8, _f32 = torch.empty, torch.int8, torch.int32, torch.uint8, torch.float32


def _ftype(name, dtype, types=_FT):
    ft = types.get(dtype)
    if ft is None:
        raise TypeError(f"{name}: {dtype} is none of {', '.join(str(t) for t in types)}")
    return ft


def _no_grad(name, *tensors):
    """Refuses what would silently come back without its gradient."""
    if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in tensors):
        raise RuntimeError(f"{name} has no gradient: call it under torch.no_grad() or with detached tensors")


def _want(name, t, dtype, dims):
    if t.dtype != dtype or t.dim() != dims or not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{name}: a contiguous {dims}-dimensional CUDA tensor of {dtype} is needed, "
                         f"got {tuple(t.shape)} of {t.dtype} on {t.device}, strides {t.stride()}")


def _float_rows(name, x):
    """x [..., K] as [M, K] with contiguous rows that do not overlap (expanded ones and windows are copied)."""
    if not x.is_cuda or x.dim() < 1:
        raise ValueError(f"{name}: rows on a CUDA device are needed, got {tuple(x.shape)} on {x.device}")
    rows = x if x.dim() == 2 else x.reshape(math.prod(x.shape[:-1]), x.shape[-1])
    if rows.is_contiguous():
        return rows
    K = rows.shape[1]
    return rows if (rows.stride(1) == 1 or K <= 1) and rows.stride(0) >= K else rows.contiguous()


def quantize_tokens(x):
    """Rows x [..., K] (float32, float16 or bfloat16) -> (codes int8 [..., K], scales float32 [...]), value =
    code * scale.  The codes' rows lie a multiple of 16 bytes apart, as `linear_i8` needs them."""
    ft = _ftype("quantize_tokens", x.dtype)
    if x.requires_grad:
        _no_grad("quantize_tokens", x)
    rows = _float_rows("quantize_tokens", x)
    M, K = rows.shape
    pitch = (K + 15) // 16 * 16
    codes = _empty((M, pitch), dtype=_i8, device=x.device)
    scale = _empty(M, dtype=_f32, device=x.device)
    F.fxpq_quantize_tokens(rows, ft, M, K, rows.stride(0), codes, pitch, scale)
    if pitch != K:
        codes = codes[:, :K]
    if x.dim() == 2:
        return codes, scale
    lead = x.shape[:-1]
    return (codes.unflatten(0, lead) if lead else codes[0]), scale.view(lead)


def linear_i8(codes, scale, w, w_scale, bias=None, out_dtype=torch.bfloat16):
    """y [M, N] = (codes [M, K] . w [N, K]^T) * scale[:, None] * w_scale + bias.  Both code tensors: rows a multiple of
    16 bytes apart (`quantize_tokens` makes such rows)."""
    ft = _ftype("linear_i8", out_dtype)
    _no_grad("linear_i8", scale, w_scale, bias)
    M, K = codes.shape
    N = w.shape[0]
    if codes.dtype != _i8 or not codes.is_cuda or (K > 1 and codes.stride(1) != 1):
        raise ValueError(f"linear_i8: int8 rows on a CUDA device are needed, got {tuple(codes.shape)} of {codes.dtype} on {codes.device}")
    _check_layer("linear_i8", w, w_scale, bias, K)
    _want("linear_i8: scale", scale, _f32, 1)
    if scale.shape[0] != M:
        raise ValueError("linear_i8: one scale for each token is needed")
    y = _empty((M, N), dtype=out_dtype, device=codes.device)
    need = F.fxpq_linear_i8_workspace(M, N, K)
    ws = _empty(need, dtype=_u8, device=codes.device) if need else None
    F.fxpq_linear_i8(codes, _pitch(codes, K), scale, w, _pitch(w, K), w_scale, bias, M, N, K, ft, y, N, ws)
    return y


def _check_layer(name, w, w_scale, bias, K):
    if w.dtype != _i8 or w.dim() != 2 or not w.is_cuda or w.shape[1] != K or (K > 1 and w.stride(1) != 1):
        raise ValueError(f"{name}: weights int8 [N, {K}] with contiguous rows on a CUDA device are needed, got {tuple(w.shape)} of "
                         f"{w.dtype} on {w.device}")
    _want(f"{name}: w_scale", w_scale, _f32, 1)
    if bias is not None:
        _want(f"{name}: bias", bias, _f32, 1)
    if w_scale.shape[0] != w.shape[0] or (bias is not None and bias.shape[0] != w.shape[0]):
        raise ValueError(f"{name}: one scale and bias for each channel are needed")


def _pitch(t, K):  # (a single row, or rows of nothing, may have any stride)
    return t.stride(0) if t.shape[0] > 1 and K else (K + 15) // 16 * 16


class Linear8:
    """A layer with 8-bit weights w int8 [N, K], one scale for each output channel: rows that are not whole 16 bytes
    are padded once.  Its tensors are constants: what they require of a gradient is dropped."""

    def __init__(self, w, w_scale, bias=None):
        _want("Linear8: w", w, _i8, 2)
        N, K = w.shape
        if K % 16 or w.data_ptr() % 16:
            padded = torch.zeros((N, (K + 15) // 16 * 16), dtype=_i8, device=w.device)
            padded[:, :K] = w
            w = padded[:, :K]
        self._set(w, w_scale, bias)

    def _set(self, w, w_scale, bias):
        self.N, self.K = w.shape
        _check_layer("Linear8", w, w_scale, bias, self.K)
        self.w, self.w_scale, self.bias = w, w_scale.detach(), None if bias is None else bias.detach()

    @classmethod
    def from_float(cls, w, bias=None):
        """Quantizes float weights [N, K]."""
        layer = cls.__new__(cls)
        layer._set(*quantize_tokens(w.detach()), None if bias is None else bias.detach().float().contiguous())
        return layer

    def __call__(self, x, out_dtype=None):
        """x [..., K] in a float type -> [..., N] in out_dtype (x's own by default): `quantize_tokens` and `linear_i8`
        as one call."""
        if x.requires_grad:
            _no_grad("Linear8", x)
        rows = _float_rows("Linear8", x)
        M, K = rows.shape
        if K != self.K:
            raise ValueError(f"Linear8: rows of {self.K} values are needed, got {tuple(x.shape)}")
        dtype = out_dtype or x.dtype
        xt, yt = _ftype("Linear8", x.dtype), _ftype("Linear8", dtype)
        lib, dev, N, w = L.lib(), x.device, self.N, self.w
        y = _empty((M, N), dtype=dtype, device=dev)
        ws = _empty(lib.fxpq_linear_tokens_workspace(M, N, K), dtype=_u8, device=dev)
        rc = lib.fxpq_linear_tokens(rows.data_ptr(), xt, rows.stride(0), w.data_ptr(), _pitch(w, K), self.w_scale.data_ptr(),
                                    None if self.bias is None else self.bias.data_ptr(), M, N, K, yt, y.data_ptr(), N, ws.data_ptr(),
                                    ws.nbytes, F._s(None))
        if rc:
            L.check("fxpq_linear_tokens", rc)
        return y if x.dim() == 2 else y.view(*x.shape[:-1], N)


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
        self.packed = bytes(self.desc)  # fxpq_kv_cache

    @classmethod
    def empty(cls, n_pages, heads, page, dim, device="cuda"):
        codes = [torch.zeros((n_pages, heads, page, dim), dtype=torch.int8, device=device) for _ in range(2)]
        return cls(*codes, *[torch.ones((n_pages, heads), dtype=torch.float32, device=device) for _ in range(2)])


def _batch(name, pages, lens, starts, T):
    """fxpq_kv_batch"""
    B, wide = pages.shape if pages.dim() == 2 else (-1, 0)
    if pages.dtype != _i32 or B < 0 or not pages.is_cuda or (wide > 1 and pages.stride(1) != 1):
        raise ValueError(f"{name}: pages must be int32 [sequences, pages] on a CUDA device")
    _want(name + ": lens", lens, _i32, 1)
    if lens.shape[0] != B:
        raise ValueError(f"{name}: {B} rows of pages and {lens.shape[0]} lengths")
    at = 0
    if starts is not None:
        _want(name + ": starts", starts, _i32, 1)
        if starts.shape[0] != B + 1:
            raise ValueError(f"{name}: starts must have {B + 1} entries")
        at = starts.data_ptr()
    elif B and T % B:
        raise ValueError(f"{name}: {T} new tokens are not the same number for each of {B} sequences (give starts)")
    return _BATCH(pages.data_ptr(), lens.data_ptr(), at, B, wide, T, 0, pages.stride(0) if B > 1 else max(wide, 1))


def _rows(name, x, T, heads, dim):
    """fxpq_kv_rows"""
    st = x.stride()
    if x.shape != (T, heads, dim) or st[2] != 1 or not x.is_cuda:
        raise ValueError(f"{name}: rows [{T}, {heads}, {dim}] with contiguous heads are needed, got {tuple(x.shape)} with "
                         f"strides {x.stride()}")
    return _ROWS(x.data_ptr(), st[0], st[1])


def kv_append(cache, pages, lens, k, v, q=None, starts=None, cos=None, sin=None, interleaved=False):
    """Appends new keys and values k, v [T, heads, dim] to the cache; returns the rotated queries [T, q_heads, dim]
    (None without q).

    pages int32 [B, n]: each sequence's pages; lens int32 [B]: tokens of each sequence, the new ones included; starts
    int32 [B + 1]: where each sequence's new tokens begin among the T rows (None: T / B each).
    cos, sin float32 [positions, rot / 2]: keys and queries turn by their positions in their first rot values, pairs
    (i, i + rot / 2) or with interleaved (2 i, 2 i + 1).  k, v and q may be views with any token and head strides."""
    if k.dim() != 3:
        raise ValueError(f"kv_append: k must be [tokens, heads, dim], got {tuple(k.shape)}")
    dtype = k.dtype
    ft = _ftype("kv_append", dtype)
    if v.dtype != dtype or (q is not None and q.dtype != dtype):
        raise TypeError("kv_append: k, v and q must have one type")
    if k.requires_grad or v.requires_grad or (q is not None and q.requires_grad):
        _no_grad("kv_append", k, v, q)
    T = k.shape[0]
    batch = _batch("kv_append", pages, lens, starts, T)
    rk, rv = _rows("kv_append: k", k, T, cache.heads, cache.dim), _rows("kv_append: v", v, T, cache.heads, cache.dim)
    rq = out = None
    heads = n_pos = rot = to = c = s = 0
    if q is not None:
        heads = q.shape[1] if q.dim() == 3 else 0
        rq = _rows("kv_append: q", q, T, heads, cache.dim)
        out = _empty((T, heads, cache.dim), dtype=dtype, device=q.device)
        to = out.data_ptr()
    if (cos is None) != (sin is None):
        raise ValueError("kv_append: cos and sin go together")
    if cos is not None:
        _want("kv_append: cos", cos, _f32, 2)
        _want("kv_append: sin", sin, _f32, 2)
        n_pos, rot = cos.shape
        if sin.shape != (n_pos, rot):
            raise ValueError("kv_append: cos and sin must have one shape")
        rot, c, s = 2 * rot, cos.data_ptr(), sin.data_ptr()
    rc = L.lib().fxpq_kv_append(cache.packed, batch, ft, rk, rv, rq, heads, to, c, s, n_pos, rot, 1 if interleaved else 0, F._s(None))
    if rc:
        L.check("fxpq_kv_append", rc)
    return out


def kv_values(cache, pages, dtype=torch.bfloat16):
    """The values code * scale of the pages int32 [n]: keys and values [n, heads, page, dim]."""
    _want("kv_values: pages", pages, _i32, 1)
    n, ft = pages.shape[0], _ftype("kv_values", dtype)
    k = _empty((n, cache.heads, cache.page, cache.dim), dtype=dtype, device=pages.device)
    v = torch.empty_like(k)
    rc = L.lib().fxpq_kv_values(cache.packed, pages.data_ptr(), n, ft, k.data_ptr(), v.data_ptr(), F._s(None))
    if rc:
        L.check("fxpq_kv_values", rc)
    return k, v


_Q_TYPES = {torch.float16: L.FT_F16, torch.bfloat16: L.FT_BF16}


def kv_attention(cache, pages, lens, q, starts=None, scale=None, causal=True, return_lse=False):
    """Softmax attention of the queries q [T, q_heads, dim] (float16 or bfloat16, any token and head strides) of the
    last tokens of each sequence over the cache, which already holds those tokens; q_heads is a multiple of the
    cache's heads.  scale: 1 / sqrt(dim) by default.  Returns [T, q_heads, dim], and with return_lse the logarithms
    float32 [T, q_heads] of the sums of exponentials; rows that see no key are zeros and -inf."""
    dtype, dim = q.dtype, cache.dim
    ft = _ftype("kv_attention", dtype, _Q_TYPES)
    if q.requires_grad:
        _no_grad("kv_attention", q)
    if q.dim() != 3:
        raise ValueError(f"kv_attention: q must be [tokens, heads, dim], got {tuple(q.shape)}")
    T, heads, _ = q.shape
    if heads == 0 or heads % cache.heads:
        raise ValueError(f"kv_attention: {heads} query heads are no multiple of {cache.heads}")
    if pages.dim() == 2 and pages.stride(0) < pages.shape[1]:  # (sequences may share a row here; it stays referenced until the launch)
        pages = pages.contiguous()
    batch, rq = _batch("kv_attention", pages, lens, starts, T), _rows("kv_attention: q", q, T, heads, dim)
    out = _empty((T, heads, dim), dtype=dtype, device=q.device)
    lse = _empty((T, heads), dtype=_f32, device=q.device) if return_lse else None
    lib, packed = L.lib(), cache.packed
    need = lib.fxpq_kv_attention_workspace(packed, batch, heads)
    ws = _empty(need, dtype=_u8, device=q.device) if need else None
    rc = lib.fxpq_kv_attention(packed, batch, ft, rq, heads, dim ** -0.5 if scale is None else scale, 1 if causal else 0, out.data_ptr(),
                               lse.data_ptr() if return_lse else None, ws.data_ptr() if need else None, need, F._s(None))
    if rc:
        L.check("fxpq_kv_attention", rc)
    return (out, lse) if return_lse else out
