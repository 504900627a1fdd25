"""Decoder layers of language models in 8 bits: rows quantized with a scale each, products of 8-bit rows,
and a paged cache of 8-bit keys and values with attention over it.

Torch tensors in, torch tensors out; every step runs in the library's kernels on the current stream, which
is also the stream that the results belong to.  Shapes and types are checked here, sizes, strides and
alignment in the library (``_lib.FxpqError``).  What a kernel finds wrong with the data (non-finite values,
page ids outside the cache, positions past the rotation tables) is latched and read by
``fxpq.fxpq_get_device_status``.

The operators are for inference and have no gradient: tensors that require one are refused while gradients are
recorded (RuntimeError).  Layers are the exception once `with_gradient` was called: then gradients reach their rows through
the frozen weights.
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
_LAYER = struct.Struct("PqPPqPPPqPqPPqiiiiiiif").pack      # fxpq_layer
_LAYER_GRAD = struct.Struct("PqPPPPPqPqqiiiiiiii").pack    # fxpq_layer_grad
_ACTS = {None: L.ACT_NONE, "relu": L.ACT_RELU, "silu": L.ACT_SILU, "gelu": L.ACT_GELU, "gelu_tanh": L.ACT_GELU_TANH}
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
    if w_scale.device != w.device or (bias is not None and bias.device != w.device):
        raise ValueError(f"{name}: weights, scales and biases must be on one device")
    if w_scale.shape[0] != w.shape[0] or (bias is not None and bias.shape[0] != w.shape[0]):
        raise ValueError(f"{name}: one scale and bias for each channel are needed")


def _pitch(t, K):  # (a single row, or rows of nothing, may have any stride)
    return t.stride(0) if t.shape[0] > 1 and K else (K + 15) // 16 * 16


def _whole_rows(w):
    """w int8 [N, K] with rows that begin at 16-byte boundaries."""
    N, K = w.shape
    if K % 16 == 0 and w.is_contiguous() and w.data_ptr() % 16 == 0:
        return w
    padded = torch.zeros((N, (K + 15) // 16 * 16), dtype=_i8, device=w.device)
    padded[:, :K] = w
    return padded[:, :K]


def _activation(name, activation):
    act = _ACTS.get(activation) if activation is None or isinstance(activation, str) else None
    if act is None:
        raise ValueError(f"{name}: activation {activation!r} is none of {', '.join(str(a) for a in _ACTS)}")
    return act


def _kept_row(N):
    """Bytes of a row of kept sums: in 32 bits, so that a slope is taken at the forward pass's own z."""
    return (N + 7) // 8 * 8 * 4


class _Layer8:
    """What layers with 8-bit weights share: w [N, K] codes, w_scale [N], bias [N] or None, and after `with_gradient` wt, the codes
    transposed."""

    wt = None
    gated = 0

    def with_gradient(self):
        """Lays out the transposed weights (one more byte for each) that a gradient is formed with, and returns the layer: from
        now on, rows (and residuals) that require a gradient get one.  The weights stay constants, and the rounding of rows to
        codes counts as the identity."""
        if self.wt is None:
            self.wt = _whole_rows(self.w.t())
        return self

    def _forward(self, name, x, dtype, norm, eps, act, residual, keep):
        """y, and with keep the sums and scales that `_gradient` reads (of an activation's layer, in one tensor)."""
        flat = x.dim() == 2
        rows = x if flat and x.is_cuda and x.is_contiguous() else _float_rows(name, x)
        M, K = rows.shape
        w, bias, dev = self.w, self.bias, x.device
        if dev.index != torch.cuda.current_device():
            with torch.cuda.device(dev):  # (its current stream)
                return self._forward(name, x, dtype, norm, eps, act, residual, keep)
        if w.device != dev or (norm is not None and norm.device != dev) or (residual is not None and residual.device != dev):
            raise ValueError(f"{name}: rows, weights, norm and residual must be on one device, rows are on {dev}, weights on {w.device}")
        N, inputs = w.shape
        if K != inputs:
            raise ValueError(f"{name}: rows of {inputs} values are needed, got {tuple(x.shape)}")
        wide = N // 2 if self.gated else N
        xt, yt = _FT.get(x.dtype), _FT.get(dtype)
        if xt is None or yt is None:
            _ftype(name, x.dtype if xt is None else dtype)
        nrm = res = res_stride = pre_at = sx_at = 0
        if norm is not None:
            if norm.dtype != _f32 or norm.dim() != 1 or norm.shape[0] != K or not norm.is_cuda or not norm.is_contiguous():
                _want(name + ": norm", norm, _f32, 1)
                raise ValueError(f"{name}: one norm weight for each of {K} inputs is needed")
            nrm = norm.data_ptr()
            if not 0.0 <= eps <= 1.0:
                raise ValueError(f"{name}: eps is 0 to 1, got {eps}")
        if residual is not None:
            if residual.dtype != dtype or residual.shape != ((M, N) if flat else x.shape[:-1] + (N,)):
                raise ValueError(f"{name}: a residual {(*x.shape[:-1], N)} of {dtype} is needed, got {tuple(residual.shape)} of {residual.dtype}")
            r = _float_rows(name + ": residual", residual)
            res, res_stride = r.data_ptr(), r.stride(0)
        y = _empty((M, wide), dtype=dtype, device=dev)
        kept = None
        if keep and act:
            room = M * _kept_row(N)
            kept = _empty(room + 4 * M, dtype=_u8, device=dev)
            pre_at = kept.data_ptr()
            sx_at = pre_at + room
        desc = _LAYER(rows.data_ptr(), rows.stride(0), nrm, w.data_ptr(), _pitch(w, K), self.w_scale.data_ptr(), 0 if bias is None else bias.data_ptr(),
                      res, res_stride, y.data_ptr(), wide, pre_at, sx_at, M, N, K, xt, yt, act, self.gated, L.FT_F32, eps)
        lib = L.lib()
        need = lib.fxpq_layer_workspace(desc)
        ws = _empty(need, dtype=_u8, device=dev) if need else None
        rc = lib.fxpq_layer_forward(desc, ws.data_ptr() if need else None, need, F._s(None))
        if rc:
            L.check(name, rc)
        if not flat:
            y = y.view(*x.shape[:-1], wide)
        return (y, kept) if keep else y

    def _gradient(self, name, dy, dtype, act, kept):
        """dx [..., K] of `dtype` for dy [..., N or N / 2] and what `_forward` kept."""
        if dy.device.index != torch.cuda.current_device():
            with torch.cuda.device(dy.device):
                return self._gradient(name, dy, dtype, act, kept)
        flat = dy.dim() == 2
        rows = dy if flat and dy.is_contiguous() else _float_rows(name, dy)
        M, (N, K), wt, bias = rows.shape[0], self.w.shape, self.wt, self.bias
        dx = _empty((M, K), dtype=dtype, device=dy.device)
        xt, yt = _FT[dtype], _FT[dy.dtype]
        pre = 0 if kept is None else kept.data_ptr()
        desc = _LAYER_GRAD(rows.data_ptr(), rows.stride(0), pre, pre and pre + M * _kept_row(N), self.w_scale.data_ptr(),
                           0 if bias is None else bias.data_ptr(), wt.data_ptr(), _pitch(wt, N), dx.data_ptr(), K, M, N, K, yt, xt, act, self.gated,
                           L.FT_F32, 0)
        lib = L.lib()
        need = lib.fxpq_layer_gradient_workspace(desc)
        ws = _empty(need, dtype=_u8, device=dy.device)
        rc = lib.fxpq_layer_gradient(desc, ws.data_ptr(), need, F._s(None))
        if rc:
            L.check(name, rc)
        return dx if flat else dx.view(*dy.shape[:-1], K)

    def _call(self, name, x, dtype, norm, eps, act, residual):
        """The forward pass, recorded where rows or residual require a gradient."""
        if torch.is_grad_enabled() and (x.requires_grad or (residual is not None and residual.requires_grad)):
            if self.wt is None:
                _no_grad(name + " without with_gradient()", x, residual)
            if norm is not None:
                raise RuntimeError(f"{name}: norm has no gradient: apply it before the layer, or call it under torch.no_grad()")
            return _LayerStep.apply(x, residual, self, name, dtype, act)
        if norm is not None and norm.requires_grad:
            _no_grad(name + ": norm", norm)
        return self._forward(name, x, dtype, norm, eps, act, residual, False)


def _step_back(ctx, dy):
    layer, name, act, dtype = ctx.what
    wants = ctx.needs_input_grad
    return layer._gradient(name, dy, dtype, act, *ctx.saved_tensors) if wants[0] else None, dy if wants[1] else None, None, None, None, None


_step_back_once = torch.autograd.function.once_differentiable(_step_back)


class _LayerStep(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, layer, name, dtype, act):
        ctx.what = layer, name, act, x.dtype
        if not ctx.needs_input_grad[0]:
            return layer._forward(name, x, dtype, None, 0.0, act, residual, False)
        y, kept = layer._forward(name, x, dtype, None, 0.0, act, residual, True)
        ctx.save_for_backward(kept)
        return y

    @staticmethod
    def backward(ctx, dy):
        # (the wrapper that refuses second derivatives takes 10 us of a small layer's backward: only where a graph of it is asked for)
        return _step_back_once(ctx, dy) if torch.is_grad_enabled() else _step_back(ctx, dy)


class Linear8(_Layer8):
    """A layer with 8-bit weights w int8 [N, K], one scale for each output channel: rows that are not whole 16 bytes
    are padded once.  Its tensors are constants: what they require of a gradient is dropped."""

    def __init__(self, w, w_scale, bias=None):
        _want("Linear8: w", w, _i8, 2)
        self._set(_whole_rows(w), w_scale, bias)

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

    def __call__(self, x, out_dtype=None, norm=None, eps=1e-5, activation=None, residual=None):
        """x [..., K] in a float type -> [..., N] in out_dtype (x's own by default): `quantize_tokens` and `linear_i8`
        as one call, with what stands around them: norm, float32 [K], turns x into x / sqrt(mean(x^2) + eps) * norm before, and
        y = activation(z) + residual after, all in fp32 with one rounding.  activation: "relu", "silu", "gelu" (z times the normal
        distribution's integral), "gelu_tanh" (its tanh form); residual: [..., N] of out_dtype."""
        if norm is not None or activation is not None or residual is not None or (self.wt is not None and x.requires_grad):
            return self._call("Linear8", x, out_dtype or x.dtype, norm, eps, _activation("Linear8", activation), residual)
        if x.requires_grad:
            _no_grad("Linear8", x)
        rows = _float_rows("Linear8", x)
        if x.device != self.w.device:
            raise ValueError(f"Linear8: rows and weights must be on one device, rows are on {x.device}, weights on {self.w.device}")
        if x.device.index != torch.cuda.current_device():
            with torch.cuda.device(x.device):  # (its current stream)
                return self(x, out_dtype)
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


class GatedLinear8(_Layer8):
    """Two layers of the same rows whose results are multiplied, as one product: activation(gate(x)) * up(x).  gate and up are int8
    [N, K] with one scale for each output channel, and may have biases; their rows are laid out alternately, once.  activation:
    as in `Linear8`, one is needed.  Its tensors are constants: what they require of a gradient is dropped."""

    gated = 1

    def __init__(self, gate, gate_scale, up, up_scale, gate_bias=None, up_bias=None, activation="silu"):
        self.act = _activation("GatedLinear8", activation)
        if not self.act:
            raise ValueError("GatedLinear8: an activation is needed")
        for side, w, scale, bias in (("gate", gate, gate_scale, gate_bias), ("up", up, up_scale, up_bias)):
            if w.dim() != 2 or w.shape != gate.shape or w.device != gate.device:
                raise ValueError("GatedLinear8: gate and up must have one shape [N, K]")
            _check_layer(f"GatedLinear8: {side}", w, scale, bias, gate.shape[1])
        if (gate_bias is None) != (up_bias is None):
            raise ValueError("GatedLinear8: gate_bias and up_bias go together")
        self.N, self.K = gate.shape
        self.w = _whole_rows(torch.stack((gate, up), 1).flatten(0, 1))
        self.w_scale = torch.stack((gate_scale.detach(), up_scale.detach()), 1).flatten()
        self.bias = None if gate_bias is None else torch.stack((gate_bias.detach(), up_bias.detach()), 1).flatten()

    @classmethod
    def from_float(cls, gate, up, gate_bias=None, up_bias=None, activation="silu"):
        """Quantizes float weights [N, K]."""
        biases = [None if b is None else b.detach().float().contiguous() for b in (gate_bias, up_bias)]
        return cls(*quantize_tokens(gate.detach()), *quantize_tokens(up.detach()), *biases, activation)

    def __call__(self, x, out_dtype=None, norm=None, eps=1e-5):
        """x [..., K] in a float type -> [..., N] in out_dtype (x's own by default); norm and eps: as in `Linear8`."""
        return self._call("GatedLinear8", x, out_dtype or x.dtype, norm, eps, self.act, None)


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
