"""Gradients of 8-bit layers held to what 32 bits give: the rows dz * sw to 2^-23 of the row's largest value, sums exact, activations' slopes
of the forward pass's own z."""
import numpy as np
import pytest
import torch

from oracle import llm as O
from paper_2203_12091_gb300 import _lib as L
from paper_2203_12091_gb300 import fxpq as F
from test_gpu_layer import ACTS, TYPES, Weights, act_spread, argument, check, host, ops, rows, status_is_clear  # noqa: F401

pytestmark = pytest.mark.gpu


def check_rows(got, dz, dz_err, W, kind):
    """dx [M, K] against (dz sw) . w in 64 bits, dz [M, n] good to dz_err.  dz * sw rounds once or twice, then to two parts: integers of 12 bits,
    and what is left of them to 2^-12 of itself, at most half of 2^-22 of the row's largest.  Weights here are so small that the first
    part's sums are exact (below 2^24); the second's round in steps of 16, 2^-11 as large.  Joining and storing round once each."""
    w, sw = W.w.astype(np.float64), W.sw.astype(np.float64)
    assert 2 ** 11 * np.abs(w).sum(0).max() < 2 ** 24
    want, t = dz * sw @ w, np.abs(dz * sw) + dz_err * sw
    top = t.max(1, keepdims=True)
    value = dz_err * sw + t * 2.0 ** -22 + np.minimum(top * 2.0 ** -23, t * 2.0 ** -12 + top * 2.0 ** -46)
    low = (len(w) / 16 + 2) * 2.0 ** -23 * top * 2.0 ** -11
    spread = (value + low) @ np.abs(w)
    check(got, want, spread + np.abs(want) * 2.0 ** -24, kind)


def small(rng, N, K, bias, sides=1):
    W = Weights(rng, N, K, bias, sides)
    W.w = rng.integers(-7, 8, W.w.shape, dtype=np.int8)
    W.sw *= np.float32(18)
    return W


@pytest.mark.parametrize("M,N,K", [(1, 512, 300), (40, 512, 300), (60, 1000, 128), (129, 100, 100), (300, 512, 256), (700, 1001, 513), (1500, 640, 1024)])
@pytest.mark.parametrize("x", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("out", ["bf16", "f32"])
def test_rows_of_the_gradient_hold_23_bits(ops, M, N, K, x, out):
    rng = np.random.default_rng(M + N + K)
    W = small(rng, N, K, False)
    layer = W.layer(ops).with_gradient()
    leaf = rows(rng, M, K, x).requires_grad_()
    dy = rows(rng, M, N, out)
    dx = torch.autograd.grad(layer(leaf, TYPES[out]), leaf, dy)[0]
    check_rows(dx, host(dy), 0.0 * host(dy), W, x)


@pytest.mark.parametrize("M,N,K", [(40, 512, 300), (300, 512, 256)])
@pytest.mark.parametrize("x", ["bf16", "f32"])
def test_small_values_beside_a_large_one(ops, M, N, K, x):
    """A channel 2^20 times the others whose weights are zero: what the others give is still good to 2^-12 of each."""
    rng = np.random.default_rng(M)
    W = small(rng, N, K, False)
    W.w[5] = 0
    layer = W.layer(ops).with_gradient()
    leaf = rows(rng, M, K, x).requires_grad_()
    dy = rows(rng, M, N, "f32")
    dy[:, 5] = 2.0 ** 20
    dx = torch.autograd.grad(layer(leaf, torch.float32), leaf, dy)[0]
    check_rows(dx, host(dy), 0.0 * host(dy), W, x)


@pytest.mark.parametrize("M,N,K", [(3, 512, 300), (40, 512, 300), (300, 512, 256), (700, 300, 512)])
@pytest.mark.parametrize("act", ACTS[2:])
@pytest.mark.parametrize("is_gated", [False, True])
@pytest.mark.parametrize("kind", ["bf16", "f16"])
def test_slopes_are_those_of_the_forward_pass(ops, M, N, K, act, is_gated, kind):
    """z as the forward pass had it, not of rounded sums: what is left is the arithmetic of the slopes."""
    rng = np.random.default_rng(M + N + K)
    N = N // 2 if is_gated else N
    W = small(rng, N, K, True, 2 if is_gated else 1)
    layer = (W.gated(ops, act) if is_gated else W.layer(ops)).with_gradient()
    leaf = rows(rng, M, K, kind).requires_grad_()
    y = layer(leaf) if is_gated else layer(leaf, activation=act)
    dy = rows(rng, M, N, kind)
    dx = torch.autograd.grad(y, leaf, dy)[0]
    z, e, _ = W.sums(leaf)
    d = host(dy)
    # slopes bend by less than 0.8 a unit of z; their exponentials and quotients are good to some steps of 2^-22 of what they are made of
    slope_err = 0.8 * e + np.minimum((16 + 8 * argument(z, act)) * 2.0 ** -22, 1) * (1 + np.abs(z))
    if is_gated:
        g, u, eg, eu = z[:, ::2], z[:, 1::2], e[:, ::2], e[:, 1::2]
        f, slope = O.activation(g, act)
        err = np.empty_like(z)
        err[:, ::2] = np.abs(d) * (np.abs(slope) * eu + (np.abs(u) + eu) * slope_err[:, ::2])
        err[:, 1::2] = np.abs(d) * (act_spread(g, eg, act) + np.abs(f) * 2.0 ** -23)
    else:
        err = np.abs(d) * slope_err
    check_rows(dx, O.layer_slopes(z, d, act, is_gated), err, W, kind)


@pytest.mark.parametrize("M", [3, 40, 300, 1300])
@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("is_gated", [False, True])
def test_relu_passes_a_gradient_where_its_own_output_is_positive(ops, M, out, is_gated):
    """Biases that take back one row's sums but for their rounding, so that z lies next to 0 on either side there."""
    rng = np.random.default_rng(M)
    N, K = 512, 2048
    W = small(rng, N // 2 if is_gated else N, K, True, 2 if is_gated else 1)
    leaf = rows(rng, M, K, "bf16").requires_grad_()
    codes, sx = O.quantize_tokens(leaf.detach().float().cpu().numpy())
    at = M // 2
    near = -(O.layer_sums(codes[at:at + 1], W.w)[0][0].astype(np.float32) * np.float32(sx[at]) * W.sw)
    if is_gated:
        W.b[::2], W.b[1::2] = near[::2], 1
    else:
        W.b[:] = near
    layer = (W.gated(ops, "relu") if is_gated else W.layer(ops)).with_gradient()
    y = layer(leaf, TYPES[out]) if is_gated else layer(leaf, TYPES[out], activation="relu")
    dy = rows(rng, M, y.shape[1], out)
    dx = torch.autograd.grad(y, leaf, dy)[0]
    z, e, _ = W.sums(leaf)
    d = host(dy)
    if is_gated:
        g, u = z[:, ::2], z[:, 1::2]
        on = (host(y) * u > 0) | (g > 1)  # (y = relu(g) u, and no u is 0 here)
        assert np.all(u != 0)
        dz, err = np.empty_like(z), np.empty_like(z)
        dz[:, ::2], dz[:, 1::2] = d * u * on, d * np.maximum(g, 0)
        err[:, ::2], err[:, 1::2] = np.abs(d) * e[:, 1::2], np.abs(d) * e[:, ::2]
    else:
        on = host(y) > 0
        dz, err = d * on, 0 * d
    assert 0.1 < on[at].mean() < 0.9 and np.all(np.abs(z[at, :: 2 if is_gated else 1]) < 1e-5)
    check_rows(dx, dz, err, W, "bf16")


@pytest.mark.parametrize("M", [3, 40, 300])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("is_gated", [False, True])
def test_nan_in_a_bias_reaches_the_gradient(ops, M, act, is_gated):
    """z is NaN in one channel: so is every slope there, and with it every row's gradient, dy of 0 or not."""
    if is_gated and act is None:
        return
    rng = np.random.default_rng(M)
    for bad in (6, 7):  # (of a gate, and of a value)
        W = small(rng, 64, 200, True, 2)
        W.b[bad] = np.nan
        layer = (W.gated(ops, act) if is_gated else W.layer(ops)).with_gradient()
        leaf = rows(rng, M, 200, "bf16").requires_grad_()
        y = layer(leaf) if is_gated else layer(leaf, activation=act)
        dy = rows(rng, M, y.shape[1], "bf16")
        dy[0] = 0
        dx = torch.autograd.grad(y, leaf, dy)[0]
        if act is None:  # (dz = dy: no z in it)
            assert bool(dx.isfinite().all())
        else:
            assert F.fxpq_get_device_status() == L.ERR_NONFINITE
            assert bool(dx.isnan().all())


@pytest.mark.parametrize("act", [L.ACT_SILU, L.ACT_GELU, L.ACT_GELU_TANH])
@pytest.mark.parametrize("is_gated", [0, 1])
@pytest.mark.parametrize("M", [3, 300])
def test_kept_sums_of_rows_next_to_the_largest_float(ops, M, act, is_gated):
    """A row's scale times the power of two of sums kept in fp16 can pass fp32 where z does not: sums of few bits, exact in either form,
    give the same gradients in both."""
    rng = np.random.default_rng(M)
    N, K = 64, 4096
    W = Weights(rng, N, K, True)
    W.w = rng.integers(-7, 8, W.w.shape, dtype=np.int8)
    W.sw[:] = 2.0 ** -126
    layer = W.layer(ops).with_gradient()
    x = torch.zeros(M, K, dtype=torch.bfloat16, device="cuda")
    x[:, 0] = 2.0 ** 125  # (a scale of 2^118.01; sums of 127 times 0 to 7, below 2^9.8; the power of two is 2^10)
    wide = N // 2 if is_gated else N
    dy, got = rows(rng, M, wide, "f32"), []
    for pre_type, kept in ((L.FT_F16, torch.float16), (L.FT_F32, torch.float32)):
        y, pre, sx = torch.empty(M, wide, device="cuda"), torch.zeros(M, N, dtype=kept, device="cuda"), torch.empty(M, device="cuda")
        d = L.LayerDesc(x.data_ptr(), K, None, layer.w.data_ptr(), K, layer.w_scale.data_ptr(), layer.bias.data_ptr(), None, 0, y.data_ptr(), wide,
                        pre.data_ptr(), sx.data_ptr(), M, N, K, L.FT_BF16, L.FT_F32, act, is_gated, pre_type, 0.0)
        F.fxpq_layer_forward(d, torch.empty(F.fxpq_layer_workspace(d), dtype=torch.uint8, device="cuda"))
        assert bool(y.isfinite().all())
        dx = torch.empty(M, K, device="cuda")
        g = L.LayerGradDesc(dy.data_ptr(), wide, pre.data_ptr(), sx.data_ptr(), layer.w_scale.data_ptr(), layer.bias.data_ptr(),
                            layer.wt.data_ptr(), layer.wt.stride(0), dx.data_ptr(), K, M, N, K, L.FT_F32, L.FT_F32, act, is_gated, pre_type, 0)
        F.fxpq_layer_gradient(g, torch.empty(F.fxpq_layer_gradient_workspace(g), dtype=torch.uint8, device="cuda"))
        got.append(dx)
    assert bool(got[1].isfinite().all()) and bool((got[1] != 0).any()) and torch.equal(*got)


@pytest.mark.parametrize("M,N,K,x", [(239, 1462, 158, "bf16"), (464, 180, 2700, "f16"), (1638, 153, 1064, "bf16"), (712, 1055, 3173, "bf16"), (224, 6872, 2541, "f16"),
                                     (599, 1128, 4017, "f32"), (819, 3243, 1427, "f32"), (1605, 3787, 691, "bf16"), (3000, 4000, 1000, "bf16"),
                                     (1659, 204, 646, "f32"), (80, 8000, 6000, "f32"), (130, 8192, 4096, "bf16")])
def test_both_parts_in_the_tiles_of_pairs(ops, M, N, K, x):
    """Tiles of either width, reductions split and whole, rows and channels past the last tile's, outputs in pairs and one by one: into rows
    with a stride of their own, of which nothing else is written."""
    rng = np.random.default_rng(M)
    W = Weights(rng, N, K, False)
    W.w = rng.integers(-1, 2, W.w.shape, dtype=np.int8)
    W.sw *= np.float32(100)
    layer = W.layer(ops).with_gradient()
    dy = rows(rng, M, N, "f32")
    dy[M // 2] = 0
    out = torch.full((M + 3, K + 6), 7.0, dtype=TYPES[x], device="cuda")
    g = L.LayerGradDesc(dy.data_ptr(), N, None, None, layer.w_scale.data_ptr(), None, layer.wt.data_ptr(), layer.wt.stride(0), out.data_ptr(), K + 6, M, N, K,
                        L.FT_F32, {"f32": L.FT_F32, "f16": L.FT_F16, "bf16": L.FT_BF16}[x], L.ACT_NONE, 0, L.FT_F32, 0)
    F.fxpq_layer_gradient(g, torch.empty(F.fxpq_layer_gradient_workspace(g), dtype=torch.uint8, device="cuda"))
    check_rows(out[:M, :K], host(dy), 0.0 * host(dy), W, x)
    assert bool((out[M:] == 7).all()) and bool((out[:, K:] == 7).all())
    leaf = rows(rng, M, K, x).requires_grad_()
    assert torch.equal(torch.autograd.grad(layer(leaf, torch.float32), leaf, dy)[0], out[:M, :K])
