"""Gradients of 8-bit layers held to what 32 bits give: the rows dz * sw to 2^-23 of the row's largest value, sums exact."""
import numpy as np
import pytest
import torch

from test_gpu_layer import TYPES, Weights, check, host, ops, rows, status_is_clear  # noqa: F401

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
