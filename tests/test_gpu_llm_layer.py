"""`Linear8` against the 64-bit oracle: tokens that its own quantizer writes as fp16 codes, at every tile width, cluster size and
tail of the product that takes them."""
import numpy as np
import pytest
import torch

from oracle import llm as O
from paper_2203_12091_gb300 import _lib as L
from paper_2203_12091_gb300 import fxpq as F

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
UNIT = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}  # relative rounding error of a stored result


@pytest.fixture(scope="module")
def ops():
    import __graft_entry__ as g
    g.build()
    from paper_2203_12091_gb300 import llm
    assert F.fxpq_get_device_status() == L.OK
    return llm


@pytest.fixture(autouse=True)
def status_is_clear():
    yield
    assert F.fxpq_get_device_status() == L.OK


def cuda(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(dtype)


def check_layer(ops, x, N, out, bias, rng):
    """x: rows on the GPU.  Codes are the oracle's bit for bit, so what the layer may add is the product's: each step of 16
    exact products rounds (or cuts) its sum to 24 bits where that can pass 2^24, three fp32 roundings, the output's own."""
    K = x.shape[-1]
    w = rng.integers(-127, 128, (N, K), dtype=np.int8)
    sw = np.exp(rng.normal(size=N)).astype(np.float32) * 0.01
    b = rng.normal(size=N).astype(np.float32) if bias else None
    y = ops.Linear8(cuda(w), cuda(sw), None if b is None else cuda(b))(x, TYPES[out])
    codes, sx = O.quantize_tokens(x.float().cpu().numpy())
    # products of codes in float64 are exact (sums stay far below 2^53)
    c64, w64 = codes.astype(np.float64), w.astype(np.float64)
    s = sx.astype(np.float64)[:, None] * sw.astype(np.float64)
    add = 0.0 if b is None else b.astype(np.float64)
    want, size = (c64 @ w64.T) * s + add, np.abs(c64) @ np.abs(w64).T
    steps = np.where(size < 2 ** 24, 0.0, (K / 16 + 1) * 2.0 ** -23)
    bound = (size * s + np.abs(add)) * (steps + 2.0 ** -22) + np.abs(want) * UNIT[out] + 2.0 ** -24 * (out == "f16")
    got = y.double().cpu().numpy()
    over = (out == "f16") & (np.abs(want) + bound >= 65520)  # (may round past float16's largest value)
    err = np.where(over & np.isinf(got), np.where(np.sign(got) == np.sign(want), 0.0, np.inf), np.abs(got - want))
    assert y.shape == (x.shape[0], N) and y.dtype == TYPES[out]
    assert np.all(err <= bound), (np.max(err / np.maximum(bound, 1e-300)), np.argwhere(err > bound)[:5])


def rows(rng, M, K, dtype):
    return cuda(rng.normal(size=(M, K)) * np.exp(rng.normal(size=(M, 1))), TYPES[dtype])


@pytest.mark.parametrize("M", [1, 2, 16, 17, 33, 64, 65, 129, 251, 256, 257])
@pytest.mark.parametrize("N,K", [(1, 1), (8, 16), (130, 100), (257, 1023), (1001, 520), (512, 2048)])
def test_layer_sizes(ops, M, N, K):
    rng = np.random.default_rng(M * 11 + N + K)
    kinds = ["bf16", "f16", "f32"]
    check_layer(ops, rows(rng, M, K, kinds[(M + K) % 3]), N, kinds[(M + N) % 3], (M + K) % 2, rng)


@pytest.mark.parametrize("M,N,K,x,out", [(1, 4096, 4096, "bf16", "bf16"), (64, 1000, 25088, "f16", "f16"), (5, 515, 25088, "f32", "f32"),
                                         (251, 1001, 4090, "bf16", "f32"), (129, 333, 8200, "f16", "f16"), (65, 129, 8191, "bf16", "bf16"),
                                         (40, 152 * 128 + 1, 64, "bf16", "bf16"), (200, 127, 33000, "f16", "f32"), (300, 1111, 4090, "bf16", "f16"),
                                         (513, 640, 8192, "f16", "f32"), (1000, 130, 12345, "bf16", "bf16")])
def test_layer_long_reductions(ops, M, N, K, x, out):
    rng = np.random.default_rng(M + N + K)
    check_layer(ops, rows(rng, M, K, x), N, out, True, rng)


@pytest.mark.parametrize("M", [3, 70, 200])
def test_layer_sums_past_24_bits(ops, M):
    rng = np.random.default_rng(1)
    check_layer(ops, torch.ones(M, 8208, device="cuda") * torch.linspace(0.5, 2, M, device="cuda")[:, None], 136, "f32", False, rng)


@pytest.mark.parametrize("M", [7, 251])
def test_layer_on_views_and_non_finite_values(ops, M):
    rng = np.random.default_rng(M)
    big = rows(rng, 2 * M, 4099, "f16")
    for view in (big[:M, 1:4092], big[::2, 5:1000], big.t()[:M]):
        check_layer(ops, view, 259, "bf16", True, rng)
    x = rows(rng, M, 2000, "bf16")
    x[M // 2, 1999], x[0, 0], x[1] = float("inf"), float("nan"), 0
    check_layer(ops, x, 130, "f32", True, rng)
    assert F.fxpq_get_device_status() == L.ERR_NONFINITE
