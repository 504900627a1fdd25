"""8-bit layers with norm, activation, gate, residual and gradient on the GPU against the 64-bit oracle.

Codes are the oracle's bit for bit, and the sums of their products are exact below 2^24.  What is left is held to bounds from the
arithmetic: `spread` below says how far a result may lie from the oracle's."""
import time

import numpy as np
import pytest
import torch

from oracle import llm as O
from paper_2203_12091_gb300 import _lib as L
from paper_2203_12091_gb300 import fxpq as F

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
UNIT = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}  # half a step of a stored result, relative
FLOOR = {"f32": 2.0 ** -149, "f16": 2.0 ** -25, "bf16": 2.0 ** -134}  # half a step of its smallest values
ACTS = [None, "relu", "silu", "gelu", "gelu_tanh"]
EPS = 1e-5


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


def host(t):
    return t.detach().double().cpu().numpy()


def rows(rng, M, K, dtype):
    return cuda(rng.normal(size=(M, K)) * np.exp(0.5 * rng.normal(size=(M, 1))), TYPES[dtype])


class Weights:
    """Codes, scales and biases of a layer (of gate and value, in turn) such that sums are of order 1."""

    def __init__(self, rng, N, K, bias, sides=1):
        n = N * sides
        self.w = rng.integers(-127, 128, (n, K), dtype=np.int8)
        self.sw = (np.exp(0.3 * rng.normal(size=n)) / (73 * np.sqrt(K))).astype(np.float32)
        self.b = rng.normal(size=n).astype(np.float32) if bias else None

    def layer(self, ops):
        return ops.Linear8(cuda(self.w), cuda(self.sw), None if self.b is None else cuda(self.b))

    def gated(self, ops, act):
        part = [[None if t is None else cuda(t[i::2]) for t in (self.w, self.sw, self.b)] for i in (0, 1)]
        return ops.GatedLinear8(*part[0][:2], *part[1][:2], part[0][2], part[1][2], act)

    def sums(self, x, norm=None):
        """z in 64 bits and how far the GPU's may lie from it."""
        f = x.detach().float().cpu().numpy()
        K = f.shape[1]
        if norm is None:
            codes, sx = O.quantize_tokens(f)
            scale_err = 0.0
        else:
            # the mean of squares: each of K + 8 additions rounds, then a division, the eps, a square root and two products
            codes, sx = O.norm_codes(f, norm, EPS)
            scale_err = (K + 8) / 2 * 2.0 ** -24 + 6 * 2.0 ** -24
        acc, size = O.layer_sums(codes, self.w)
        s = sx.astype(np.float64)[:, None] * self.sw.astype(np.float64)
        b = 0.0 if self.b is None else self.b.astype(np.float64)
        # steps of 16 exact products round (or cut) a sum that can pass 2^24; scale, scale and bias round once each
        steps = np.where(size < 2 ** 24, 0.0, (K / 16 + 1) * 2.0 ** -23)
        z = acc * s + b
        return z, size * s * steps + np.abs(acc * s) * (2.0 ** -23 + scale_err) + np.abs(z) * 2.0 ** -24, np.abs(acc * s)


def argument(z, act):
    """The largest argument of an exponential in act (or its like for erfc)."""
    return np.abs(z) if act == "silu" else 1.6 * np.abs(z + 0.0447 * z ** 3) if act == "gelu_tanh" else z * z


def act_spread(z, dz, act):
    """How far act of z off by dz lies from act(z): slopes are below 1.13; exponentials are good to (2 + 1.2 |v|) steps of 2^-23 and
    their argument v to four, quotients and erfc to six.  Past 88 the exponential leaves fp32: what is left is below 1e-35."""
    f, v = np.abs(O.activation(z, act)[0]), argument(z, act)
    return 1.13 * dz + (0 if act in (None, "relu") else f * np.minimum((8 + 6 * v) * 2.0 ** -23, 1) + 1e-35)


def check(got, want, spread, out):
    got = host(got)
    bound = spread + np.abs(want) * UNIT[out] + FLOOR[out]
    bound = bound + spread * UNIT[out]
    assert got.shape == want.shape
    err = np.abs(got - want)
    assert np.all(err <= bound), (np.max(err / bound), np.argwhere(~(err <= bound))[:5])


def check_layer(ops, rng, M, N, K, x, out, act, bias, res, norm, rows_in=None):
    x = rows(rng, M, K, x) if rows_in is None else rows_in
    W = Weights(rng, N, K, bias)
    wt = np.exp(0.2 * rng.normal(size=K)).astype(np.float32) if norm else None
    r = rows(rng, M, N, out) if res else None
    y = W.layer(ops)(x, TYPES[out], norm=None if wt is None else cuda(wt), eps=EPS, activation=act, residual=r)
    z, dz, _ = W.sums(x, wt)
    want = O.layer(z, act, None if r is None else host(r))
    spread = act_spread(z, dz, act) + (0 if r is None else np.abs(want) * 2.0 ** -24)
    assert y.dtype == TYPES[out]
    check(y, want, spread, out)


def check_gated(ops, rng, M, N, K, x, out, act, bias, norm, rows_in=None):
    x = rows(rng, M, K, x) if rows_in is None else rows_in
    W = Weights(rng, N, K, bias, 2)
    wt = np.exp(0.2 * rng.normal(size=K)).astype(np.float32) if norm else None
    y = W.gated(ops, act)(x, TYPES[out], norm=None if wt is None else cuda(wt), eps=EPS)
    z, dz, _ = W.sums(x, wt)
    g, u, dg, du = z[:, ::2], z[:, 1::2], dz[:, ::2], dz[:, 1::2]
    f, df = O.activation(g, act)[0], act_spread(g, dg, act)
    spread = np.abs(f) * du + np.abs(u) * df + du * df + np.abs(f * u) * 2.0 ** -24
    assert y.shape == (M, N) and y.dtype == TYPES[out]
    check(y, O.gated(z, act), spread, out)


def pick(*a):
    """x, out, act and three flags that vary with the sizes."""
    i = sum(a)
    kinds = ["bf16", "f16", "f32"]
    return kinds[i % 3], kinds[(i // 3) % 3], ACTS[i % 5], i % 2, (i // 2) % 2, (i // 4) % 2


SIZES = [(1, 1), (8, 16), (130, 100), (257, 1023), (1001, 520), (512, 2048), (128, 128)]


@pytest.mark.parametrize("M", [1, 2, 16, 17, 33, 64, 65, 129, 251, 256, 257, 600])
@pytest.mark.parametrize("N,K", SIZES)
def test_layer_sizes(ops, M, N, K):
    rng = np.random.default_rng(M * 11 + N + K)
    x, out, act, bias, res, norm = pick(M, N, K)
    check_layer(ops, rng, M, N, K, x, out, act, bias, res, norm)


@pytest.mark.parametrize("M", [1, 2, 16, 17, 33, 64, 65, 129, 251, 256, 257, 600])
@pytest.mark.parametrize("N,K", SIZES)
def test_gated_sizes(ops, M, N, K):
    rng = np.random.default_rng(M * 13 + N + K)
    x, out, act, bias, _, norm = pick(M, N, K)
    check_gated(ops, rng, M, N, K, x, out, act or "silu", bias, norm)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("out", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("M", [5, 300])
def test_every_activation(ops, M, act, out):
    rng = np.random.default_rng(M)
    check_layer(ops, rng, M, 200, 256, "bf16", out, act, True, True, True)
    check_layer(ops, rng, M, 200, 256, "f16", out, act, False, True, False)
    if act:
        check_gated(ops, rng, M, 150, 256, "bf16", out, act, True, True)
        check_gated(ops, rng, M, 151, 256, "f16", out, act, False, False)


@pytest.mark.parametrize("M,N,K,x,out", [(1, 4096, 4096, "bf16", "bf16"), (64, 1000, 25088, "f16", "f16"), (251, 1001, 4090, "bf16", "f32"),
                                         (40, 152 * 128 + 1, 64, "bf16", "bf16"), (300, 1111, 4090, "bf16", "f16"), (2000, 1366, 777, "f16", "bf16"),
                                         (513, 640, 8192, "f16", "f32"), (1000, 130, 12345, "bf16", "bf16"), (3000, 2048, 512, "bf16", "bf16")])
def test_long_reductions_and_wide_layers(ops, M, N, K, x, out):
    rng = np.random.default_rng(M + N + K)
    check_layer(ops, rng, M, N, K, x, out, "silu", True, True, True)
    check_gated(ops, rng, M, N // 2 + 1, K, x, out, "silu", True, True)


def test_more_rows_than_a_grid_dimension(ops):
    rng = np.random.default_rng(0)
    check_layer(ops, rng, 70001, 20, 32, "bf16", "bf16", "relu", True, True, True)
    check_gated(ops, rng, 66000, 130, 136, "bf16", "bf16", "silu", False, False)


@pytest.mark.parametrize("M", [7, 300])
def test_views_and_shapes(ops, M):
    rng = np.random.default_rng(M)
    big = rows(rng, 2 * M, 1099, "f16")
    for view in (big[:M, 1:1092], big[::2, 5:1000], big.t()[:M], big[:1, :96].expand(M, 96)):
        check_layer(ops, rng, view.shape[0], 259, view.shape[1], None, "bf16", "gelu", True, True, True, view)
        check_gated(ops, rng, view.shape[0], 131, view.shape[1], None, "bf16", "silu", True, True, view)
    W = Weights(rng, 70, 96, True)
    layer, x = W.layer(ops), rows(rng, 6 * M, 96, "bf16")
    wide = rows(rng, 6 * M, 145, "bf16")
    flat = layer(x, activation="silu", residual=wide[:, 3:73].contiguous())
    assert torch.equal(layer(x, activation="silu", residual=wide[:, 3:73]), flat)  # a residual with rows of its own stride
    assert torch.equal(layer(x.view(M, 2, 3, 96), activation="silu", residual=wide[:, 3:73].reshape(M, 2, 3, 70)), flat.view(M, 2, 3, 70))
    gate = W.gated(ops, "gelu")
    assert torch.equal(gate(x.view(M, 2, 3, 96)), gate(x).view(M, 2, 3, 35))
    assert layer(x[:0], activation="relu").shape == (0, 70) and gate(x[:0]).shape == (0, 35)
    assert torch.equal(layer(x[5], activation="relu"), layer(x[5:6], activation="relu")[0])


@pytest.mark.parametrize("M", [3, 300])
def test_plain_calls_and_calls_with_nothing_to_do_agree(ops, M):
    """A residual of zeros goes another way than a layer alone; sums below 2^24 are exact on both."""
    rng = np.random.default_rng(M)
    layer, x = Weights(rng, 333, 512, True).layer(ops), rows(rng, M, 512, "bf16")
    assert torch.equal(layer(x), layer(x, residual=torch.zeros(M, 333, dtype=torch.bfloat16, device="cuda")))


@pytest.mark.parametrize("power", [-120, -70, -40, 0, 40, 70, 120])
def test_norm_of_huge_and_tiny_rows(ops, power):
    """Rows times a power of two have the same norm (eps 0), so the same results."""
    rng = np.random.default_rng(5)
    x = np.clip(np.abs(rng.normal(size=(9, 300))), 0.1, 3) * rng.choice([-1, 1], (9, 300))
    layer, wt = Weights(rng, 64, 300, True).layer(ops), torch.ones(300, device="cuda")
    x = cuda(x, torch.bfloat16)
    want = layer(x, torch.float32, norm=wt, eps=0.0)
    got = layer((x.double() * 2.0 ** power).bfloat16(), torch.float32, norm=wt, eps=0.0)
    if power < -100:  # (a row below 2^-100 is zero)
        assert torch.equal(got, layer(torch.zeros_like(x), torch.float32))
    else:
        assert torch.allclose(got, want, rtol=0, atol=2.0 ** -20 * want.abs().max().item())


@pytest.mark.parametrize("M", [7, 300])
def test_rows_of_zeros_and_non_finite_values(ops, M):
    rng = np.random.default_rng(M)
    x = rows(rng, M, 500, "bf16")
    x[1] = 0
    check_layer(ops, rng, M, 130, 500, None, "f32", "silu", True, True, True, x)
    assert F.fxpq_get_device_status() == L.OK
    x[M // 2, 499], x[0, 0], x[2, 7] = float("inf"), float("nan"), -float("inf")
    check_layer(ops, rng, M, 130, 500, None, "f32", "silu", True, True, True, x)
    assert F.fxpq_get_device_status() == L.ERR_NONFINITE
    check_gated(ops, rng, M, 130, 500, None, "f32", "silu", True, False, x)
    assert F.fxpq_get_device_status() == L.ERR_NONFINITE


@pytest.mark.parametrize("M", [4, 280])
def test_far_arguments(ops, M):
    """z up to some thousands either way: activations at their limits, no NaN."""
    rng = np.random.default_rng(M)
    W = Weights(rng, 150, 256, False, 2)
    W.sw *= np.float32(1000)
    x = rows(rng, M, 256, "bf16")
    z = W.sums(x)[0]
    assert z.min() < -300 and z.max() > 300
    for act in ACTS[1:]:
        y = host(W.gated(ops, act)(x, torch.float32))
        want = O.gated(z, act)
        assert np.all(np.isfinite(y)) and np.all(np.abs(y - want) <= np.abs(want) * 2.0 ** -9 + 1e-30)
        y = host(W.layer(ops)(x, torch.float32, activation=act))
        assert np.all(np.isfinite(y))


# ------------------------------------------------------------------------------ gradients
def check_gradient(ops, rng, M, N, K, x, out, act, bias, is_gated, res=False, dy=None):
    """dx against the oracle's.  Kept sums are rounded to fp16 (exact in fp32), which moves z and with it act' (whose slope is below
    0.8) and act; dz * sw is rounded to fp16 or to 2^-22 of the row's largest; products are exact, their sums round."""
    x = rows(rng, M, K, x).requires_grad_()
    W = Weights(rng, N, K, bias, 2 if is_gated else 1)
    layer = (W.gated(ops, act) if is_gated else W.layer(ops)).with_gradient()
    wide32 = x.dtype == torch.float32 or out == "f32"
    r = rows(rng, M, N, out).requires_grad_() if res else None
    y = layer(x, TYPES[out]) if is_gated else layer(x, TYPES[out], activation=act, residual=r)
    dy = (rows(rng, M, N, out) * 0.01 if dy is None else dy).to(TYPES[out])
    if M > 2:
        dy[1] = 0
    grads = torch.autograd.grad(y, [x, r] if res else [x], dy)
    z, dz, mag = W.sums(x)
    e = dz + mag * (0 if wide32 else 2.0 ** -11)
    d = host(dy)
    want = O.layer_slopes(z, d, act, is_gated)
    v = 0 if act in (None, "relu") else np.minimum((16 + 8 * argument(z, act)) * 2.0 ** -22, 1) * (1 + np.abs(z))
    bend = 0.0 if act in (None, "relu") else 0.8
    slope_err = bend * e + v
    if is_gated:
        g, u, eg, eu = z[:, ::2], z[:, 1::2], e[:, ::2], e[:, 1::2]
        f, slope = O.activation(g, act)
        spread = np.empty_like(z)
        spread[:, ::2] = np.abs(d) * (np.abs(slope) * eu + (np.abs(u) + eu) * slope_err[:, ::2])
        spread[:, 1::2] = np.abs(d) * (act_spread(g, eg, act) + np.abs(f) * 2.0 ** -23)
    else:
        spread = np.abs(d) * slope_err
    sw, w = W.sw.astype(np.float64), np.abs(W.w.astype(np.float64))
    spread = (spread + np.abs(want) * 2.0 ** -22) * sw
    t = np.abs(want * sw) + spread
    top = t.max(1, keepdims=True)
    parts = x.dtype == torch.float32
    spread = spread + (top * 2.0 ** -22 if parts else t * 2.0 ** -11 + top * 2.0 ** -39)
    steps = (W.w.shape[0] / 16 + 2) * 2.0 ** -23
    kind = {v: k for k, v in TYPES.items()}[x.dtype]
    check(grads[0], (want * sw) @ W.w.astype(np.float64), spread @ w + (t @ w) * steps, kind)
    assert grads[0].dtype == x.dtype
    if res:
        assert torch.equal(grads[1], dy)


@pytest.mark.parametrize("M", [1, 2, 17, 64, 129, 257, 600])
@pytest.mark.parametrize("N,K", [(1, 1), (8, 16), (131, 100), (257, 515), (512, 1024), (128, 128)])
def test_gradient_sizes(ops, M, N, K):
    rng = np.random.default_rng(M * 5 + N + K)
    x, out, act, bias, res, _ = pick(M, N, K)
    act = "silu" if act == "relu" else act
    check_gradient(ops, rng, M, N, K, x, out, act, bias, False, res)
    check_gradient(ops, rng, M, N, K, x, out, act or "gelu", bias, True)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("x", ["bf16", "f16", "f32"])
def test_gradient_of_every_activation(ops, act, x):
    rng = np.random.default_rng(9)
    for M in (5, 300):
        check_gradient(ops, rng, M, 200, 256, x, x, act, act != "relu", False, True)  # (without a bias a sum's sign is exact)
        if act:
            check_gradient(ops, rng, M, 150, 256, x, "f32", act, act != "relu", True)


@pytest.mark.parametrize("M,N,K,x", [(1, 4096, 1024, "bf16"), (64, 8192, 512, "f16"), (251, 1001, 1090, "f32"), (700, 1366, 777, "bf16"), (1500, 640, 2048, "f16")])
def test_gradient_of_long_reductions(ops, M, N, K, x):
    rng = np.random.default_rng(M + N + K)
    check_gradient(ops, rng, M, N, K, x, x, None, False, False)
    check_gradient(ops, rng, M, N, K, x, x, "silu", True, True)


def test_gradient_against_differences(ops):
    """The quantizer counts as the identity, so a difference is taken where it is one: rows of whole codes, moved by whole codes."""
    rng = np.random.default_rng(2)
    W = Weights(rng, 40, 64, True, 2)
    layer = W.gated(ops, "silu").with_gradient()
    c = rng.integers(-60, 61, (3, 64)).astype(np.float32)
    c[:, 0] = 127  # (every row's scale is 2^-10 * 1)
    x = cuda(c * np.float32(2.0 ** -10)).requires_grad_()
    dy = rows(rng, 3, 40, "f32")
    dx = torch.autograd.grad(layer(x), x, dy)[0]
    for k in (1, 7, 63):
        step = torch.zeros_like(x)
        step[:, k] = 2.0 ** -10
        with torch.no_grad():
            diff = (layer(x + step) - layer(x - step)).double().mul(dy.double()).sum(1) / 2.0 ** -9
        # a step moves each z by at most 127 sw 2^-10: third derivatives, below 3 |u| + 3, times its square over 6, and fp32 results
        # (good to 2^-20 of a few units) over the step
        h = 127 * W.sw.max() * 2.0 ** -10
        bound = (dy.abs().double().sum(1) * (20 * h ** 3 * 2 ** 10 + 2.0 ** -20 * 40 * 2 ** 9)).cpu()
        assert torch.all((dx[:, k].double().cpu() - diff.cpu()).abs() <= bound), k


def test_gradients_that_are_views_expanded_or_not_finite(ops):
    rng = np.random.default_rng(4)
    layer = Weights(rng, 96, 128, True).layer(ops).with_gradient()
    x = rows(rng, 33, 128, "bf16").requires_grad_()
    y = layer(x, activation="silu")
    ones = torch.autograd.grad(y, x, torch.ones_like(y), retain_graph=True)[0]
    assert torch.equal(torch.autograd.grad(y.sum(), x, retain_graph=True)[0], ones)  # an expanded gradient
    dy = rows(rng, 96, 33, "bf16")
    assert torch.equal(torch.autograd.grad(y, x, dy.t(), retain_graph=True)[0], torch.autograd.grad(y, x, dy.t().contiguous(), retain_graph=True)[0])
    cube = layer(x.view(3, 11, 128), activation="silu")
    assert torch.equal(torch.autograd.grad(cube, x, dy.t().reshape(3, 11, 96))[0], torch.autograd.grad(y, x, dy.t(), retain_graph=True)[0])
    bad = torch.ones_like(y)
    bad[4, 7], bad[9, 0] = float("inf"), float("nan")
    dx = torch.autograd.grad(y, x, bad)[0]
    assert F.fxpq_get_device_status() == L.ERR_NONFINITE
    assert bool(dx[[4, 9]].isnan().all()) and torch.equal(dx[:4], ones[:4]) and torch.equal(dx[10:], ones[10:])


def test_gradients_reach_what_lies_below(ops):
    """A feed-forward block between trainable weights: gradients accumulate through both of its layers and its residual."""
    torch.manual_seed(0)
    below = torch.randn(64, 64, device="cuda", requires_grad=True)
    block = ops.GatedLinear8.from_float(torch.randn(100, 64, device="cuda") / 8, torch.randn(100, 64, device="cuda") / 8).with_gradient()
    down = ops.Linear8.from_float(torch.randn(64, 100, device="cuda") / 10).with_gradient()
    x = torch.randn(20, 64, device="cuda")
    h = x @ below
    down(block(h), residual=h).square().sum().backward()
    once = below.grad.clone()
    h = x @ below
    y = down(block(h), residual=h)
    dy = 2 * y.detach()
    dh = torch.autograd.grad(y, h, dy)[0]
    assert torch.equal(once, x.t() @ dh) or torch.allclose(once, x.t() @ dh, rtol=1e-5, atol=1e-4)


def test_what_is_refused(ops):
    rng = np.random.default_rng(1)
    W = Weights(rng, 32, 64, True)
    layer, gate = W.layer(ops), W.gated(ops, "silu")
    x = rows(rng, 4, 64, "bf16")
    for call in (lambda v: layer(v), lambda v: layer(v, activation="relu"), lambda v: gate(v)):
        with pytest.raises(RuntimeError):
            call(x.clone().requires_grad_())
    with pytest.raises(RuntimeError):
        layer(x, residual=rows(rng, 4, 32, "bf16").requires_grad_())
    norm = torch.ones(64, device="cuda")
    with pytest.raises(RuntimeError):
        layer(x, norm=norm.clone().requires_grad_())
    with pytest.raises(RuntimeError):
        W.layer(ops).with_gradient()(x.clone().requires_grad_(), norm=norm)
    with torch.no_grad():
        layer(x.clone().requires_grad_(), norm=norm.clone().requires_grad_())
    for kw in (dict(activation="tanh"), dict(residual=rows(rng, 4, 33, "bf16")), dict(residual=rows(rng, 4, 32, "f16")), dict(residual=rows(rng, 3, 32, "bf16")),
               dict(norm=torch.ones(63, device="cuda")), dict(norm=norm.half()), dict(norm=norm.cpu()), dict(norm=norm, eps=-1.0), dict(norm=norm, eps=2.0)):
        with pytest.raises(ValueError):
            layer(x, **kw)
    with pytest.raises(ValueError):
        layer(x[:, :60], activation="relu")
    with pytest.raises(ValueError):
        gate(x[:, :60])
    with pytest.raises(ValueError):
        gate(x.cpu())
    with pytest.raises(TypeError):
        gate(x, torch.float64)
    w, s = cuda(W.w[:16]), cuda(W.sw[:16])
    b = torch.zeros(16, device="cuda")
    for args in ((w, s, w[:15].contiguous(), s[:15].contiguous()), (w, s, w, s, b), (w, s, w, s, None, b), (w, s[:15].contiguous(), w, s), (w, s, w.float(), s),
                 (w, s, w, s, None, None, None), (w, s, w, s, None, None, "tanh")):
        with pytest.raises(ValueError):
            ops.GatedLinear8(*args)


# ------------------------------------------------------------------------------ streams, graphs, repetition
@pytest.mark.parametrize("M", [3, 200, 700])
def test_streams_graphs_and_repetition(ops, M):
    rng = np.random.default_rng(M)
    W = Weights(rng, 512, 640, True, 2)
    layer, gate = W.layer(ops).with_gradient(), W.gated(ops, "silu").with_gradient()
    norm = torch.ones(640, device="cuda")
    xs = [rows(rng, M, 640, "bf16") for _ in range(3)]
    dy, res = rows(rng, M, 512, "bf16"), rows(rng, M, 1024, "bf16")

    def step(x):
        a = layer(x, norm=norm, activation="gelu", residual=res)
        b = gate(x)
        with torch.enable_grad():
            leaf = x.detach().requires_grad_()
            return a, b, torch.autograd.grad(gate(leaf), leaf, dy)[0]
    want = [step(x) for x in xs]
    for _ in range(3):
        for x, w in zip(xs, want):
            assert all(torch.equal(p, q) for p, q in zip(step(x), w))
    streams = [torch.cuda.Stream() for _ in xs]
    torch.cuda.synchronize()
    got = [None] * 3
    for _ in range(4):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i] = step(xs[i])
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert all(torch.equal(p, q) for p, q in zip(g, w))
    held = xs[0].clone()
    graphs = []
    for _ in range(2):  # two graphs of the same layers, replayed in turn
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            step(held)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = step(held)
        graphs.append((g, out))
    for x, w in zip(xs + xs, want + want):
        held.copy_(x)
        for g, _ in graphs:
            g.replay()
        torch.cuda.synchronize()
        for _, out in graphs:
            assert all(torch.equal(p, q) for p, q in zip(out, w))


def test_the_binding(ops):
    """The header's entry points by their names, into rows with a stride of their own."""
    rng = np.random.default_rng(6)
    W = Weights(rng, 50, 90, True)
    layer = W.layer(ops).with_gradient()
    x = rows(rng, 33, 90, "f16").requires_grad_()
    want = layer(x, torch.float32, activation="silu")
    dy = rows(rng, 33, 50, "f32")
    want_dx = torch.autograd.grad(want, x, dy)[0]
    y = torch.full((33, 55), -7.0, device="cuda")
    pre, sx = torch.empty(33, 56, device="cuda"), torch.empty(33, device="cuda")
    d = L.LayerDesc(x.data_ptr(), 90, None, layer.w.data_ptr(), 96, layer.w_scale.data_ptr(), layer.bias.data_ptr(), None, 0, y.data_ptr(), 55,
                    pre.data_ptr(), sx.data_ptr(), 33, 50, 90, L.FT_F16, L.FT_F32, L.ACT_SILU, 0, L.FT_F32, 0.0)
    ws = torch.empty(F.fxpq_layer_workspace(d), dtype=torch.uint8, device="cuda")
    F.fxpq_layer_forward(d, ws)
    assert torch.equal(y[:, :50], want.detach()) and bool((y[:, 50:] == -7).all())
    dx = torch.full((33, 93), 3.0, dtype=torch.float16, device="cuda")
    g = L.LayerGradDesc(dy.data_ptr(), 50, pre.data_ptr(), sx.data_ptr(), layer.w_scale.data_ptr(), layer.bias.data_ptr(), layer.wt.data_ptr(), 64,
                        dx.data_ptr(), 93, 33, 50, 90, L.FT_F32, L.FT_F16, L.ACT_SILU, 0, L.FT_F32, 0)
    ws = torch.empty(F.fxpq_layer_gradient_workspace(g), dtype=torch.uint8, device="cuda")
    F.fxpq_layer_gradient(g, ws)
    assert torch.equal(dx[:, :90], want_dx) and bool((dx[:, 90:] == 3).all())
    with pytest.raises(L.FxpqError):
        F.fxpq_layer_gradient(g, ws[:256])


@pytest.mark.parametrize("M", [1, 3, 9, 16, 17, 300])
@pytest.mark.parametrize("power", [-98, -60, 0, 60, 118])
def test_rows_far_from_one(ops, M, power):
    """Rows times a power of two (without a norm, whose eps would show): results times that power, exactly but for float32's end, which
    the definition's first product, the sum times the row's scale, passes at 2^118: (some 2^17) * (3.5 to 3.9 / 127) * 2^118 > 2^128."""
    rng = np.random.default_rng(M)
    x = rows(rng, M, 500, "bf16").float().clamp(-3.9, 3.9)
    x[:, 0] = 3.5  # (no row's largest value falls below 2^-100)
    W = Weights(rng, 140, 500, False)
    layer = W.layer(ops)
    want = layer(x, activation="relu")
    got = layer(x * 2.0 ** power, activation="relu")
    codes, sx = O.quantize_tokens((x * 2.0 ** power).cpu().numpy())
    past = torch.from_numpy(O.layer_sums(codes, W.w)[0] * sx.astype(np.float64)[:, None] >= 2.0 ** 128 - 2.0 ** 103).cuda()
    assert power == 118 or not past.any()
    assert torch.equal(got, torch.where(past, float("inf"), want * 2.0 ** power))


@pytest.mark.parametrize("M,K", [(1, 25088), (2, 32768), (3, 20000), (16, 4096), (16, 4095), (9, 7281), (1, 8), (5, 7), (16, 129)])
@pytest.mark.parametrize("x", ["bf16", "f32"])
def test_rows_whose_codes_the_product_forms(ops, M, K, x):
    rng = np.random.default_rng(M + K)
    for N in (130, 512):
        check_layer(ops, rng, M, N, K, x, "f32", "silu", True, True, True)
        check_gated(ops, rng, M, N // 2, K, x, "bf16", "silu", True, False)


def test_no_second_derivative(ops):
    """A graph of the gradient may be asked for, but nothing may silently differentiate through it."""
    rng = np.random.default_rng(3)
    layer = Weights(rng, 32, 64, True).layer(ops).with_gradient()
    x = rows(rng, 4, 64, "f32").requires_grad_()
    plain = torch.autograd.grad(layer(x, activation="silu").sum(), x)[0]
    dx = torch.autograd.grad(layer(x, activation="silu").sum(), x, create_graph=True)[0]
    assert torch.equal(dx.detach(), plain)
    with pytest.raises(RuntimeError):
        dx.sum().backward()


def test_backward_frees_what_it_kept(ops):
    rng = np.random.default_rng(3)
    layer = Weights(rng, 1024, 1024, False).layer(ops).with_gradient()
    x = rows(rng, 2000, 1024, "bf16").requires_grad_()
    y = layer(x, activation="silu")
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    torch.autograd.grad(y, x, torch.ones_like(y))
    for _ in range(100):  # (the engine's thread lets go of them on its own time)
        if torch.cuda.memory_allocated() <= before - 2000 * 1024 * 2:  # the sums
            break
        time.sleep(0.02)
    else:
        raise AssertionError("the kept sums are still there")
    with pytest.raises(RuntimeError):
        torch.autograd.grad(y, x, torch.ones_like(y))


@pytest.mark.parametrize("M,K", [(64, 512), (63, 520), (9, 3640), (17, 1920), (24, 1365), (25, 1310), (40, 819), (33, 8), (64, 1), (48, 100)])
@pytest.mark.parametrize("x", ["bf16", "f32"])
def test_more_rows_whose_codes_the_product_forms(ops, M, K, x):
    rng = np.random.default_rng(M + K)
    for N in (130, 512):
        check_layer(ops, rng, M, N, K, x, "f32", "silu", True, True, True)
        check_gated(ops, rng, M, N // 2, K, x, "bf16", "silu", True, False)


def test_layers_without_channels_or_inputs(ops):
    """No inputs: the biases alone; no channels: no gradient."""
    one = torch.ones(24, device="cuda")
    layer = ops.Linear8(torch.zeros((24, 0), dtype=torch.int8, device="cuda"), one, one * 3).with_gradient()
    y = layer(torch.zeros(70, 0, device="cuda"), activation="silu", norm=torch.zeros(0, device="cuda"))
    assert torch.allclose(y, torch.nn.functional.silu(one * 3).expand(70, 24))
    none = ops.Linear8(torch.zeros((0, 48), dtype=torch.int8, device="cuda"), one[:0].contiguous()).with_gradient()
    x = torch.ones(70, 48, device="cuda", requires_grad=True)
    y = none(x, activation="silu")
    assert y.shape == (70, 0) and torch.equal(torch.autograd.grad(y, x, torch.zeros_like(y))[0], torch.zeros_like(x))


def test_a_residual_that_is_the_output(ops):
    """The header lets a residual be y itself, on every path."""
    rng = np.random.default_rng(0)
    for M, N, K in ((3, 256, 512), (40, 256, 2048), (300, 256, 512), (300, 255, 512), (700, 512, 8192), (1000, 4096, 256)):
        layer, x, r = Weights(rng, N, K, True).layer(ops), rows(rng, M, K, "bf16"), rows(rng, M, N, "bf16")
        want = layer(x, activation="silu", residual=r)
        pitch = (K + 15) // 16 * 16
        d = L.LayerDesc(x.data_ptr(), K, None, layer.w.data_ptr(), pitch, layer.w_scale.data_ptr(), layer.bias.data_ptr(), r.data_ptr(), N, r.data_ptr(),
                        N, None, None, M, N, K, L.FT_BF16, L.FT_BF16, L.ACT_SILU, 0, L.FT_F16, 0.0)
        ws = torch.empty(max(1, F.fxpq_layer_workspace(d)), dtype=torch.uint8, device="cuda")
        F.fxpq_layer_forward(d, ws)
        assert torch.equal(r, want), (M, N, K)


@pytest.mark.parametrize("M", [90, 140, 300, 1300])
def test_unaligned_tensors(ops, M):
    """Outputs, residuals, gradients and kept sums that begin or step at odd places give what aligned ones give."""
    rng = np.random.default_rng(M)
    W = Weights(rng, 256, 512, True)
    layer, x = W.layer(ops).with_gradient(), rows(rng, M, 512, "bf16").requires_grad_()
    wide = rows(rng, M, 261, "bf16")
    r, dy = wide[:, 3:259], rows(rng, M, 259, "bf16")[:, 2:258]
    y = layer(x, activation="silu", residual=r.contiguous())
    assert torch.equal(layer(x, activation="silu", residual=r), y)
    dx = torch.autograd.grad(y, x, dy.contiguous(), retain_graph=True)[0]
    assert torch.equal(torch.autograd.grad(y, x, dy)[0], dx)
    big = torch.zeros(M * 257 + 1, dtype=torch.bfloat16, device="cuda")
    d = L.LayerDesc(x.data_ptr(), 512, None, layer.w.data_ptr(), 512, layer.w_scale.data_ptr(), layer.bias.data_ptr(), r.data_ptr(), 261,
                    big.data_ptr() + 2, 257, None, None, M, 256, 512, L.FT_BF16, L.FT_BF16, L.ACT_SILU, 0, L.FT_F16, 0.0)
    F.fxpq_layer_forward(d, torch.empty(max(1, F.fxpq_layer_workspace(d)), dtype=torch.uint8, device="cuda"))
    got = big[1:].view(M, 257)
    assert torch.equal(got[:, :256], y.detach()) and not got[:, 256].any()


@pytest.mark.parametrize("N", [9000, 12285, 12288, 12290, 16384, 20001, 24576, 24584])
def test_gradient_of_very_wide_layers(ops, N):
    """Rows of more channels than a block keeps: what does not fit is formed again."""
    rng = np.random.default_rng(N)
    check_gradient(ops, rng, 5, N, 40, "bf16", "bf16", "silu", True, False)
    check_gradient(ops, rng, 70, N // 2, 24, "f16", "f16", "gelu", False, True)
    check_gradient(ops, rng, 3, N, 16, "f32", "f32", None, False, False)


@pytest.mark.parametrize("M", [7, 100, 300, 1300, 10000])
@pytest.mark.parametrize("out", ["bf16", "f32"])
def test_nan_stays_in_its_channel(ops, M, out):
    """A NaN scale or bias gives its own channel NaN, whatever the activation, and leaves every other as it is."""
    rng = np.random.default_rng(M)
    W = Weights(rng, 256, 512, True, 2)
    x, r = rows(rng, M, 512, "bf16"), rows(rng, M, 512, out)
    calls = lambda act: (W.layer(ops)(x, TYPES[out], activation=act, residual=r), W.gated(ops, act or "silu")(x, TYPES[out]))
    before = {act: calls(act) for act in ACTS}
    W.b[6], W.sw[201], W.b[510] = np.nan, np.nan, np.nan
    for act in ACTS:
        for y, want, bad in zip(calls(act), before[act], ([6, 201, 510], [3, 100, 255])):
            good = [c for c in range(y.shape[1]) if c not in bad]
            assert bool(y[:, bad].isnan().all()), act
            assert torch.equal(y[:, good], want[:, good]), act


@pytest.mark.parametrize("M", [100, 300, 1300, 10000])
@pytest.mark.parametrize("act", ACTS)
def test_gradients_of_many_rows_that_are_not_finite(ops, M, act):
    rng = np.random.default_rng(M)
    layer = Weights(rng, 256, 512, True).layer(ops).with_gradient()
    x = rows(rng, M, 512, "bf16").requires_grad_()
    y = layer(x, activation=act)
    bad = rows(rng, M, 256, "bf16")
    want = torch.autograd.grad(y, x, bad, retain_graph=True)[0]
    at = [4, M // 2, M - 1]
    bad[at[0], 7], bad[at[1], 0], bad[at[2], 255] = float("nan"), float("nan"), float("nan")
    dx = torch.autograd.grad(y, x, bad)[0]
    assert F.fxpq_get_device_status() == L.ERR_NONFINITE
    good = [m for m in range(M) if m not in at]
    assert bool(dx[at].isnan().all()) and torch.equal(dx[good], want[good])


@pytest.mark.parametrize("N", [6, 50, 512, 9000])
@pytest.mark.parametrize("is_gated", [False, True])
@pytest.mark.parametrize("dx_type", ["f32", "bf16"])
def test_kept_sums_of_any_type_with_a_gradient_of_any(ops, N, is_gated, dx_type):
    """fp32 gradients with sums kept in fp16: what the same gradients in bfloat16 give, bit for bit."""
    rng = np.random.default_rng(N)
    M, K = 37, 90
    W = Weights(rng, N, K, True)
    layer = W.layer(ops).with_gradient()
    ft = {"f32": L.FT_F32, "bf16": L.FT_BF16}
    x, pitch = rows(rng, M, K, "bf16"), (N + 7) // 8 * 8
    wide = N // 2 if is_gated else N
    for pre_type, kept in ((L.FT_F16, torch.float16), (L.FT_F32, torch.float32)):
        y, pre, sx = torch.empty(M, wide, device="cuda"), torch.zeros(M, pitch, dtype=kept, device="cuda"), torch.empty(M, device="cuda")
        d = L.LayerDesc(x.data_ptr(), K, None, layer.w.data_ptr(), 96, layer.w_scale.data_ptr(), layer.bias.data_ptr(), None, 0, y.data_ptr(), wide,
                        pre.data_ptr(), sx.data_ptr(), M, N, K, L.FT_BF16, L.FT_F32, L.ACT_GELU, int(is_gated), pre_type, 0.0)
        F.fxpq_layer_forward(d, torch.empty(F.fxpq_layer_workspace(d), dtype=torch.uint8, device="cuda"))
        dy, got = rows(rng, M, wide, "bf16"), []
        for t in ("bf16", "f32"):
            g_dy, dx = dy.to(TYPES[t]), torch.empty(M, K, dtype=TYPES[dx_type], device="cuda")
            g = L.LayerGradDesc(g_dy.data_ptr(), wide, pre.data_ptr(), sx.data_ptr(), layer.w_scale.data_ptr(), layer.bias.data_ptr(),
                                layer.wt.data_ptr(), layer.wt.stride(0), dx.data_ptr(), K, M, N, K, ft[t], ft[dx_type], L.ACT_GELU, int(is_gated),
                                pre_type, 0)
            F.fxpq_layer_gradient(g, torch.empty(F.fxpq_layer_gradient_workspace(g), dtype=torch.uint8, device="cuda"))
            got.append(dx)
        assert torch.equal(*got) and bool(got[0].isfinite().all()) and bool((got[0] != 0).any())


@pytest.mark.parametrize("M,K", [(1, 32768), (1, 32769), (2, 16384), (2, 16385), (3, 10922), (3, 10923), (4, 8192), (8, 4096), (8, 4097), (9, 1820),
                                 (9, 1821), (16, 1024), (16, 1025), (13, 1260), (5, 6553), (1, 16896)])
@pytest.mark.parametrize("x", ["bf16", "f16", "f32"])
def test_both_sides_of_the_rule_for_rows_whose_codes_the_product_forms(ops, M, K, x):
    """At most 32768 values of up to 8 rows, or 16384 of up to 16: the last size of that form, the first of the other, and shares of 32 blocks."""
    rng = np.random.default_rng(M + K)
    need = F.fxpq_layer_workspace(L.LayerDesc(None, K, None, None, (K + 15) // 16 * 16, None, None, None, 0, None, 130, None, None, M, 130, K, L.FT_BF16,
                                              L.FT_BF16, L.ACT_RELU, 0, L.FT_F16, 0.0))
    assert (need == 0) == (M * K <= (32768 if M <= 8 else 16384))
    for N in (130, 512):
        check_layer(ops, rng, M, N, K, x, "f32", "silu", True, True, True)
        check_layer(ops, rng, M, N, K, x, "bf16", None, False, False, True)
        check_gated(ops, rng, M, N // 2, K, x, "bf16", "silu", True, False)
