"""The 8-bit language-model operators on the GPU against the 64-bit oracle.

Codes, scales and fp32 rotations compare bit for bit.  Floating outputs are held to bounds that follow from
the arithmetic (tests below state them), not to measured differences."""
import math

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
def status_is_clear(request):
    yield
    assert F.fxpq_get_device_status() == L.OK


def cuda(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(dtype)


def host(t):
    return t.double().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


# ------------------------------------------------------------------------------ rows to codes
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("M,K", [(1, 1), (3, 7), (5, 8), (2, 64), (17, 100), (1, 4096), (4, 8191), (3, 8200), (2, 25088), (300, 129)])
def test_quantize_tokens(ops, dtype, M, K):
    rng = np.random.default_rng(M * 1000 + K)
    x = cuda(rng.normal(size=(M, K)) * np.exp(rng.normal(size=(M, 1)) * 3), TYPES[dtype])
    if M > 2:
        x[1] = 0
    codes, scale = ops.quantize_tokens(x)
    want, ws = O.quantize_tokens(x.float().cpu().numpy())
    assert np.array_equal(codes.cpu().numpy(), want) and np.array_equal(scale.cpu().numpy(), ws)
    if M > 1:
        assert codes.stride(0) % 16 == 0


def test_quantize_tokens_views_ties_and_tiny_rows(ops):
    rng = np.random.default_rng(5)
    big = cuda(rng.normal(size=(9, 203)), torch.float16)
    for view in (big[:, 1:102], big[::2, :200], big[:, :64], big.t()[:50]):
        codes, scale = ops.quantize_tokens(view)
        want, ws = O.quantize_tokens(view.float().cpu().numpy())
        assert np.array_equal(codes.cpu().numpy(), want) and np.array_equal(scale.cpu().numpy(), ws)
    x = torch.tensor([[127.0, 0.5, 1.5, 2.5, -0.5, -1.5]], device="cuda")
    assert ops.quantize_tokens(x)[0].tolist() == [[127, 0, 2, 2, 0, -2]]
    x = torch.tensor([[2.0 ** -101, 0.0], [2.0 ** -100, 2.0 ** -101], [2.0 ** -140, 2.0 ** -149]], device="cuda")
    codes, scale = ops.quantize_tokens(x)
    assert codes.tolist() == [[0, 0], [127, 64], [0, 0]] and scale[0] == 0 and scale[1] > 0 and scale[2] == 0
    y, s = ops.quantize_tokens(cuda(rng.normal(size=(2, 3, 40)), torch.bfloat16))
    assert y.shape == (2, 3, 40) and s.shape == (2, 3)
    assert ops.quantize_tokens(x[:0])[0].shape == (0, 2)


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_quantize_tokens_latches_non_finite_values(ops, value):
    x = torch.ones(3, 70, device="cuda")
    x[1, 69] = value
    codes, scale = ops.quantize_tokens(x)
    assert F.fxpq_get_device_status() == L.ERR_NONFINITE
    want, ws = O.quantize_tokens(x.cpu().numpy())
    assert np.array_equal(codes.cpu().numpy(), want) and np.array_equal(scale.cpu().numpy(), ws) and codes[1, 69] == 0


# ------------------------------------------------------------------------------ the product
def check_linear(ops, M, N, K, out, bias, rng, codes=None, w=None):
    codes = rng.integers(-127, 128, (M, K), dtype=np.int8) if codes is None else codes
    w = rng.integers(-127, 128, (N, K), dtype=np.int8) if w is None else w
    sx, sw = np.exp(rng.normal(size=M)).astype(np.float32) * 0.01, np.exp(rng.normal(size=N)).astype(np.float32) * 0.01
    b = rng.normal(size=N).astype(np.float32) if bias else None
    layer = ops.Linear8(cuda(w), cuda(sw), None if b is None else cuda(b))
    pitch = (K + 15) // 16 * 16
    x = torch.zeros((M, pitch), dtype=torch.int8, device="cuda")
    x[:, :K] = cuda(codes)
    if pitch != K:
        x[:, K:] = 77  # bytes past a row's end are not used
    y = ops.linear_i8(x[:, :K], cuda(sx), layer.w, layer.w_scale, layer.bias, TYPES[out])
    want, mag = O.linear(codes, sx, w, sw, b)
    # exact products; each step of 16 rounds (or cuts) its sum to 24 bits; three fp32 roundings; the output's own
    exact = np.abs(codes.astype(np.int64)) @ np.abs(w.astype(np.int64)).T < 2 ** 24
    steps = np.where(exact, 0.0, (K / 16 + 1) * 2.0 ** -23)
    bound = mag * (steps + 2.0 ** -22) + np.abs(want) * UNIT[out] + 2.0 ** -24 * (out == "f16")
    err = np.abs(host(y) - want)
    assert y.shape == (M, N) and y.dtype == TYPES[out]
    assert np.all(err <= bound), (np.max(err / np.maximum(bound, 1e-300)), np.argwhere(err > bound)[:5])


@pytest.mark.parametrize("M", [1, 2, 7, 16, 17, 33, 64, 65, 129, 251])
@pytest.mark.parametrize("N,K", [(1, 1), (8, 16), (100, 64), (130, 100), (257, 1023), (1001, 520), (512, 2048)])
def test_linear_sizes(ops, M, N, K):
    rng = np.random.default_rng(M * 7 + N + K)
    check_linear(ops, M, N, K, ["bf16", "f16", "f32"][(M + N) % 3], (M + K) % 2, rng)


@pytest.mark.parametrize("M,N,K,out", [(1, 4096, 4096, "bf16"), (5, 4096, 25088, "f32"), (64, 1000, 25088, "f16"), (300, 4096, 4090, "f32"),
                                       (1000, 1111, 777, "bf16"), (2048, 2048, 512, "f16"), (1500, 4100, 128, "f32"), (40, 152 * 128 + 1, 64, "bf16"),
                                       (513, 640, 8192, "f32"), (260, 5000, 1600, "f32")])
def test_linear_large(ops, M, N, K, out):
    check_linear(ops, M, N, K, out, True, np.random.default_rng(M + N + K))


@pytest.mark.parametrize("M", [3, 200])
@pytest.mark.parametrize("a,b", [(127, 127), (-128, -128), (-128, 127)])
def test_linear_sums_past_24_bits(ops, M, a, b):
    rng = np.random.default_rng(1)
    check_linear(ops, M, 136, 8192 + 16, "f32", False, rng, np.full((M, 8208), a, np.int8), np.full((136, 8208), b, np.int8))
    check_linear(ops, M, 136, 1008, "f32", False, rng, np.full((M, 1008), a, np.int8), np.full((136, 1008), b, np.int8))  # exact


def test_linear_into_views_streams_and_empty(ops):
    rng = np.random.default_rng(8)
    c, w = rng.integers(-127, 128, (50, 96), dtype=np.int8), rng.integers(-127, 128, (70, 96), dtype=np.int8)
    one = torch.ones(200, device="cuda")
    want = (c.astype(np.int64) @ w.T.astype(np.int64)).astype(np.float32)
    big = torch.full((50, 75), -5.0, device="cuda")  # rows with a stride of their own, columns past N untouched
    tx, tw = cuda(c), cuda(w)
    need = F.fxpq_linear_i8_workspace(50, 70, 96)
    ws = torch.empty(max(need, 1), dtype=torch.uint8, device="cuda")
    F.fxpq_linear_i8(tx, 96, one, tw, 96, one, None, 50, 70, 96, L.FT_F32, big[:, 2:], 75, ws)
    assert np.array_equal(big[:, 2:72].cpu().numpy(), want) and bool((big[:, :2] == -5).all()) and bool((big[:, 72:] == -5).all())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y = ops.linear_i8(tx, one[:50], tw, one[:70], None, torch.float32)
    side.synchronize()
    assert np.array_equal(y.cpu().numpy(), want)
    assert ops.linear_i8(tx[:0], one[:0], tw, one[:70]).shape == (0, 70)
    empty = torch.empty((3, 0), dtype=torch.int8, device="cuda")
    y = ops.linear_i8(empty, one[:3], torch.empty((5, 0), dtype=torch.int8, device="cuda"), one[:5], one[5:10] * 2, torch.float32)
    assert bool((y == 2).all())


def test_linear_layer_from_floats(ops):
    torch.manual_seed(0)
    w, x, b = torch.randn(200, 330, device="cuda") / 18, torch.randn(2, 9, 330, device="cuda").bfloat16(), torch.randn(200, device="cuda")
    layer = ops.Linear8.from_float(w, b)
    y = layer(x, torch.float32)
    assert y.shape == (2, 9, 200)
    # each operand's values are within half a code of theirs: sum over 330 of the two errors' products with the other
    sx, sw = x.float().abs().amax(-1, keepdim=True) / 127, w.abs().amax(-1) / 127
    bound = 0.5 * (sx * w.abs().sum(-1) + sw * x.float().abs().sum(-1, keepdim=True) + 0.5 * 330 * sx * sw) * 1.001
    assert bool(((y - (x.float() @ w.t() + b)).abs() <= bound).all())


def test_linear_layers_on_two_streams_and_in_a_graph(ops):
    """Calls of growing and shrinking size on two streams at once, and a captured one replayed after others."""
    torch.manual_seed(1)
    layers = [ops.Linear8.from_float(torch.randn(200, 256, device="cuda")) for _ in range(2)]
    xs = [torch.randn(m, 256, device="cuda").half() for m in (3, 700, 40, 1500, 1)]
    want = [[lay(x) for x in xs] for lay in layers]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(20):
        for s, lay, g in zip(streams, layers, got):
            with torch.cuda.stream(s):
                g[:] = [lay(x) for x in xs]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for w, g in zip(want, got) for a, b in zip(w, g))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = layers[0](xs[2])
    big = [layers[1](torch.randn(4000, 256, device="cuda").half()) for _ in range(3)]
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want[0][2]) and len(big) == 3


# ------------------------------------------------------------------------------ appending
def make(rng, lens, page, heads, dim, **kw):
    c, table = O.paged(rng, lens, page, heads, dim, **kw)
    return c, table


def on_gpu(ops, c):
    return ops.KVCache(cuda(c.k), cuda(c.v), cuda(c.k_scale), cuda(c.v_scale))


def same_cache(gpu, c):
    assert np.array_equal(gpu.k_scale.cpu().numpy(), c.k_scale) and np.array_equal(gpu.v_scale.cpu().numpy(), c.v_scale)
    assert np.array_equal(gpu.k.cpu().numpy(), c.k) and np.array_equal(gpu.v.cpu().numpy(), c.v)


def check_append(ops, news, ctxs, page, hq, hkv, dim, dtype, rot, inter, ragged, seed=0, layout="fused", arbitrary=False, spread=1.0):
    rng = np.random.default_rng(seed)
    lens = [a + b for a, b in zip(news, ctxs)]
    c, table = make(rng, lens, page, hkv, dim, arbitrary=arbitrary)
    gpu = on_gpu(ops, c)
    T, W = sum(news), hq + 2 * hkv
    vals = rng.normal(size=(T, W, dim)) * np.exp(spread * rng.normal(size=(T, W, 1)))
    if layout == "fused":
        x = cuda(vals, TYPES[dtype])
    elif layout == "odd":  # strides and addresses that are no multiple of an access
        x = torch.zeros((T, W * (dim + 1) + 3), dtype=TYPES[dtype], device="cuda")[:, 1:1 + W * (dim + 1)].unflatten(1, (W, dim + 1))[:, :, :dim]
        x.copy_(cuda(vals))
    else:  # heads outermost
        x = cuda(vals.transpose(1, 0, 2), TYPES[dtype]).transpose(0, 1)
    q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
    cos, sin = O.rope_tables(max(lens + [1]), rot) if rot else (None, None)
    starts = np.concatenate([[0], np.cumsum(news)]).astype(np.int32)
    args = dict(q=q, starts=cuda(starts) if ragged else None, cos=None if cos is None else cuda(cos), sin=None if sin is None else cuda(sin),
                interleaved=inter)
    f = x.float().cpu().numpy()
    want = O.append(c, table, lens, starts, f[:, hq:hq + hkv], f[:, hq + hkv:], f[:, :hq], cos, sin, inter)
    for _ in range(2):  # appending the same rows again changes nothing
        out = ops.kv_append(gpu, cuda(table), cuda(np.array(lens, np.int32)), k, v, **args)
        same_cache(gpu, c)
        assert torch.equal(out.float().cpu(), torch.from_numpy(want).to(TYPES[dtype]).float())


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("dtype,rot,inter", [("bf16", 64, False), ("f16", 32, True), ("f32", 8, False), ("bf16", 0, False), ("f16", 24, False)])
def test_append_single_tokens(ops, dim, page, dtype, rot, inter):
    ctxs = [0, 1, page - 1, page, page + 1, 2 * page - 1, 5]
    check_append(ops, [1] * 7, ctxs, page, 6, 2, dim, dtype, rot, inter, ragged=False, seed=page + dim)


@pytest.mark.parametrize("page", [16, 64, 128])
@pytest.mark.parametrize("dtype,rot,inter,layout", [("bf16", 128, False, "fused"), ("f16", 64, True, "odd"), ("f32", 128, True, "outer"),
                                                    ("bf16", 128, True, "odd"), ("f32", 64, False, "odd")])
def test_append_chunks(ops, page, dtype, rot, inter, layout):
    news, ctxs = [0, 1, page, 2 * page + 1, 37, 0, page - 1, 3, 200], [4, page - 1, 0, 7, 2 * page, 0, 1, 0, 3]
    check_append(ops, news, ctxs, page, 3, 3, 128, dtype, rot, inter, ragged=True, seed=page, layout=layout)


@pytest.mark.parametrize("n", [2, 7, 8, 100])
def test_append_same_count_each(ops, n):
    check_append(ops, [n] * 5, [0, 3, 15, 16, 200], 16, 8, 1, 64, "bf16", 64, False, ragged=False, seed=n)


def test_append_many_sequences(ops):
    rng = np.random.default_rng(3)
    news, ctxs = rng.integers(0, 5, 1100).tolist(), rng.integers(0, 40, 1100).tolist()
    check_append(ops, news, ctxs, 16, 1, 1, 64, "bf16", 64, False, ragged=True)


def test_append_to_blocks_with_any_scale_and_wild_values(ops):
    check_append(ops, [1] * 6, [1, 3, 15, 31, 20, 0], 16, 2, 2, 64, "f32", 64, False, ragged=False, arbitrary=True)
    check_append(ops, [9] * 6, [1, 3, 15, 31, 20, 0], 16, 2, 2, 64, "f32", 64, False, ragged=False, arbitrary=True, spread=20.0)


def test_append_extremes(ops):
    """Zero blocks take the smallest scale, huge values the largest; non-finite ones code 0 and the status."""
    c = ops.KVCache.empty(3, 1, 16, 64)
    pages, lens = torch.tensor([[0], [1], [2]], dtype=torch.int32, device="cuda"), torch.ones(3, dtype=torch.int32, device="cuda")
    k = torch.zeros(3, 1, 64, device="cuda")
    k[1] = 3e38
    k[2, 0, 5] = 2.0
    ops.kv_append(c, pages, lens, k, -k)
    assert c.k_scale[:, 0].tolist() == [2.0 ** -40, 2.0 ** 32, 2.0 ** -5] and c.k[1, 0, 0, 0] == 127 and c.v[1, 0, 0, 0] == -128
    assert c.k[2, 0, 0, 5] == 64 and c.v[2, 0, 0, 5] == -64
    k[2, 0, 6], k[2, 0, 7] = float("inf"), float("nan")
    ops.kv_append(c, pages, lens, k, -k)
    assert F.fxpq_get_device_status() == L.ERR_NONFINITE
    assert c.k[2, 0, 0, 4:9].tolist() == [0, 64, 0, 0, 0] and c.k_scale[2, 0] == 2.0 ** -5


def test_append_padding_bad_pages_and_positions(ops):
    rng = np.random.default_rng(4)
    x = torch.randn(4, 3, 64, device="cuda")
    cos, sin = (cuda(t) for t in O.rope_tables(20, 64))
    c = ops.KVCache.empty(4, 1, 16, 64)
    lens = torch.tensor([3, 0, 21, 5], dtype=torch.int32, device="cuda")  # 0: padding; 21: past the tables
    pages = torch.tensor([[0, -1], [-1, -1], [1, 2], [9, -1]], dtype=torch.int32, device="cuda")
    before = [t.clone() for t in (c.k, c.v, c.k_scale, c.v_scale)]
    q = ops.kv_append(c, pages[:3], lens[:3], x[:3, 1:2], x[:3, 2:3], q=x[:3, :1], cos=cos, sin=sin)
    assert F.fxpq_get_device_status() == L.ERR_RANGE
    assert bool(q[0].any()) and not bool(q[1].any()) and not bool(q[2].any())
    assert torch.equal(c.k[1:], before[0][1:]) and bool(c.k[0, 0, 2].any())
    ops.kv_append(c, pages[3:], lens[3:], x[3:, 1:2], x[3:, 2:3])  # page 9 of 4
    assert F.fxpq_get_device_status() == L.ERR_RANGE
    assert torch.equal(c.k[1:], before[0][1:]) and torch.equal(c.v[1:], before[1][1:]) and torch.equal(c.v_scale[1:], before[3][1:])
    long = torch.tensor([33], dtype=torch.int32, device="cuda")  # token 32 is on a third page of two
    ops.kv_append(c, pages[2:3], long, x[:1, :1], x[:1, :1])
    assert F.fxpq_get_device_status() == L.ERR_RANGE


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("page,heads,dim", [(16, 1, 64), (64, 3, 128), (128, 8, 128)])
def test_values(ops, dtype, page, heads, dim):
    rng = np.random.default_rng(page)
    c, _ = make(rng, [5 * page], page, heads, dim, arbitrary=True)
    gpu = on_gpu(ops, c)
    ids = np.array([3, 0, 3, 6], np.int32)
    k, v = ops.kv_values(gpu, cuda(ids), TYPES[dtype])
    for got, codes, scale in ((k, c.k, c.k_scale), (v, c.v, c.v_scale)):
        want = torch.from_numpy(codes[ids].astype(np.float32) * scale[ids][:, :, None, None]).to(TYPES[dtype])
        assert torch.equal(got.cpu(), want)
    k, _ = ops.kv_values(gpu, torch.tensor([99, -1], dtype=torch.int32, device="cuda"), TYPES[dtype])
    assert F.fxpq_get_device_status() == L.ERR_RANGE and not bool(k.any())


# ------------------------------------------------------------------------------ attention
def check_attention(ops, news, ctxs, page, hq, hkv, dim, dtype, causal, ragged, seed=0, layout="plain", arbitrary=True, scale=None, size=1.0,
                    lens=None):
    rng = np.random.default_rng(seed)
    lens = [a + b for a, b in zip(news, ctxs)] if lens is None else lens
    c, table = make(rng, lens, page, hkv, dim, arbitrary=arbitrary)
    gpu = on_gpu(ops, c)
    T = sum(news)
    vals = rng.normal(size=(T, hq, dim)) * size
    if layout == "odd":
        q = torch.zeros((T, hq * (dim + 3) + 5), dtype=TYPES[dtype], device="cuda")[:, 1:1 + hq * (dim + 3)].unflatten(1, (hq, dim + 3))[:, :, :dim]
        q.copy_(cuda(vals))
    elif layout == "outer":
        q = cuda(vals.transpose(1, 0, 2), TYPES[dtype]).transpose(0, 1)
    else:
        q = cuda(vals, TYPES[dtype])
    starts = np.concatenate([[0], np.cumsum(news)]).astype(np.int32)
    scale = O.default_scale(dim) if scale is None else scale
    out, lse = ops.kv_attention(gpu, cuda(table), cuda(np.array(lens, np.int32)), q, starts=cuda(starts) if ragged else None, scale=scale,
                                causal=causal, return_lse=True)
    want, wl, spread, slack = O.attention(c, table, lens, starts, q.double().cpu().numpy(), scale, causal)
    compare_attention(out, lse, want, wl, spread, slack, dtype, max(lens), np.abs(c.v).max() * c.v_scale.max())
    return gpu


def compare_attention(out, lse, want, wl, spread, slack, dtype, n, vmax):
    """Scores: 128 exact products summed in fp32 and a few fp32 roundings, at most slack 2^-16 off; each weight then
    relatively twice that, 2^-10 for its rounding to fp16 and the exponential; weights below fp16's range 2^-25 of
    the largest each; the output's rounding."""
    s = slack[:, :, None] * 2.0 ** -16
    bound = (2 * s + 2.0 ** -10) * 2 * spread + n * 2.0 ** -25 * vmax + np.abs(want) * UNIT[dtype] + 2.0 ** -24
    err = np.abs(host(out) - want)
    assert np.all(err <= bound), (np.nanmax(err / bound), np.argwhere(~(err <= bound))[:4])
    got = host(lse)
    dead = np.isneginf(wl)
    assert np.array_equal(np.isneginf(got), dead) and not np.isnan(got).any()
    lb = s[:, :, 0] + n * 2.0 ** -24 + 2.0 ** -18 + np.abs(np.where(dead, 0, wl)) * 2.0 ** -22
    assert np.all(np.abs(np.where(dead, 0, got) - np.where(dead, 0, wl)) <= lb)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("hq,hkv,dtype", [(2, 2, "bf16"), (10, 2, "f16"), (8, 1, "bf16"), (33, 3, "f16"), (24, 1, "bf16")])
def test_attention_single_tokens(ops, dim, page, hq, hkv, dtype):
    ctxs = [0, 1, page - 1, page, 31, 32, 33, 127, 300, 64]
    check_attention(ops, [1] * 10, ctxs, page, hq, hkv, dim, dtype, True, False, seed=page + hq)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("page", [16, 64, 128])
@pytest.mark.parametrize("hq,hkv,dim,dtype,layout", [(4, 1, 128, "bf16", "plain"), (2, 2, 64, "f16", "odd"), (16, 2, 64, "bf16", "outer"),
                                                     (5, 1, 128, "f16", "odd"), (1, 1, 128, "bf16", "plain")])
def test_attention_chunks(ops, causal, page, hq, hkv, dim, dtype, layout):
    news, ctxs = [3, 0, 130, 1, 67, 257, 16], [0, 9, 0, page, 2 * page + 5, 130, 500]
    check_attention(ops, news, ctxs, page, hq, hkv, dim, dtype, causal, True, seed=page + hq + causal, layout=layout)


@pytest.mark.parametrize("n,hq,hkv", [(2, 8, 2), (4, 32, 8), (7, 5, 1), (8, 4, 1), (9, 16, 4), (31, 3, 3), (64, 8, 1)])
def test_attention_few_tokens_over_caches(ops, n, hq, hkv):
    check_attention(ops, [n] * 3, [0, 513, 70], 32, hq, hkv, 128, "bf16", True, False, seed=n)


@pytest.mark.parametrize("n", [1, 5, 40, 300])
@pytest.mark.parametrize("dim,page", [(64, 16), (128, 128)])
def test_attention_long_caches_are_split(ops, n, dim, page):
    check_attention(ops, [n, n], [9000 - n, 4097], page, 4, 2, dim, "bf16", True, False, seed=n)


@pytest.mark.parametrize("page,dim,hq,hkv,dtype,causal", [(16, 64, 8, 1, "bf16", True), (64, 128, 8, 2, "f16", True), (128, 128, 5, 1, "bf16", False),
                                                          (32, 64, 16, 2, "f16", False)])
def test_attention_of_many_rows_expands_the_codes_first(ops, page, dim, hq, hkv, dtype, causal):
    check_attention(ops, [301, 260, 0, 513], [0, 77, 9, 130], page, hq, hkv, dim, dtype, causal, True, seed=page)
    check_attention(ops, [600, 600], [0, 1], page, hq, hkv, dim, dtype, causal, False, seed=page + 1)
    check_attention(ops, [400] * 3, None, page, hq, hkv, dim, dtype, causal, False, lens=[390, 0, 400])


def test_attention_of_many_rows_masks_bad_pages(ops):
    rng = np.random.default_rng(17)
    c, table = make(rng, [400], 32, 1, 64)
    q, tl = cuda(rng.normal(size=(150, 8, 64)), torch.bfloat16), torch.tensor([400], dtype=torch.int32, device="cuda")
    bad = table.copy()
    bad[0, 2], bad[0, 5] = -7, len(c.k)
    out, lse = ops.kv_attention(on_gpu(ops, c), cuda(bad), tl, q, return_lse=True)
    assert F.fxpq_get_device_status() == L.ERR_RANGE
    keep = [i for i in range(table.shape[1]) if i not in (2, 5)]
    want, wl, spread, slack = O.attention(c, table[:, keep], [400 - 64], [0, 150], q.double().cpu().numpy(), O.default_scale(64), True)
    compare_attention(out, lse, want, wl, spread, slack, "bf16", 400, np.abs(c.v).max() * c.v_scale.max())


@pytest.mark.parametrize("rows", [150, 260, 300])  # the last two are of more than 2048 rows a key head: their codes are expanded
def test_attention_of_more_rows_masks_bad_pages(ops, rows):
    rng = np.random.default_rng(rows)
    c, table = make(rng, [700, 333], 32, 1, 64)
    q, tl = cuda(rng.normal(size=(2 * rows, 8, 64)), torch.float16), torch.tensor([700, 333], dtype=torch.int32, device="cuda")
    bad = table.copy()
    bad[0, 1], bad[0, 4], bad[0, 9], bad[1, 0] = -1, len(c.k), 2**31 - 1, -5
    out, lse = ops.kv_attention(on_gpu(ops, c), cuda(bad), tl, q, causal=False, return_lse=True)
    assert F.fxpq_get_device_status() == L.ERR_RANGE
    for b, (n, gone) in enumerate([(700, (1, 4, 9)), (333, (0,))]):
        keep = [i for i in range(-(-n // 32)) if i not in gone]
        mine = slice(b * rows, (b + 1) * rows)
        want, wl, spread, slack = O.attention(c, table[b:b + 1, keep], [n - 32 * len(gone)], [0, rows], q[mine].double().cpu().numpy(),
                                              O.default_scale(64), False)
        compare_attention(out[mine], lse[mine], want, wl, spread, slack, "f16", n, np.abs(c.v).max() * c.v_scale.max())


@pytest.mark.parametrize("dim,dtype", [(64, "bf16"), (128, "f16")])
@pytest.mark.parametrize("causal", [True, False])
def test_attention_of_more_rows_expanded_and_ragged(ops, dim, dtype, causal):
    check_attention(ops, [700, 513, 1, 1100], [0, 77, 900, 130], 64, 8, 2, dim, dtype, causal, True, seed=dim)
    check_attention(ops, [2100, 2100], [3, 0], 16, 1, 1, dim, dtype, causal, False, seed=dim + 1)
    check_attention(ops, [600] * 3, None, 128, 4, 1, dim, dtype, causal, False, lens=[590, 0, 600])


@pytest.mark.parametrize("n", [40, 300, 600])
@pytest.mark.parametrize("dim", [64, 128])
def test_attention_maxima_that_grow_in_either_half_of_a_step(ops, n, dim):
    """Keys that grow along the sequence, so that the running maximum moves in most steps, by turns in either 64 of 128."""
    rng = np.random.default_rng(n + dim)
    c, table = make(rng, [1500], 64, 1, dim)
    c.k[:] = np.sign(rng.normal(size=dim) + 0.2)[None, None, None] * 20
    block = np.argsort(np.argsort(table[0]))
    for i, p in enumerate(table[0]):
        c.k[p, 0, :, :] = np.clip(c.k[p, 0] * (1 + block[i] % 5), -127, 127)
        c.k_scale[p] = 2.0 ** (-9 + i // 4)
    q = cuda(np.abs(rng.normal(size=(n, 4, dim))) * np.sign(c.k[table[0, 0], 0, 0]), torch.float16)
    tl = torch.tensor([1500], dtype=torch.int32, device="cuda")
    out, lse = ops.kv_attention(on_gpu(ops, c), cuda(table), tl, q, causal=False, return_lse=True)
    want, wl, spread, slack = O.attention(c, table, [1500], [0, n], q.double().cpu().numpy(), O.default_scale(dim), False)
    compare_attention(out, lse, want, wl, spread, slack, "f16", 1500, np.abs(c.v).max() * c.v_scale.max())


def test_attention_rows_that_see_nothing(ops):
    # length 0, fewer tokens than new rows, and a sequence without pages, in both sizes of batch
    check_attention(ops, [1] * 4, None, 16, 4, 2, 64, "bf16", True, False, lens=[0, 1, 5, 0])
    check_attention(ops, [6, 6, 6], None, 16, 4, 2, 128, "bf16", True, False, lens=[4, 0, 6])
    check_attention(ops, [140, 140, 140], None, 16, 4, 2, 64, "f16", True, False, lens=[4, 0, 139])
    check_attention(ops, [140, 140, 140], None, 16, 4, 2, 64, "f16", False, False, lens=[4, 0, 141])


@pytest.mark.parametrize("n", [1, 150])
@pytest.mark.parametrize("size,scale", [(1e-3, None), (300.0, 0.01), (1.0, 3.0), (1.0, 1e-6)])
def test_attention_sharp_flat_and_scaled(ops, n, size, scale):
    check_attention(ops, [n, n], [700, 90], 64, 4, 2, 128, "bf16", True, False, seed=n, size=size, scale=scale)


@pytest.mark.parametrize("n", [1, 150])
def test_attention_blocks_of_very_unequal_scales(ops, n):
    """Values of one block 2^30 times another's, keys from nothing to dominating."""
    rng = np.random.default_rng(n)
    c, table = make(rng, [400], 16, 1, 64)
    c.v_scale[:] = np.exp2(rng.integers(-25, 6, c.v_scale.shape)).astype(np.float32)
    c.k_scale[:] = np.exp2(rng.integers(-12, -4, c.k_scale.shape)).astype(np.float32)
    q = cuda(rng.normal(size=(n, 2, 64)), torch.bfloat16)
    out, lse = ops.kv_attention(on_gpu(ops, c), cuda(table), torch.tensor([400], dtype=torch.int32, device="cuda"), q, return_lse=True)
    want, wl, spread, slack = O.attention(c, table, [400], [0, n], q.double().cpu().numpy(), O.default_scale(64), True)
    # (weights times their block's scale are what is rounded: the floor is 2^-25 of the largest value's contribution)
    compare_attention(out, lse, want, wl, spread, slack, "bf16", 400, spread.max(axis=2, keepdims=True) + 127 * 32 * 2.0 ** -25)


@pytest.mark.parametrize("n", [1, 150])
def test_attention_rows_do_not_touch_one_another(ops, n):
    """A row of NaN or infinite queries leaves the other rows' results as they are."""
    rng = np.random.default_rng(2)
    c, table = make(rng, [300, 200], 32, 2, 128)
    gpu, lens = on_gpu(ops, c), torch.tensor([300, 200], dtype=torch.int32, device="cuda")
    q = cuda(rng.normal(size=(2 * n, 8, 128)), torch.bfloat16)
    clean = ops.kv_attention(gpu, cuda(table), lens, q)
    q[0, 1, 5], q[n, 3, 0], q[n, 4] = float("nan"), float("inf"), 0
    got = ops.kv_attention(gpu, cuda(table), lens, q)
    keep = torch.ones(2 * n, 8, dtype=torch.bool, device="cuda")
    keep[0, 1] = keep[n, 3] = keep[n, 4] = False
    assert torch.equal(got[keep], clean[keep])
    assert bool(got[0, 1].isnan().all()) and bool(got[n, 3].isnan().any()) and bool(got[n, 4].isfinite().all())


@pytest.mark.parametrize("n", [1, 150])
def test_attention_ignores_what_lies_past_a_sequence(ops, n):
    """Codes in slots past the length, other pages and table entries past the last page do not matter."""
    rng = np.random.default_rng(6)
    lens = [n + 37, n + 3]
    c, table = make(rng, lens, 64, 2, 64)
    q, tl = cuda(rng.normal(size=(2 * n, 4, 64)), torch.float16), cuda(np.array(lens, np.int32))
    a = ops.kv_attention(on_gpu(ops, c), cuda(table), tl, q)
    for b, m in enumerate(lens):
        last = table[b, (m - 1) // 64]
        c.k[last, :, (m - 1) % 64 + 1:] = 127
        c.v[last, :, (m - 1) % 64 + 1:] = -128
    wide = np.concatenate([table, np.full((2, 5), 2 ** 30, np.int32)], 1)
    assert torch.equal(a, ops.kv_attention(on_gpu(ops, c), cuda(wide), tl, q))


@pytest.mark.parametrize("n", [1, 150])
def test_attention_bad_pages_are_masked(ops, n):
    rng = np.random.default_rng(7)
    c, table = make(rng, [400], 32, 1, 64)
    q, tl = cuda(rng.normal(size=(n, 2, 64)), torch.bfloat16), torch.tensor([400], dtype=torch.int32, device="cuda")
    bad = table.copy()
    bad[0, 2], bad[0, 5] = -7, len(c.k)
    out, lse = ops.kv_attention(on_gpu(ops, c), cuda(bad), tl, q, return_lse=True)
    assert F.fxpq_get_device_status() == L.ERR_RANGE
    # what is left: the same keys without those two pages, which all lie before the rows' own positions
    keep = [i for i in range(table.shape[1]) if i not in (2, 5)]
    want, wl, spread, slack = O.attention(c, table[:, keep], [400 - 64], [0, n], q.double().cpu().numpy(), O.default_scale(64), True)
    compare_attention(out, lse, want, wl, spread, slack, "bf16", 400, np.abs(c.v).max() * c.v_scale.max())


def test_long_pools_pass_32_bit_offsets(ops):
    """Pages past 2^31 bytes of codes: appended, read back and attended to."""
    page, heads, dim = 128, 8, 128
    n = (1 << 31) // (page * heads * dim) + 40
    gpu = ops.KVCache.empty(n, heads, page, dim)
    rng = np.random.default_rng(9)
    ids = np.array([[n - 1, n - 30, n - 7]], np.int32)
    small, _ = make(rng, [300], page, heads, dim, spare=0)
    tab = np.array([[0, 1, 2]], np.int32)
    for name in ("k", "v", "k_scale", "v_scale"):
        getattr(gpu, name)[torch.from_numpy(ids[0]).long().cuda()] = cuda(getattr(small, name))
    x = rng.normal(size=(2, 3 * heads, dim)).astype(np.float32)
    lens = torch.tensor([302], dtype=torch.int32, device="cuda")
    ops.kv_append(gpu, cuda(ids), lens, cuda(x[:, heads:2 * heads]), cuda(x[:, 2 * heads:]))
    O.append(small, tab, [302], [0, 2], x[:, heads:2 * heads], x[:, 2 * heads:])
    k, v = ops.kv_values(gpu, cuda(ids[0]), torch.float32)
    assert np.array_equal(k.cpu().numpy(), small.k.astype(np.float32) * small.k_scale[:, :, None, None])
    assert np.array_equal(v.cpu().numpy(), small.v.astype(np.float32) * small.v_scale[:, :, None, None])
    for rows in (2, 200):
        q = cuda(rng.normal(size=(rows, heads, dim)), torch.bfloat16)
        out, lse = ops.kv_attention(gpu, cuda(ids), lens, q, return_lse=True)
        want, wl, spread, slack = O.attention(small, tab, [302], [0, rows], q.double().cpu().numpy(), O.default_scale(dim), True)
        compare_attention(out, lse, want, wl, spread, slack, "bf16", 302, 127 * small.v_scale.max())


def test_attention_is_deterministic_on_any_stream(ops):
    rng = np.random.default_rng(11)
    c, table = make(rng, [6000, 10], 64, 2, 128)
    gpu, t, lens = on_gpu(ops, c), cuda(table), torch.tensor([6000, 10], dtype=torch.int32, device="cuda")
    q = cuda(rng.normal(size=(2, 8, 128)), torch.bfloat16)
    first = ops.kv_attention(gpu, t, lens, q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = [ops.kv_attention(gpu, t, lens, q) for _ in range(3)]
    side.synchronize()
    assert all(torch.equal(first, s) for s in second)


def test_append_and_attention_in_a_graph(ops):
    """A captured decoding step replayed with other lengths and rows."""
    rng = np.random.default_rng(12)
    page, hq, hkv, dim, B = 32, 4, 2, 64, 3
    c, table = make(rng, [200] * B, page, hkv, dim)
    gpu, t = on_gpu(ops, c), cuda(table)
    cos, sin = O.rope_tables(200, dim)
    gcos, gsin = cuda(cos), cuda(sin)
    lens, x = torch.full((B,), 1, dtype=torch.int32, device="cuda"), torch.zeros(B, hq + 2 * hkv, dim, device="cuda", dtype=torch.bfloat16)

    def step():
        q = ops.kv_append(gpu, t, lens, x[:, hq:hq + hkv], x[:, hq + hkv:], q=x[:, :hq], cos=gcos, sin=gsin)
        return ops.kv_attention(gpu, t, lens, q, return_lse=True)
    saved = [a.clone() for a in (gpu.k, gpu.v, gpu.k_scale, gpu.v_scale)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = step()
    for a, b in zip((gpu.k, gpu.v, gpu.k_scale, gpu.v_scale), saved):
        a.copy_(b)
    for n in ([1, 50, 199], [2, 51, 200], [33, 52, 7]):
        vals = cuda(rng.normal(size=x.shape), torch.bfloat16)
        x.copy_(vals)
        lens.copy_(torch.tensor(n, dtype=torch.int32))
        graph.replay()
        f = vals.float().cpu().numpy()
        rq = O.append(c, table, n, [0, 1, 2, 3], f[:, hq:hq + hkv], f[:, hq + hkv:], f[:, :hq], cos, sin, False)
        same_cache(gpu, c)
        rq = torch.from_numpy(rq).bfloat16().double().numpy()
        want, wl, spread, slack = O.attention(c, table, n, [0, 1, 2, 3], rq, O.default_scale(dim), True)
        compare_attention(out, lse, want, wl, spread, slack, "bf16", 200, np.abs(c.v).max() * c.v_scale.max())


# ------------------------------------------------------------------------------ refusals of the Python layer
def test_python_refusals(ops):
    x = torch.zeros(4, 2, 64, device="cuda")
    c = ops.KVCache.empty(4, 2, 16, 64)
    pages, lens = torch.zeros(4, 1, dtype=torch.int32, device="cuda"), torch.ones(4, dtype=torch.int32, device="cuda")
    for call, err in [
            (lambda: ops.quantize_tokens(torch.zeros(3, 4)), ValueError),
            (lambda: ops.quantize_tokens(torch.zeros(3, 4, device="cuda", dtype=torch.int32)), TypeError),
            (lambda: ops.linear_i8(x[:, 0].to(torch.int8), lens.float(), x[:, 0, :60].to(torch.int8), lens.float()), ValueError),
            (lambda: ops.linear_i8(x[:, 0].to(torch.int8), lens.float()[:2], x[:, 0].to(torch.int8), lens.float()), ValueError),
            (lambda: ops.KVCache(c.k, c.v, c.k_scale, c.v_scale[:2]), ValueError),
            (lambda: ops.KVCache(c.k.float(), c.v, c.k_scale, c.v_scale), ValueError),
            (lambda: ops.KVCache.empty(2, 2, 24, 64) and ops.kv_values(ops.KVCache.empty(2, 2, 24, 64), lens), L.FxpqError),
            (lambda: ops.kv_append(c, pages, lens, x, x[:, :1]), ValueError),
            (lambda: ops.kv_append(c, pages, lens, x, x.half()), TypeError),
            (lambda: ops.kv_append(c, pages, lens.long(), x, x), ValueError),
            (lambda: ops.kv_append(c, pages[:3], lens, x, x), ValueError),
            (lambda: ops.kv_append(c, pages, lens, x[:3], x[:3]), ValueError),
            (lambda: ops.kv_append(c, pages, lens, x, x, cos=x[0]), ValueError),
            (lambda: ops.kv_append(c, pages, lens, x, x, starts=lens), ValueError),
            (lambda: ops.kv_attention(c, pages, lens, x), TypeError),
            (lambda: ops.kv_attention(c, pages, lens, x[:, :1].half()), ValueError),
            (lambda: ops.kv_attention(c, pages, lens, x.half(), scale=0.0), L.FxpqError),
            (lambda: ops.kv_attention(c, pages, lens, x.half()[:, :, ::2]), ValueError)]:
        with pytest.raises(err):
            call()
    assert math.isfinite(ops.kv_attention(c, pages, lens, x.half()).sum().item())
