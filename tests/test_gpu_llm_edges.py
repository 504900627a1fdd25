"""The language-model operators where their numbers or arguments are extreme: long caches with few keys that matter, queries
near the ends of their type, tables without pages, rows that share memory, tensors that want a gradient."""
import math

import numpy as np
import pytest
import torch

from oracle import llm as O
from paper_2203_12091_gb300 import _lib as L
from paper_2203_12091_gb300 import fxpq as F

pytestmark = pytest.mark.gpu


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


def ints(*a):
    return torch.tensor(a, dtype=torch.int32, device="cuda")


# ------------------------------------------------------------------------------ attention: the range of the weights
@pytest.mark.parametrize("seqs,n", [(512, 1), (152, 40), (1, 38912)])  # few rows, a block of rows, codes expanded before
def test_attention_keeps_the_small_weights_of_a_long_cache(ops, seqs, n):
    """2^20 keys, four of them (in the first four tiles) with 2^26.5 times the weight of any other and values of zero: the result
    is what the others add, 2^20 2^-26.5 / 4 of their value."""
    page, dim, keys, gap = 128, 64, 1 << 20, 26.5
    c = ops.KVCache.empty(keys // page, 1, page, dim)
    c.k_scale.fill_(2.0 ** -4)
    c.v_scale.fill_(2.0 ** -6)
    c.v.fill_(64)  # 1
    for t in (0, 32, 64, 96):
        c.k[0, 0, t, 0], c.v[0, 0, t] = 127, 0
    pages = torch.arange(keys // page, dtype=torch.int32, device="cuda").repeat(seqs, 1)
    q = torch.zeros(seqs * n, 1, dim, dtype=torch.float16, device="cuda")
    q[..., 0] = 1
    out, lse = ops.kv_attention(c, pages, torch.full((seqs,), keys, dtype=torch.int32, device="cuda"), q,
                                scale=gap * math.log(2) / (127 / 16), causal=False, return_lse=True)
    total = 4 * 2.0 ** gap + keys - 4
    want = (keys - 4) / total
    # a small weight is at least 2^-20.5 (the largest lie between 2^6 and 2^7), a step of fp16 there 2^-24; and 2^-8 for the
    # normaliser, where fp32 may lose what the small ones add to it, and the output's own rounding
    assert (out.double() - want).abs().max().item() <= want * (2.0 ** -4.5 + 2.0 ** -8)
    assert (lse.double() - math.log(total)).abs().max().item() <= 2.0 ** -8


# ------------------------------------------------------------------------------ attention: queries near the ends of their type
@pytest.mark.parametrize("n", [1, 150])
@pytest.mark.parametrize("power", [100, 115, 120, -90, -105, -112])
def test_attention_of_huge_and_tiny_queries(ops, n, power):
    """Queries times 2^p under a scale of 2^-p: the same numbers, scaled exactly, so the same results."""
    rng = np.random.default_rng(n)
    c, table = O.paged(rng, [300, 200], 32, 2, 64)
    gpu = ops.KVCache(*[torch.from_numpy(t).cuda() for t in (c.k, c.v, c.k_scale, c.v_scale)])
    q = rng.normal(size=(2 * n, 8, 64))
    q = torch.from_numpy(np.copysign(np.maximum(np.abs(q), 2.0 ** -8), q)).bfloat16().cuda()  # (none becomes subnormal)
    args = gpu, torch.from_numpy(table).cuda(), ints(300, 200)
    want = ops.kv_attention(*args, q, scale=0.125, return_lse=True)
    got = ops.kv_attention(*args, (q.double() * 2.0 ** power).bfloat16(), scale=0.125 * 2.0 ** -power, return_lse=True)
    assert bool(want[0].isfinite().all()) and torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("n", [1, 150])
@pytest.mark.parametrize("large", [32768.0, 65504.0])
def test_attention_keeps_every_bit_of_float16_queries(ops, n, large):
    """A row's largest value past 2^15, the others with their last bit at 2^-24, float16's smallest step: scores of 63 of the small
    ones alone, whose last bits are 2^-10 of them."""
    dim, small = 64, (1 + 2.0 ** -10) * 2.0 ** -14
    c = ops.KVCache.empty((n + 15) // 16, 1, 16, dim)
    c.k.fill_(100)
    c.k[..., 0] = 0
    q = torch.full((n, 1, dim), small, dtype=torch.float16, device="cuda")
    q[..., 0] = large
    score = 50.0
    lse = ops.kv_attention(c, torch.arange((n + 15) // 16, dtype=torch.int32, device="cuda")[None], ints(n), q,
                           scale=score / (63 * 100 * small), causal=False, return_lse=True)[1]
    # 63 products summed in fp32, log2(e) * scale and its product with the sum rounded, log2 and its way back: 2^-18 is ample
    assert (lse.double() - score - math.log(n)).abs().max().item() <= 50 * 2.0 ** -18


# ------------------------------------------------------------------------------ attention: tables
@pytest.mark.parametrize("n", [1, 40, 2100])  # few rows, a block of rows, codes expanded before
def test_attention_over_a_table_without_pages(ops, n):
    c = ops.KVCache.empty(3, 1, 16, 64)
    q = torch.randn(2 * n, 1, 64, device="cuda").half()
    pages, lens = torch.empty((2, 0), dtype=torch.int32, device="cuda"), ints(0, 0)
    out, lse = ops.kv_attention(c, pages, lens, q, return_lse=True)
    assert not bool(out.any()) and bool((lse == -math.inf).all())


def test_attention_of_sequences_that_share_their_row_of_pages(ops):
    rng = np.random.default_rng(21)
    c, table = O.paged(rng, [100], 16, 1, 64)
    gpu = ops.KVCache(*[torch.from_numpy(t).cuda() for t in (c.k, c.v, c.k_scale, c.v_scale)])
    pages, lens, q = torch.from_numpy(table).cuda(), ints(100, 100, 100), torch.from_numpy(rng.normal(size=(3, 2, 64))).half().cuda()
    want = ops.kv_attention(gpu, pages.repeat(3, 1), lens, q)
    assert torch.equal(ops.kv_attention(gpu, pages.expand(3, -1), lens, q), want)


# ------------------------------------------------------------------------------ rows that share memory
@pytest.mark.parametrize("rows", ["expanded", "windows"])
def test_rows_that_share_memory(ops, rows):
    x = torch.randn(1, 96, device="cuda").expand(5, -1) if rows == "expanded" else torch.randn(150, device="cuda").unfold(0, 96, 3)
    codes, scale = ops.quantize_tokens(x)
    want = ops.quantize_tokens(x.clone(memory_format=torch.contiguous_format))
    assert torch.equal(codes, want[0]) and torch.equal(scale, want[1])
    layer = ops.Linear8.from_float(torch.randn(40, 96, device="cuda"))
    assert torch.equal(layer(x), layer(x.clone(memory_format=torch.contiguous_format)))


# ------------------------------------------------------------------------------ gradients
def test_tensors_that_want_a_gradient_are_refused(ops):
    """The operators have no gradient: a result without one, and no word of it, would leave a model untrained."""
    c = ops.KVCache.empty(4, 2, 16, 64)
    pages, lens = ints(0, 1, 2, 3)[:, None], ints(1, 1, 1, 1)
    x = torch.randn(4, 2, 64, device="cuda").half()
    g = x.clone().requires_grad_()
    w, b = torch.nn.Parameter(torch.randn(40, 128, device="cuda")), torch.nn.Parameter(torch.randn(40, device="cuda"))
    layer = ops.Linear8.from_float(w, b)  # (a layer's own weights are constants)
    flat = g.view(4, 128)
    codes, scale = ops.quantize_tokens(x.view(4, 128))
    calls = [lambda: ops.quantize_tokens(flat), lambda: layer(flat),
             lambda: ops.linear_i8(codes, scale, layer.w, layer.w_scale, b),
             lambda: ops.linear_i8(codes, scale.clone().requires_grad_(), layer.w, layer.w_scale),
             lambda: ops.kv_append(c, pages, lens, g, x), lambda: ops.kv_append(c, pages, lens, x, g),
             lambda: ops.kv_append(c, pages, lens, x, x, q=g), lambda: ops.kv_attention(c, pages, lens, g)]
    for call in calls:
        with pytest.raises(RuntimeError, match="gradient"):
            call()
        with torch.no_grad():
            call()
    y = layer(x.view(4, 128))
    assert not y.requires_grad and not layer.bias.requires_grad and not layer.w_scale.requires_grad
    assert not ops.Linear8(layer.w.contiguous(), layer.w_scale, b)(x.view(4, 128)).requires_grad


@pytest.mark.parametrize("n", [1, 150])
def test_attention_of_scores_that_are_steps_of_fp32_apart(ops, n):
    """Scores near 2^27, where fp32 has steps of 16 between their exponents of two, growing by one or two from a warp's tile to its next:
    the result is a mean of values between 0.5 and 1 all the same."""
    pages, page = 160, 16
    c = ops.KVCache.empty(pages, 1, page, 64)
    c.k[..., 0] = 100
    c.k_scale[:, 0] = torch.from_numpy((2.0 ** -4 * (1 + np.arange(pages) // 8 * 2.0 ** -23)).astype(np.float32)).cuda()
    c.v.copy_(torch.randint(64, 129, c.v.shape, device="cuda").clamp(max=127))
    c.v_scale.fill_(2.0 ** -7)
    q = torch.zeros(n, 1, 64, dtype=torch.float16, device="cuda")
    q[..., 0] = 1
    out, lse = ops.kv_attention(c, torch.arange(pages, dtype=torch.int32, device="cuda")[None], ints(pages * page), q,
                                scale=1.5 * 2 ** 27 * math.log(2) / 6.25, causal=False, return_lse=True)
    assert bool(lse.isfinite().all()) and 0.5 * (1 - 2.0 ** -10) <= out.min().item() <= out.max().item() <= 1 + 2.0 ** -10
