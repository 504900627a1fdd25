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
