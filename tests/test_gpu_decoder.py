"""The 8-bit decoder that runs the language-model operators together."""
import numpy as np
import pytest
import torch

from oracle import llm as O
from paper_2203_12091_gb300 import _lib as L
from paper_2203_12091_gb300 import fxpq as F

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def decoder():
    import __graft_entry__ as g
    g.build()
    from paper_2203_12091_gb300 import decoder
    return decoder


def rms(x, w):
    f = x.astype(np.float64)
    return f / np.sqrt((f * f).mean(-1, keepdims=True) + 1e-5) * w


def bf(x):
    return torch.from_numpy(np.asarray(x, dtype=np.float64)).bfloat16().double().numpy()


def linear(layer, x):
    """The layer's definition on the oracle's side, rounded to bfloat16 like the activations in between."""
    c, s = O.quantize_tokens(x.astype(np.float32))
    return bf(O.linear(c, s, layer.w.cpu().numpy(), layer.w_scale.cpu().numpy())[0])


def oracle_layer(layer, cache, x, pages, lens, starts, cos, sin):
    T, h, g, d = len(x), layer.heads, layer.kv_heads, layer.dim
    qkv = linear(layer.qkv, bf(rms(x, 1.0))).reshape(T, h + 2 * g, d).astype(np.float32)
    q = O.append(cache, pages, lens, starts, qkv[:, h:h + g], qkv[:, h + g:], qkv[:, :h], cos, sin, False)
    a = O.attention(cache, pages, lens, starts, bf(q), O.default_scale(d), True)[0]
    x = bf(x + linear(layer.out, bf(a).reshape(T, h * d)))
    gate, up = np.split(linear(layer.gate_up, bf(rms(x, 1.0))), 2, -1)
    return bf(x + linear(layer.down, bf(bf(gate / (1 + np.exp(-gate))) * up)))


def test_layer_against_the_oracle(decoder):
    """A ragged batch of prompts, then two single-token steps, through one layer.  The two sides round the same numbers to
    bfloat16 at other places of their sums and so differ by some activations' code: a code is 1 / 127 of its row's largest
    value, some 2^-5 of a typical one, so 2% of the output's norm leaves room for half of them to differ by one."""
    m = decoder.Decoder(vocab=50, width=256, layers=1, heads=4, kv_heads=2, dim=64, hidden=384, max_seqs=3, max_tokens=100, page=16, seed=3)
    layer, rng = m.layers[0], np.random.default_rng(0)
    c = layer.cache
    oc = O.Cache(*[t.cpu().numpy() for t in (c.k, c.v, c.k_scale, c.v_scale)])
    pages, cos, sin = m.pages.cpu().numpy(), m.cos.cpu().numpy(), m.sin.cpu().numpy()
    lens = np.array([37, 5, 16], np.int32)
    for news in ([37, 5, 16], [1, 1, 1], [1, 1, 1]):
        starts = np.concatenate([[0], np.cumsum(news)]).astype(np.int32)
        x = bf(rng.normal(size=(sum(news), 256)))
        got = layer(torch.from_numpy(x).bfloat16().cuda(), m.pages, torch.from_numpy(lens).cuda(),
                    torch.from_numpy(starts).cuda() if sum(news) > 3 else None, m.cos, m.sin).double().cpu().numpy()
        want = oracle_layer(layer, oc, x, pages, lens, starts, cos, sin)
        assert np.linalg.norm(got - want) <= 0.02 * np.linalg.norm(want - x)
        lens = lens + 1
    assert F.fxpq_get_device_status() == L.OK


def test_generation_continues_its_prompts(decoder):
    m = decoder.Decoder(seed=1, max_seqs=4, max_tokens=200)
    prompts = [[3, 1, 4, 1, 5], [9] * 33, list(range(64)), [2]]
    a = m.generate(prompts, 12)
    assert a.shape == (4, 12) and int(a.min()) >= 0 and int(a.max()) < 1000
    assert torch.equal(a, decoder.Decoder(seed=1, max_seqs=4, max_tokens=200).generate(prompts, 12))  # the same from an empty cache
    # one sequence alone in the batch decodes what it decodes among others, but for rounding to other codes: its first token
    alone = decoder.Decoder(seed=1, max_seqs=4, max_tokens=200).generate(prompts[:1], 1)
    assert torch.equal(alone[0], a[0, :1])
    with pytest.raises(ValueError):
        m.generate([[1] * 200], 1)
    assert F.fxpq_get_device_status() == L.OK
