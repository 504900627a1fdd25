"""The 8-bit decoder whose norms, gates and residual sums are parts of its layers' kernels, against the 64-bit oracle and against the
form that leaves them to torch."""
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


def bf(x):
    return torch.from_numpy(np.asarray(x, dtype=np.float64)).bfloat16().double().numpy()


def normed(layer, x, weight):
    """z of a layer under a norm, by the definition."""
    c, s = O.norm_codes(x.astype(np.float32), weight.cpu().numpy(), 1e-5)
    return O.layer_sums(c, layer.w.cpu().numpy())[0] * s[:, None] * layer.w_scale.double().cpu().numpy()


def plain(layer, x):
    c, s = O.quantize_tokens(x.astype(np.float32))
    return O.layer_sums(c, layer.w.cpu().numpy())[0] * s.astype(np.float64)[:, None] * layer.w_scale.double().cpu().numpy()


def oracle_layer(layer, cache, x, pages, lens, starts, cos, sin):
    T, h, g, d = len(x), layer.heads, layer.kv_heads, layer.dim
    qkv = bf(normed(layer.qkv, x, layer.norm1)).reshape(T, h + 2 * g, d).astype(np.float32)
    q = O.append(cache, pages, lens, starts, qkv[:, h:h + g], qkv[:, h + g:], qkv[:, :h], cos, sin, False)
    a = O.attention(cache, pages, lens, starts, bf(q), O.default_scale(d), True)[0]
    x = bf(x + plain(layer.out, bf(a).reshape(T, h * d)))
    return bf(x + plain(layer.down, bf(O.gated(normed(layer.gate_up, x, layer.norm2), "silu"))))


def test_layer_against_the_oracle(decoder):
    """A ragged batch of prompts, then two single-token steps.  As for the other form, 2% of what the layer adds leaves room for
    activations whose code differs by one."""
    m = decoder.Decoder(vocab=50, width=256, layers=1, heads=4, kv_heads=2, dim=64, hidden=384, max_seqs=3, max_tokens=100, page=16, seed=3, fused=True)
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


def test_both_forms_have_the_same_weights_and_close_logits(decoder):
    """Their activations round to bfloat16 at other places: 2^-9 of a value each time, some ten times a layer, and codes that then differ
    by one (1 / 127 of a row's largest value): 5% of the logits' norm leaves room for all of it."""
    models = [decoder.Decoder(seed=1, max_seqs=2, max_tokens=100, fused=f) for f in (False, True)]
    gate, up = models[0].layers[1].gate_up.w.chunk(2)
    assert torch.equal(models[1].layers[1].gate_up.w[::2], gate) and torch.equal(models[1].layers[1].gate_up.w[1::2], up)
    tokens = torch.arange(60, device="cuda")
    lens = torch.tensor([30, 30], dtype=torch.int32, device="cuda")
    a, b = (m.forward(tokens, lens) for m in models)
    assert (a - b).norm() <= 0.05 * a.norm()
    assert F.fxpq_get_device_status() == L.OK


def test_generation(decoder):
    prompts = [[3, 1, 4, 1, 5], [9] * 33, list(range(64)), [2]]
    a = decoder.Decoder(seed=1, max_seqs=4, max_tokens=200, fused=True).generate(prompts, 12)
    assert a.shape == (4, 12) and int(a.min()) >= 0 and int(a.max()) < 1000
    assert torch.equal(a, decoder.Decoder(seed=1, max_seqs=4, max_tokens=200, fused=True).generate(prompts, 12))
    assert F.fxpq_get_device_status() == L.OK


def test_a_captured_step(decoder):
    """A single-token step of the whole decoder in a graph, replayed as lengths grow."""
    m = decoder.Decoder(seed=2, max_seqs=3, max_tokens=100, fused=True)
    twin = decoder.Decoder(seed=2, max_seqs=3, max_tokens=100, fused=True)
    tokens, lens = torch.tensor([5, 6, 7], device="cuda"), torch.ones(3, dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        m.forward(tokens, lens)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = m.forward(tokens, lens)
    for step in range(1, 5):
        tokens.copy_(torch.tensor([step, 2 * step, 3 * step], device="cuda"))
        lens.fill_(step)
        g.replay()
        assert torch.equal(out, twin.forward(tokens, lens))
    assert F.fxpq_get_device_status() == L.OK
