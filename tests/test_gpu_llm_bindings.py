"""The binding's entry points of the language-model operators (the header's names) give what the operators give."""
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
    return llm


def test_linear_tokens(ops):
    torch.manual_seed(0)
    layer = ops.Linear8.from_float(torch.randn(70, 90, device="cuda"), torch.randn(70, device="cuda"))
    x, y = torch.randn(33, 90, device="cuda").half(), torch.empty(33, 70, device="cuda")
    ws = torch.empty(F.fxpq_linear_tokens_workspace(33, 70, 90), dtype=torch.uint8, device="cuda")
    F.fxpq_linear_tokens(x, L.FT_F16, 90, layer.w, 96, layer.w_scale, layer.bias, 33, 70, 90, L.FT_F32, y, 70, ws)
    assert torch.equal(y, layer(x, torch.float32))
    with pytest.raises(L.FxpqError):
        F.fxpq_linear_tokens(x, L.FT_F16, 90, layer.w, 96, layer.w_scale, layer.bias, 33, 70, 90, L.FT_F32, y, 70, ws[:256])


def test_cache(ops):
    rng = np.random.default_rng(0)
    c, table = O.paged(rng, [3000, 70], 32, 2, 64)
    caches = [ops.KVCache(*[torch.from_numpy(t).cuda() for t in (c.k, c.v, c.k_scale, c.v_scale)]) for _ in range(2)]
    pages, lens = torch.from_numpy(table).cuda(), torch.tensor([3000, 70], dtype=torch.int32, device="cuda")
    x = torch.from_numpy(rng.normal(size=(2, 8, 64))).half().cuda()
    cos, sin = (torch.from_numpy(t).cuda() for t in O.rope_tables(3000, 64))
    batch = L.KVBatchDesc(pages.data_ptr(), lens.data_ptr(), None, 2, table.shape[1], 2, 0, table.shape[1])
    rows = [L.KVRows(t.data_ptr(), 512, 64) for t in (x[:, 4:6], x[:, 6:], x)]
    want = ops.kv_append(caches[0], pages, lens, x[:, 4:6], x[:, 6:], q=x[:, :4], cos=cos, sin=sin)
    q = torch.empty_like(want)
    F.fxpq_kv_append(caches[1].desc, batch, L.FT_F16, rows[0], rows[1], rows[2], 4, q, cos, sin, 3000, 64, 0)
    assert torch.equal(q, want) and all(torch.equal(getattr(caches[0], n), getattr(caches[1], n)) for n in ("k", "v", "k_scale", "v_scale"))
    ids = torch.tensor([3, 0], dtype=torch.int32, device="cuda")
    k, v = (torch.empty(2, 2, 32, 64, device="cuda") for _ in range(2))
    F.fxpq_kv_values(caches[1].desc, ids, 2, L.FT_F32, k, v)
    want_k, want_v = ops.kv_values(caches[0], ids, torch.float32)
    assert torch.equal(k, want_k) and torch.equal(v, want_v)
    out, lse = torch.empty_like(q), torch.empty(2, 4, device="cuda")
    need = F.fxpq_kv_attention_workspace(caches[1].desc, batch, 4)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    assert need > 0
    F.fxpq_kv_attention(caches[1].desc, batch, L.FT_F16, L.KVRows(q.data_ptr(), 256, 64), 4, 0.125, 1, out, lse, ws)
    a, b = ops.kv_attention(caches[0], pages, lens, q, return_lse=True)
    assert torch.equal(out, a) and torch.equal(lse, b)
    assert F.fxpq_get_device_status() == L.OK
