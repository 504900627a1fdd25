"""Arguments that the C entry points of the language-model operators must refuse before they launch anything, because a kernel
would read or write through them."""
import ctypes

import pytest

from paper_2203_12091_gb300 import _lib as L
from paper_2203_12091_gb300 import build as B

P = ctypes.c_void_p(4096)


@pytest.fixture(scope="module")
def lib():
    B.build()
    return L.lib()


def test_rows_of_nothing_but_padding_need_memory_for_it(lib):
    """Codes K .. codes_stride - 1 are zeroed, so rows without values still write."""
    def call(codes, stride, K=0):
        return lib.fxpq_quantize_tokens(P, L.FT_F32, 2, K, 64, codes, stride, P, None)
    assert call(None, 16) == L.ERR_INVALID_ARG
    assert call(None, 1) == L.ERR_INVALID_ARG
    assert call(None, 64, K=64) == L.ERR_INVALID_ARG


@pytest.mark.parametrize("off", [1, 2, 3])
def test_misaligned_integers_and_scales(lib, off):
    bad = 4096 + off
    rows = L.KVRows(4096, 128, 64)

    def cache(**kw):
        a = {**dict(k=4096, v=4096, ks=4096, vs=4096), **kw}
        return L.KVCacheDesc(a["k"], a["v"], a["ks"], a["vs"], 4, 16, 2, 64)

    def batch(**kw):
        a = {**dict(pages=4096, lens=4096, starts=None), **kw}
        return L.KVBatchDesc(a["pages"], a["lens"], a["starts"], 2, 3, 4, 0, 3)

    def append(c, b):
        return lib.fxpq_kv_append(ctypes.byref(c), ctypes.byref(b), L.FT_BF16, ctypes.byref(rows), ctypes.byref(rows), None, 0, None, None, None,
                                  0, 0, 0, None)

    def attend(c, b):
        n = lib.fxpq_kv_attention_workspace(ctypes.byref(c), ctypes.byref(b), 4)
        return lib.fxpq_kv_attention(ctypes.byref(c), ctypes.byref(b), L.FT_BF16, ctypes.byref(rows), 4, 0.1, 1, P, None, P, n, None)
    for c in (cache(ks=bad), cache(vs=bad)):
        assert append(c, batch()) == attend(c, batch()) == L.ERR_INVALID_ARG
        assert lib.fxpq_kv_values(ctypes.byref(c), P, 1, L.FT_F32, P, P, None) == L.ERR_INVALID_ARG
    for b in (batch(pages=bad), batch(lens=bad), batch(starts=bad)):
        assert append(cache(), b) == attend(cache(), b) == L.ERR_INVALID_ARG
    assert lib.fxpq_kv_values(ctypes.byref(cache()), ctypes.c_void_p(bad), 1, L.FT_F32, P, P, None) == L.ERR_INVALID_ARG
