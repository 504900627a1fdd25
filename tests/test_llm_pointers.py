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
