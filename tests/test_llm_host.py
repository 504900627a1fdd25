"""The 8-bit language-model operators without a GPU: the oracle against hand-worked values, and every refusal
of the C entry points (which return before any launch)."""
import ctypes
from fractions import Fraction

import numpy as np
import pytest

from oracle import llm as O
from paper_2203_12091_gb300 import _lib as L
from paper_2203_12091_gb300 import build as B

P = ctypes.c_void_p(4096)
ODD = ctypes.c_void_p(4097)


@pytest.fixture(scope="module")
def lib():
    B.build()
    return L.lib()


# ------------------------------------------------------------------------------ the oracle
def test_oracle_token_codes_by_hand():
    codes, scale = O.quantize_tokens(np.array([[127.0, -63.5, 0.5, 1.5], [0, 0, 0, 0], [-254.0, 1.0, 3.0, np.inf]]))
    assert codes[0].tolist() == [127, -64, 0, 2]  # ties to even: -63.5 -> -64, 0.5 -> 0, 1.5 -> 2
    assert scale[0] == np.float32(127) * (np.float32(1) / np.float32(127)) and scale[1] == 0 and not codes[1].any()
    assert codes[2].tolist()[0] == -127 and codes[2, 3] == 0


@pytest.mark.parametrize("a,fl", [(127.0, 0), (127.0000076, -1), (63.5, 1), (1.0, 6), (0.0, 40), (1e30, -32), (2.0 ** -60, 40),
                                  (0.9921875, 7), (0.99218756, 6)])
def test_oracle_block_scale(a, fl):
    assert O.block_scale(np.float32(a)) == 2.0 ** -fl


def test_oracle_rotation_is_a_rotation():
    rng = np.random.default_rng(0)
    x = rng.normal(size=(3, 64)).astype(np.float32)
    cos, sin = O.rope_tables(50, 32)
    for inter in (False, True):
        y = O.rotate(x, 49, cos, sin, 32, inter)
        assert np.array_equal(y[:, 32:], x[:, 32:])
        np.testing.assert_allclose((y.astype(np.float64) ** 2).sum(1), (x.astype(np.float64) ** 2).sum(1), rtol=1e-5)
        assert np.array_equal(O.rotate(x, 0, cos, sin, 32, inter), x)
    # a unit vector in the first place turns to (cos, sin) in its pair's places
    e = np.zeros(64, np.float32)
    e[0] = 1
    assert O.rotate(e, 7, cos, sin, 32, False)[16] == sin[7, 0] and O.rotate(e, 7, cos, sin, 32, True)[1] == sin[7, 0]


def test_oracle_growing_block_rounds_older_codes_to_even():
    c = O.Cache(*[np.zeros((1, 1, 16, 64), np.int8)] * 2, *[np.ones((1, 1), np.float32)] * 2)
    x = np.zeros((1, 1, 64), np.float32)
    x[0, 0, :4] = [5, 3, 1, 127]
    O.append(c, [[0]], [1], [0, 1], x, x)
    assert c.k_scale[0, 0] == 1 and c.k[0, 0, 0, :4].tolist() == [5, 3, 1, 127]
    y = np.zeros((1, 1, 64), np.float32)
    y[0, 0, 0] = 200
    O.append(c, [[0]], [2], [0, 1], y, y)
    assert c.k_scale[0, 0] == 2 and c.k[0, 0, 0, :4].tolist() == [2, 2, 0, 64] and c.k[0, 0, 1, 0] == 100
    O.append(c, [[0]], [2], [0, 1], y, y)  # again: nothing changes
    assert c.k[0, 0, 0, :4].tolist() == [2, 2, 0, 64] and c.k_scale[0, 0] == 2


def test_oracle_attention_against_fractions():
    # two keys whose scores differ by a power of e that is exact to bound: equal scores give the mean
    c = O.Cache(np.ones((1, 1, 16, 64), np.int8), np.arange(16 * 64).reshape(1, 1, 16, 64) % 100 - 50, np.ones((1, 1)), np.full((1, 1), 0.5))
    q = np.ones((1, 2, 64), np.float32)
    out, lse, _, _ = O.attention(c, [[0]], [5], [0, 1], q, 0.125, True)
    want = [sum(Fraction(int(c.v[0, 0, t, d]), 2) for t in range(5)) / 5 for d in range(64)]
    np.testing.assert_allclose(out[0, 1], [float(w) for w in want], rtol=1e-12, atol=1e-12)
    np.testing.assert_allclose(lse, 64 * 0.125 + np.log(5))
    out, lse, _, _ = O.attention(c, [[0]], [0], [0, 1], q, 0.125, True)
    assert not out.any() and np.all(np.isneginf(lse))


# ------------------------------------------------------------------------------ refusals
def test_quantize_tokens_refuses(lib):
    ok = dict(x=P, t=L.FT_BF16, M=2, K=64, xs=64, c=P, cs=64, s=P)
    bad = [dict(x=None), dict(t=3), dict(t=-1), dict(M=-1), dict(K=-1), dict(xs=63), dict(c=None), dict(cs=63), dict(s=None),
           dict(x=ODD), dict(s=ODD)]
    for b in bad:
        a = {**ok, **b}
        assert lib.fxpq_quantize_tokens(a["x"], a["t"], a["M"], a["K"], a["xs"], a["c"], a["cs"], a["s"], None) == L.ERR_INVALID_ARG, b
    assert lib.fxpq_quantize_tokens(None, L.FT_F32, 0, 64, 64, None, 64, None, None) == L.OK


def test_linear_refuses(lib):
    ok = dict(x=P, xs=64, sx=P, w=P, ws=64, sw=P, b=None, M=2, N=3, K=60, t=L.FT_F16, y=P, ys=3)

    def call(**kw):
        a = {**ok, **kw}
        n = lib.fxpq_linear_i8_workspace(a["M"], a["N"], a["K"])
        return lib.fxpq_linear_i8(a["x"], a["xs"], a["sx"], a["w"], a["ws"], a["sw"], a["b"], a["M"], a["N"], a["K"], a["t"],
                                  a["y"], a["ys"], P, n, None)
    for b in [dict(x=None), dict(w=None), dict(sx=None), dict(sw=None), dict(y=None), dict(x=ODD), dict(w=ctypes.c_void_p(4104)), dict(xs=60),
              dict(xs=48), dict(ws=72), dict(ys=2), dict(t=3), dict(M=-1), dict(N=-1), dict(K=-1), dict(b=ODD), dict(y=ODD)]:
        assert call(**b) == L.ERR_INVALID_ARG, b
    assert call(M=0) == L.OK and call(N=0) == L.OK
    for M, N, K in ((1, 4096, 4096), (64, 4096, 25088)):
        n = lib.fxpq_linear_i8_workspace(M, N, K)
        if n:
            for ws, nb in ((None, n), (P, n - 1), (ctypes.c_void_p(4112), n)):
                assert lib.fxpq_linear_i8(P, K, P, P, K, P, None, M, N, K, L.FT_F16, P, N, ws, nb, None) == L.ERR_WORKSPACE


def test_linear_tokens_refuses(lib):
    ok = dict(x=P, t=L.FT_BF16, xs=64, w=P, ws=64, sw=P, b=None, M=2, N=3, K=60, yt=L.FT_F16, y=P, ys=3)

    def call(work=P, short=0, **kw):
        a = {**ok, **kw}
        n = lib.fxpq_linear_tokens_workspace(a["M"], a["N"], a["K"])
        return lib.fxpq_linear_tokens(a["x"], a["t"], a["xs"], a["w"], a["ws"], a["sw"], a["b"], a["M"], a["N"], a["K"], a["yt"], a["y"],
                                      a["ys"], work, n - short, None)
    for b in [dict(x=None), dict(w=None), dict(sw=None), dict(y=None), dict(x=ODD), dict(w=ODD), dict(xs=59), dict(ws=72), dict(ys=2),
              dict(t=3), dict(yt=-1), dict(M=-1), dict(N=-1), dict(K=-1), dict(b=ODD), dict(y=ODD)]:
        assert call(**b) == L.ERR_INVALID_ARG, b
    assert call(work=None) == call(short=1) == call(work=ctypes.c_void_p(4112)) == L.ERR_WORKSPACE
    assert call(M=0) == L.OK and call(N=0) == L.OK


def _cache(**kw):
    a = dict(k=4096, v=4096, ks=4096, vs=4096, n=4, page=16, heads=2, dim=64)
    a.update(kw)
    return L.KVCacheDesc(a["k"], a["v"], a["ks"], a["vs"], a["n"], a["page"], a["heads"], a["dim"])


def _batch(**kw):
    a = dict(pages=4096, lens=4096, starts=None, B=2, wide=3, T=4, stride=3)
    a.update(kw)
    return L.KVBatchDesc(a["pages"], a["lens"], a["starts"], a["B"], a["wide"], a["T"], 0, a["stride"])


BAD_CACHES = [dict(k=None), dict(v=None), dict(ks=None), dict(vs=None), dict(n=0), dict(page=24), dict(page=256), dict(heads=0),
              dict(dim=96), dict(k=4104)]
BAD_BATCHES = [dict(pages=None), dict(lens=None), dict(B=-1), dict(T=-1), dict(T=3), dict(stride=2), dict(wide=-1), dict(B=0)]


def test_append_refuses(lib):
    def call(cache=None, batch=None, t=L.FT_BF16, k=L.KVRows(4096, 128, 64), v=L.KVRows(4096, 128, 64), q=None, qh=0, qo=None, cos=P, sin=P,
             n=10, rot=64, inter=0):
        c, b = cache or _cache(), batch or _batch()
        return lib.fxpq_kv_append(ctypes.byref(c), ctypes.byref(b), t, ctypes.byref(k) if k else None, ctypes.byref(v) if v else None,
                                  ctypes.byref(q) if q else None, qh, qo, cos, sin, n, rot, inter, None)
    for c in BAD_CACHES:
        assert call(cache=_cache(**c)) == L.ERR_INVALID_ARG, c
    for b in BAD_BATCHES:
        assert call(batch=_batch(**b)) == L.ERR_INVALID_ARG, b
    rows = L.KVRows(4096, 128, 64)
    for kw in [dict(t=3), dict(k=None), dict(v=None), dict(k=L.KVRows(None, 1, 1)), dict(k=L.KVRows(4097, 128, 64)), dict(rot=65),
               dict(rot=12), dict(rot=-8), dict(rot=72), dict(cos=None), dict(sin=None), dict(cos=ctypes.c_void_p(4104)), dict(n=-1),
               dict(inter=2), dict(q=rows, qh=0, qo=P), dict(q=rows, qh=2, qo=None), dict(q=rows, qh=2, qo=ctypes.c_void_p(4104))]:
        assert call(**kw) == L.ERR_INVALID_ARG, kw
    assert call(batch=_batch(T=0)) == L.OK
    assert call(batch=_batch(B=0, T=0)) == L.OK


def test_values_refuses(lib):
    c = _cache()
    r = ctypes.byref(c)
    for a in [(None, P, 1, L.FT_F32, P, P), (r, None, 1, L.FT_F32, P, P), (r, P, -1, L.FT_F32, P, P), (r, P, 1, 3, P, P),
              (r, P, 1, L.FT_F32, ctypes.c_void_p(4104), P)]:
        assert lib.fxpq_kv_values(*a, None) == L.ERR_INVALID_ARG, a
    assert lib.fxpq_kv_values(r, None, 0, L.FT_F32, P, P, None) == L.OK
    assert lib.fxpq_kv_values(r, P, 1, L.FT_F32, None, None, None) == L.OK


def test_attention_refuses(lib):
    def call(cache=None, batch=None, t=L.FT_BF16, q=L.KVRows(4096, 128, 64), qh=4, scale=0.1, causal=1, out=P, lse=None, ws=P, nb=None):
        c, b = cache or _cache(), batch or _batch()
        n = lib.fxpq_kv_attention_workspace(ctypes.byref(c), ctypes.byref(b), qh) if nb is None else nb
        return lib.fxpq_kv_attention(ctypes.byref(c), ctypes.byref(b), t, ctypes.byref(q) if q else None, qh, scale, causal, out, lse, ws,
                                     n, None)
    for c in BAD_CACHES:
        assert call(cache=_cache(**c)) == L.ERR_INVALID_ARG, c
    for b in BAD_BATCHES:
        assert call(batch=_batch(**b)) == L.ERR_INVALID_ARG, b
    for kw in [dict(t=3), dict(q=None), dict(q=L.KVRows(None, 1, 1)), dict(qh=0), dict(qh=3), dict(scale=0.0), dict(scale=-1.0),
               dict(scale=float("nan")), dict(scale=float("inf")), dict(causal=2), dict(out=None), dict(out=ctypes.c_void_p(4104)), dict(lse=ODD)]:
        assert call(**kw) == L.ERR_INVALID_ARG, kw
    assert call(t=L.FT_F32) == L.ERR_UNSUPPORTED
    assert call(batch=_batch(T=0)) == L.OK
    b, c = _batch(B=1, wide=4096, stride=4096, T=1), _cache(dim=128)
    n = lib.fxpq_kv_attention_workspace(ctypes.byref(c), ctypes.byref(b), 4)
    if n:
        for ws, nb in ((None, n), (P, n - 1), (ctypes.c_void_p(4112), n)):
            assert call(cache=c, batch=b, ws=ws, nb=nb) == L.ERR_WORKSPACE


def test_struct_layouts_match_the_header(tmp_path):
    import os
    import shutil
    import subprocess
    if shutil.which("gcc") is None:
        pytest.skip("no host C compiler")
    mirrors = {"fxpq_kv_cache": L.KVCacheDesc, "fxpq_kv_batch": L.KVBatchDesc, "fxpq_kv_rows": L.KVRows}
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "fxpq.h"', "int main(void) {"]
    for c, py in mirrors.items():
        lines.append(f'printf("%zu", sizeof({c}));')
        lines += [f'printf(" %zu", offsetof({c}, {f}));' for f, _ in py._fields_] + ['printf("\\n");']
    (tmp_path / "l.c").write_text("\n".join(lines + ["return 0; }"]))
    inc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")
    subprocess.run(["gcc", "-I", inc, str(tmp_path / "l.c"), "-o", str(tmp_path / "l")], check=True)
    got = subprocess.run([str(tmp_path / "l")], capture_output=True, text=True, check=True).stdout.splitlines()
    for line, py in zip(got, mirrors.values()):
        assert [int(x) for x in line.split()] == [ctypes.sizeof(py)] + [getattr(py, f).offset for f, _ in py._fields_]
