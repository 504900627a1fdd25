"""8-bit layers with norm, activation, gate, residual and gradient, without a GPU: the oracle against hand-worked values and
differences, the descriptors' layout, and every refusal of the C entry points (which return before any launch)."""
import ctypes
import math
import os
import re
import shutil
import subprocess

import numpy as np
import pytest
import torch

from oracle import llm as O
from paper_2203_12091_gb300 import _lib as L
from paper_2203_12091_gb300 import build as B
from paper_2203_12091_gb300 import llm

ACTS = [None, "relu", "silu", "gelu", "gelu_tanh"]


@pytest.fixture(scope="module")
def lib():
    B.build()
    return L.lib()


# ------------------------------------------------------------------------------ the oracle
def test_oracle_norm_by_hand():
    x = np.array([[3.0, -4.0, 0.0, 0.0], [0, 0, 0, 0], [1.0, np.inf, 1.0, 1.0]], np.float32)
    codes, scale = O.norm_codes(x, np.array([1, 2, 1, 1], np.float32), 0.0)
    assert codes[0].tolist() == [48, -127, 0, 0]  # 3 and -8: 47.6 and -127
    assert scale[0] * 127 == pytest.approx(8 / math.sqrt(25 / 4), rel=1e-6)
    assert not codes[1].any() and scale[1] == 0
    assert codes[2].tolist() == [127, 0, 127, 127] and scale[2] * 127 == pytest.approx(1 / math.sqrt(3 / 4), rel=1e-6)


def test_oracle_activations_by_hand():
    z = np.array([-1.0, 0.0, 2.0])
    sig = [1 / (1 + math.exp(1)), 0.5, 1 / (1 + math.exp(-2))]
    np.testing.assert_allclose(O.activation(z, "silu")[0], z * sig)
    np.testing.assert_allclose(O.activation(z, "gelu")[0], [-0.15865525393145707, 0, 1.9544997361036416])
    np.testing.assert_allclose(O.activation(z, "gelu_tanh")[0],
                               [0.5 * v * (1 + math.tanh(math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3))) for v in z])
    assert O.activation(z, "relu")[0].tolist() == [0, 0, 2] and O.activation(z, "relu")[1].tolist() == [0, 0, 1]


@pytest.mark.parametrize("act", ACTS)
def test_oracle_slopes_against_differences(act):
    z = np.array([-30.0, -5.0, -1.3, -0.2, 0.4, 1.0, 3.0, 25.0])
    h = 1e-5
    diff = (O.activation(z + h, act)[0] - O.activation(z - h, act)[0]) / (2 * h)
    np.testing.assert_allclose(O.activation(z, act)[1], diff, atol=1e-8)


@pytest.mark.parametrize("act", ACTS[1:])
@pytest.mark.parametrize("is_gated", [False, True])
def test_oracle_gradient_against_differences(act, is_gated):
    """The gradient to rows of values (what codes stand for) through weights of codes."""
    rng = np.random.default_rng(3)
    w, v, b = rng.normal(size=(6, 5)), rng.normal(size=(2, 5)), rng.normal(size=6)
    dy = rng.normal(size=(2, 3 if is_gated else 6))

    def loss(v):
        z = v @ w.T + b
        return np.sum((O.gated(z, act) if is_gated else O.layer(z, act, z * 0)) * dy)
    dx = O.layer_slopes(v @ w.T + b, dy, act, is_gated) @ w
    h = 1e-6
    for i in range(2):
        for j in range(5):
            e = np.zeros_like(v)
            e[i, j] = h
            assert dx[i, j] == pytest.approx((loss(v + e) - loss(v - e)) / (2 * h), abs=1e-7)


# ------------------------------------------------------------------------------ descriptors
def test_descriptors_match_the_header(tmp_path):
    if shutil.which("gcc") is None:
        pytest.skip("no host C compiler")
    mirrors = {"fxpq_layer": L.LayerDesc, "fxpq_layer_grad": L.LayerGradDesc}
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "fxpq.h"', "int main(void) {"]
    for c, py in mirrors.items():
        lines.append(f'printf("{c} sizeof %zu\\n", sizeof({c}));')
        lines += [f'printf("{c} {f} %zu\\n", offsetof({c}, {f}));' for f, _ in py._fields_]
    src = tmp_path / "layout.c"
    src.write_text("\n".join(lines + ["return 0; }"]))
    subprocess.run(["gcc", "-I", B.INCLUDE, str(src), "-o", str(tmp_path / "layout")], check=True)
    got = dict()
    for ln in subprocess.run([str(tmp_path / "layout")], capture_output=True, text=True, check=True).stdout.splitlines():
        c, f, v = ln.split()
        got[c, f] = int(v)
    for c, py in mirrors.items():
        assert got[c, "sizeof"] == ctypes.sizeof(py)
        for f, _ in py._fields_:
            assert got[c, f] == getattr(py, f).offset, (c, f)
    # the packed forms that small calls use
    a = list(range(1, 23))
    assert llm._LAYER(*a[:21], 0.25) == bytes(L.LayerDesc(*a[:21], 0.25))
    assert llm._LAYER_GRAD(*a[:19]) == bytes(L.LayerGradDesc(*a[:19]))


# ------------------------------------------------------------------------------ refusals
def layer(**kw):
    a = dict(x=4096, xs=64, norm=None, w=4096, ws=64, sw=4096, b=None, res=None, rs=0, y=4096, ys=8, pre=None, sx=None, M=2, N=8, K=60,
             xt=L.FT_BF16, yt=L.FT_F16, act=L.ACT_SILU, gated=0, pt=L.FT_F16, eps=1e-5)
    a.update(kw)
    return L.LayerDesc(a["x"], a["xs"], a["norm"], a["w"], a["ws"], a["sw"], a["b"], a["res"], a["rs"], a["y"], a["ys"], a["pre"], a["sx"], a["M"],
                       a["N"], a["K"], a["xt"], a["yt"], a["act"], a["gated"], a["pt"], a["eps"])


def run(lib, d, work=4096, short=0):
    n = lib.fxpq_layer_workspace(ctypes.byref(d))
    return lib.fxpq_layer_forward(ctypes.byref(d), work, n - short if n else 0, None)


@pytest.mark.parametrize("bad", [dict(x=None), dict(x=4097), dict(xs=59), dict(norm=4098), dict(w=None), dict(w=4104), dict(ws=72), dict(ws=48),
                                 dict(sw=None), dict(sw=4097), dict(b=4097), dict(res=4097, rs=8), dict(res=4096, rs=7), dict(y=None),
                                 dict(y=4097), dict(ys=7), dict(pre=4097), dict(pre=4098, pt=L.FT_F32), dict(sx=4097), dict(M=-1), dict(N=-1),
                                 dict(K=-1), dict(M=2 ** 31), dict(xt=3), dict(yt=-1), dict(act=5), dict(act=-1), dict(gated=2), dict(pt=L.FT_BF16),
                                 dict(eps=-1.0), dict(eps=2.0), dict(eps=float("nan")), dict(gated=1, N=7), dict(gated=1, act=L.ACT_NONE),
                                 dict(gated=1, res=4096, rs=8), dict(gated=1, ys=3)])
def test_layer_refuses(lib, bad):
    assert run(lib, layer(**bad)) == L.ERR_INVALID_ARG


def test_layer_refuses_workspaces(lib):
    many = layer(M=140)
    assert run(lib, many, work=None) == run(lib, many, short=1) == run(lib, many, work=4112) == L.ERR_WORKSPACE
    assert run(lib, layer(M=0)) == run(lib, layer(N=0)) == L.OK
    assert lib.fxpq_layer_forward(None, None, 0, None) == L.ERR_INVALID_ARG and lib.fxpq_layer_workspace(None) == 0


def grad(**kw):
    a = dict(dy=4096, ds=8, pre=4096, sx=4096, sw=4096, b=None, wt=4096, ws=16, dx=4096, dxs=60, M=2, N=8, K=60, yt=L.FT_F16, xt=L.FT_BF16,
             act=L.ACT_SILU, gated=0, pt=L.FT_F16)
    a.update(kw)
    return L.LayerGradDesc(a["dy"], a["ds"], a["pre"], a["sx"], a["sw"], a["b"], a["wt"], a["ws"], a["dx"], a["dxs"], a["M"], a["N"], a["K"],
                           a["yt"], a["xt"], a["act"], a["gated"], a["pt"], 0)


def run_grad(lib, d, work=4096, short=0):
    n = lib.fxpq_layer_gradient_workspace(ctypes.byref(d))
    return lib.fxpq_layer_gradient(ctypes.byref(d), work, n - short if n else 0, None)


@pytest.mark.parametrize("bad", [dict(dy=None), dict(dy=4097), dict(ds=7), dict(pre=None), dict(pre=4097), dict(pre=4098, pt=L.FT_F32), dict(sx=None),
                                 dict(sx=4097), dict(sw=None), dict(sw=4098), dict(b=4097), dict(wt=None), dict(wt=4104), dict(ws=24), dict(ws=0),
                                 dict(dx=None), dict(dx=4097), dict(dxs=59), dict(M=-1), dict(M=2 ** 30), dict(N=-1), dict(K=-1), dict(yt=3),
                                 dict(xt=-1), dict(act=7), dict(gated=-1), dict(pt=L.FT_BF16), dict(gated=1, N=7), dict(gated=1, act=L.ACT_NONE),
                                 dict(gated=1, ds=3)])
def test_gradient_refuses(lib, bad):
    assert run_grad(lib, grad(**bad)) == L.ERR_INVALID_ARG


@pytest.mark.parametrize("gated", [0, 1])
def test_relus_gradient_refuses_rounded_sums(lib, gated):
    """z > 0 of a rounded sum is not what the forward pass cut."""
    bad = grad(act=L.ACT_RELU, gated=gated)
    assert run_grad(lib, bad) == L.ERR_INVALID_ARG
    assert run_grad(lib, grad(act=L.ACT_RELU, gated=gated, pt=L.FT_F32), short=1) == L.ERR_WORKSPACE  # (past that check)
    assert run_grad(lib, grad(act=L.ACT_RELU, gated=gated, N=0, dy=None, pre=None), short=1) == L.ERR_WORKSPACE  # (nothing to cut)


def test_gradient_refuses_workspaces(lib):
    assert run_grad(lib, grad(), work=None) == run_grad(lib, grad(), short=1) == run_grad(lib, grad(), work=4112) == L.ERR_WORKSPACE
    assert run_grad(lib, grad(M=0)) == run_grad(lib, grad(K=0)) == L.OK
    assert lib.fxpq_layer_gradient(None, None, 0, None) == L.ERR_INVALID_ARG and lib.fxpq_layer_gradient_workspace(None) == 0


@pytest.mark.parametrize("name", ["tanh", "SILU", 2, True])
def test_unknown_activations_are_refused(name):
    with pytest.raises(ValueError):
        llm._activation("layer", name)


class OnDevice:
    """As much of a CUDA tensor as the checks look at."""
    requires_grad = False
    is_cuda = True

    def __init__(self, shape, dtype, index):
        self.shape, self.dtype, self.device, self.nbytes = torch.Size(shape), dtype, torch.device("cuda", index), 0

    def dim(self):
        return len(self.shape)

    def stride(self, i=None):
        s = (*self.shape[1:], 1)
        return s if i is None else s[i]

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 4096

    def detach(self):
        return self


def test_a_layers_tensors_are_on_one_device():
    w, scale = OnDevice((32, 64), torch.int8, 1), OnDevice((32,), torch.float32, 1)
    llm._check_layer("layer", w, scale, scale, 64)
    for bad in ((w, OnDevice((32,), torch.float32, 0), None), (w, scale, OnDevice((32,), torch.float32, 0))):
        with pytest.raises(ValueError):
            llm._check_layer("layer", *bad, 64)
        with pytest.raises(ValueError):
            llm.Linear8(*bad)
    with pytest.raises(ValueError):
        llm.GatedLinear8(w, scale, w, OnDevice((32,), torch.float32, 0))


def test_rows_on_another_device(monkeypatch):
    """Rows on another device than the weights are refused; on another than the current one the call is made there."""
    current, calls = [0], []

    class Device:
        def __init__(self, device):
            self.to = device.index

        def __enter__(self):
            self.was, current[0] = current[0], self.to

        def __exit__(self, *_):
            current[0] = self.was

    class Lib:
        def fxpq_linear_tokens_workspace(self, *_):
            return 0

        def fxpq_linear_tokens(self, *_):
            calls.append(current[0])
            return 0
    monkeypatch.setattr(torch.cuda, "current_device", lambda: current[0])
    monkeypatch.setattr(torch.cuda, "device", Device)
    monkeypatch.setattr(L, "lib", Lib)
    monkeypatch.setattr(llm.F, "_s", lambda _: 0)
    monkeypatch.setattr(llm, "_empty", lambda shape, dtype, device: OnDevice(shape if isinstance(shape, tuple) else (shape,), dtype, device.index))
    layer = llm.Linear8(OnDevice((32, 64), torch.int8, 1), OnDevice((32,), torch.float32, 1))
    y = layer(OnDevice((5, 64), torch.float32, 1))
    assert y.shape == (5, 32) and y.device.index == 1 and calls == [1] and current == [0]
    with pytest.raises(ValueError):
        layer(OnDevice((5, 64), torch.float32, 0))
    assert calls == [1]


def test_the_normal_tails_coefficients():
    """GELU's tail Phi(-a) = e^(-a^2 / 2) t P(t) with the source's own coefficients, in 64 bits: 7e-8 of itself, as its comment says."""
    from scipy.special import erfcx
    src = open(os.path.join(B.CSRC, "fxpq_layer.cuh")).read()
    body = src[src.index("float normal_tail("):src.index("float gelu(")]
    number = r"(-?[0-9.]+(?:e[-+]?[0-9]+)?)f"
    slope, = re.findall(rf"fmaf\({number}, a, 1.0f\)", body)
    coefficients = re.findall(rf"float p = {number};", body) + re.findall(rf"p = fmaf\(p, t, {number}\);", body)
    assert len(coefficients) == 10
    a = np.linspace(0, 40, 400001)
    t = 1 / (1 + np.float64(np.float32(slope)) * a)
    p = np.polyval([np.float64(np.float32(c)) for c in coefficients], t)
    assert np.max(np.abs(t * p / (0.5 * erfcx(a / math.sqrt(2))) - 1)) <= 7e-8
