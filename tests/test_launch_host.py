"""The launches of the 8-bit products without a GPU (`tests/launch_host.cu`: the library's host code on a runtime made there): every call's are
within the device's limits, the same whatever was called before, and possible on every device."""
import concurrent.futures as cf
import os
import random
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SRC = os.path.join(ROOT, "tests", "launch_host.cu")
BIN = os.path.join(ROOT, "tests", "_build", "launch_host")


@pytest.fixture(scope="module")
def launches():
    """launches(calls): a line for each call, its launches and its status, all in one new process."""
    from paper_2203_12091_gb300 import build as B
    if not os.path.exists(B.nvcc()):
        pytest.skip("nvcc not available")
    deps = [SRC, os.path.join(B.INCLUDE, "fxpq.h")] + [os.path.join(B.CSRC, f) for f in os.listdir(B.CSRC) if f.startswith(("fxpq_l", "fxpq_common", "fxpq_ptx"))]
    if not os.path.exists(BIN) or any(os.path.getmtime(d) > os.path.getmtime(BIN) for d in deps):
        os.makedirs(os.path.dirname(BIN), exist_ok=True)
        arch = ["-gencode", "arch=compute_103a,code=compute_103a"]  # (no kernel runs: they stay unassembled)

        def piece(i):
            cmd = [B.nvcc(), *arch, "-O1", "-std=c++17", "--expt-relaxed-constexpr", f"-I{B.INCLUDE}", f"-I{B.CSRC}", f"-DPIECE={i}", "-c", SRC, "-o", f"{BIN}{i}.o"]
            r = subprocess.run(cmd, capture_output=True, text=True)
            assert r.returncode == 0, r.stdout + r.stderr
            return cmd[-1]
        with cf.ThreadPoolExecutor(3) as ex:
            objs = list(ex.map(piece, range(3)))
        r = subprocess.run([B.nvcc(), *arch, *objs, "-o", BIN + ".tmp"], capture_output=True, text=True)
        assert r.returncode == 0, r.stdout + r.stderr
        os.replace(BIN + ".tmp", BIN)

    def run(calls):
        r = subprocess.run([BIN], input="\n".join(calls) + "\n", capture_output=True, text=True, timeout=120)
        assert r.returncode == 0, r.stderr
        return r.stdout.splitlines()
    return run


def some_calls(rng, count):
    def log(lo, hi):
        return max(lo, min(hi, round(lo * (hi / lo) ** rng.random())))
    calls = []
    for _ in range(count):
        M, N, K = log(1, 20000) if rng.random() < 0.7 else rng.randint(1, 64), log(1, 40000), log(1, 40000)
        kind = rng.choice(["linear", "layer", "layer", "grad"])
        more = {"linear": "", "layer": f" {rng.randint(0, 2)} {rng.randint(0, 1)} {rng.randint(0, 1)} {rng.randint(0, 1)}",
                "grad": f" {rng.randint(0, 2)} {rng.choice([0, 2])}"}[kind]
        if kind == "layer" and more.split()[2] == "1":
            N += N % 2
        calls.append(f"{kind} {M} {N} {K}{more}")
    return calls


EDGES = [f"layer {M} {N} {K} 2 {norm} 0 0" for norm in (0, 1) for N in (1, 300, 4096, 200000)
         for M, K in ((1, 32768), (1, 32769), (2, 16384), (2, 16385), (8, 4096), (8, 4097), (9, 1820), (9, 1821), (16, 1024), (16, 1025), (17, 1024), (1, 25088))]
LARGE = ["layer 4000000 100 64 2 0 0 0", "layer 300000 4096 256 2 1 0 1", "grad 5000000 200 100 2 0", "grad 5000000 200 100 0 2", "grad 300000 256 4096 2 2",
         "linear 4000000 100 64", "layer 3 8000000 64 2 0 0 0"]


def test_launches_are_within_the_limits(launches):
    calls = EDGES + LARGE + some_calls(random.Random(1), 3000)
    for call, line in zip(calls, launches(calls), strict=True):
        assert line.endswith(" = 0") and "REFUSED" not in line, (call, line)


def test_launches_do_not_depend_on_the_calls_before(launches):
    rng = random.Random(2)
    calls = list(dict.fromkeys(EDGES + some_calls(rng, 400)))
    alone = dict(zip(calls, launches(calls)))
    for call in rng.sample(calls, 60):  # each in a process of its own
        assert launches([call]) == [alone[call]], call
    for _ in range(5):
        rng.shuffle(calls)
        assert {c: line for c, line in zip(calls, launches(calls))} == alone


def test_every_device_is_set_up(launches):
    calls = [c for c in EDGES[::5] + some_calls(random.Random(3), 200)]
    first = launches(["device 0"] + calls)
    for other in (1, 15, 16, 63):
        assert launches(["device 0"] + calls + [f"device {other}"] + calls) == first + first
