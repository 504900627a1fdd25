"""A layer's results and its kernels' choices rest on sizes and types, not on the calls before: each order of calls in a process of its own."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CALLS = """
import hashlib, sys
import torch
from paper_2203_12091_gb300 import llm
gen = torch.Generator(device="cuda").manual_seed(1)
layers = {}
for M, N, K in ((1, 4096, 25088), (1, 4096, 4096), (8, 512, 4096), (2, 1000, 16384), (16, 512, 1024), (1, 200, 32768), (40, 512, 8192)):
    # codes next to 127 all over, so that sums pass 2^24 and their order shows
    w = torch.randint(100, 128, (N, K), dtype=torch.int8, device="cuda", generator=gen)
    x = 1 + 0.2 * torch.rand(M, K, device="cuda", generator=gen)
    layers[M, K] = llm.Linear8(w, torch.full((N,), 2.0 ** -24, device="cuda")), x
for at in sys.argv[1].split():
    layer, x = layers[tuple(map(int, at.split(",")))]
    y = layer(x, torch.float32, activation="relu")
    print(at, hashlib.sha256(y.cpu().numpy().tobytes()).hexdigest())
"""


def results(*order):
    r = subprocess.run([sys.executable, "-c", CALLS, " ".join(order)], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
    return dict(line.split() for line in r.stdout.split("\n") if line)


def test_results_do_not_depend_on_the_calls_before():
    import __graft_entry__ as g
    g.build()
    all_of = ["1,25088", "1,4096", "8,4096", "2,16384", "16,1024", "1,32768", "40,8192"]
    alone = {}
    for at in all_of:
        alone.update(results(at))
    assert results(*all_of) == alone
    assert results(*all_of[::-1]) == alone
