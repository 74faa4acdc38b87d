"""Captured feed-forward operators where a capture has no work space left: what needs none runs, and what has
to have some says so.

The captures of a process share 4 GiB that are never given back, so the cases run in a process of their own,
which first takes them by captures that are never replayed."""
from __future__ import annotations

import os
import subprocess
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module", autouse=True)
def gpu():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"


CODE = r"""
import sys
sys.path[:0] = [%r, %r]
import numpy as np, torch
import paper_2104_05755_amd as tpp
import test_gpu_residual as res
from ffn_common import blank, down, draw, up
from test_gpu_q8 import Rows

graphs = []


def captured(call, replays=0):
    s, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    status = None
    with torch.cuda.graph(g, stream=s):
        torch.zeros(1, device="cuda").add_(1)          # no graph is empty
        try:
            call(s.cuda_stream)
        except tpp.TppError as e:
            status = e.status
    graphs.append(g)
    for _ in range(replays if status is None else 0):
        g.replay()
        torch.cuda.synchronize()
    return status


# ---- take all that captures may have: layers of ever fewer tokens of 16 entries, never replayed ------------------
one = torch.zeros(1 << 12, dtype=torch.int64, device="cuda")
P, Q = one.data_ptr(), one.data_ptr() + 4096
for bits in range(27, 4, -1):
    d = tpp.tpp_q8_gemm_desc(1, 1 << bits, 16, 17, 16, 1, tpp.TPP_DT_F32, tpp.TPP_DT_F32, 0)
    while (status := captured(lambda s: tpp.tpp_q8_linear(d, P, P, P, Q, None, s))) is None:
        pass
    assert status == tpp.TPP_ERR_NO_MEMORY, status
print("work space of captures taken by", len(graphs), "captures", flush=True)

# ---- layers ------------------------------------------------------------------------------------------------------
def layer(m, n, k, lda, first, free):
    rng = np.random.default_rng(n + k)
    a = torch.zeros(max(m * k, (m - 1) * lda + k) + 16 + first, dtype=torch.int8, device="cuda")[first:]
    for i in range(m):
        a[i * lda:i * lda + k] = up(rng.integers(-127, 128, k).astype(np.int8))
    sa, x, c = torch.ones(m, device="cuda"), up(draw(rng, n, k, k, "f32")), blank(n, m, "f32")
    d = tpp.tpp_q8_gemm_desc(m, n, k, lda, k, m, tpp.TPP_DT_F32, tpp.TPP_DT_F32, 0)
    want = blank(n, m, "f32")
    tpp.tpp_q8_linear(d, a, sa, x, want, None, tpp.current_stream())
    status = captured(lambda s: tpp.tpp_q8_linear(d, a, sa, x, c, None, s), 2)
    assert status == (None if free else tpp.TPP_ERR_NO_MEMORY), (m, n, k, lda, first, status)
    if free:
        assert np.array_equal(down(c), down(want))

layer(40, 16, 768, 768, 0, True)
layer(40, 17, 128, 128, 0, False)              # more than 16 tokens
layer(40, 13, 945, 960, 0, False)              # 13 of 1024, as whole stages of 128
layer(40, 12, 945, 960, 0, True)
layer(40, 1, 12288, 12288, 0, True)
layer(40, 1, 12289, 12304, 0, False)
layer(40, 1, 1001, 1008, 0, True)
layer(40, 1, 1001, 1001, 0, False)             # weights at odd bytes
layer(40, 1, 1001, 1008, 1, False)
layer(1, 1, 1001, 8388592, 0, True)
layer(1, 1, 1001, 8388608, 0, False)
print("layers: ok", flush=True)

# ---- the other operators: only sums over tokens need work space --------------------------------------------------
k = Rows((300, 200, 64, "bf16", "silu", 1, 0, 0), 5)
q, s = k.room(k.W)
z, gh, dz, db = up(k.z), up(k.gh), blank(300, 400, "bf16"), blank(1, 400, "f32")
tpp.tpp_q8_act(k.desc(tpp), 300, z, 400, None, 0, q, 405, s, s.shape[1], tpp.current_stream())
back = lambda b: lambda st: tpp.tpp_q8_act_backward(k.desc(tpp), 300, q, 405, s, s.shape[1], gh, 200, dz, 400, None, 0, b, st)
assert captured(back(db)) == tpp.TPP_ERR_NO_MEMORY
assert captured(back(None), 1) is None
first = down(dz).copy()
back(None)(tpp.current_stream())
assert np.array_equal(down(dz), first)
for f in (500, 9000):
    c = res.Case((20, f, "rms", "layer", "identity", 0, "bf16", "f32", 0, 0), 8)
    r = draw(np.random.default_rng(9), 20, f, f, "bf16")
    for want, status in (({"dx", "db"}, None), ({"dx", "dw_after"}, tpp.TPP_ERR_NO_MEMORY),
                         ({"dgate"}, tpp.TPP_ERR_NO_MEMORY)):
        keep = {}
        eager = res.backward(tpp, c, r, want=want, keep=keep)
        got = captured(keep["call"], 1)
        assert got == status, (f, want, got)
        for name in want:
            assert np.array_equal(down(keep["out"][name]), eager[name], equal_nan=True)
print("sums over tokens: ok", flush=True)
"""


def test_without_work_space():
    tests = os.path.join(ROOT, "tests")
    r = subprocess.run([sys.executable, "-u", "-c", CODE % (ROOT, tests)], capture_output=True, text=True,
                       timeout=100, cwd=ROOT)
    print(r.stdout, r.stderr[-3000:], flush=True)
    assert r.returncode == 0 and "sums over tokens: ok" in r.stdout
