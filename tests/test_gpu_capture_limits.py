"""Captured attention operators where a capture has no work space left: what needs none runs, what has an
unsplit form takes it, and what has to have work space says so.

The captures of a process share 4 GiB that are never given back, so the cases run in a process of their own,
which first takes them by captures that are never replayed."""
from __future__ import annotations

import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import oracle
from helpers import values
from test_gpu_attention import U, Paged, close, draw, up

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module", autouse=True)
def gpu():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"


@pytest.mark.parametrize("D,hq,hk,dtype,max_len", [(128, 64, 4, "bf16", 1 << 25), (77, 64, 4, "f32", 1 << 26),
                                                   (128, 64, 1, "bf16", 1 << 27)])
def test_attention_captured_without_work_space(D, hq, hk, dtype, max_len):
    """Room for sequences so long that the partial results (512 heads' spans, at most 4096 positions each)
    would pass what captures may take: a span of several blocks for every sequence, the outputs written
    directly."""
    import paper_2104_05755_amd as tpp
    lens, f, scale = [3000, 2500, 1025, 1024, 700, 0, 5, 2049], hq * D, D ** -0.5
    pc = Paged(lens, D, hk, 1024, dtype, seed=D, holes=[(0, 1), (3, 0), (7, 2)], room=max_len)
    n, q = len(lens), draw(pc.rng, (len(lens), f), dtype)
    out, lse = torch.full((n, f), 9.0, device="cuda"), torch.full((n, hq), 9.0, device="cuda")
    qd, desc = up(q), tpp.tpp_attn_desc(hq, tpp.TPP_DT_F32, scale, 0, max_len)
    print(f"attention D{D} {hq}x{hk} {dtype} max_len {max_len}, captured", flush=True)
    s, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=s):
        tpp.tpp_paged_attention(desc, pc.c(tpp), n, qd, f, pc.d_lens, pc.d_pages, pc.pages.shape[1], out, f, lse,
                                None, None, 0, s.cuda_stream)
    k, v = pc.host()
    mag = {"f32": np.abs, "bf16": lambda x: x & 0x7FFF}[dtype]
    args = (dtype, D, hk, 1024, pc.n_pages, pc.strides, pc.pages, q, f, hq, lens, scale)
    ref, ref_lse, _ = oracle.paged_attention(k, v, *args)
    big, _, _ = oracle.paged_attention(k, mag(v), *args)
    # the bounds of test_gpu_attention
    qn = np.abs(values(q, dtype)).reshape(n, hq, D).sum(-1)
    ds = (D + 4) * U * scale * qn * np.nanmax(np.abs(values(k, dtype)))
    rel = 2 * ds + (64 + max(lens)) * U + 2.0 ** -20
    for _ in range(2):
        out.fill_(9), lse.fill_(9)
        g.replay()
        torch.cuda.synchronize()
        close(out.cpu().numpy().reshape(n, hq, D), ref, (rel + (2.0 ** -16 if dtype == "bf16" else 0))[..., None] * big,
              "f32", "out")
        close(lse.cpu().numpy().astype(np.float64), ref_lse, rel, "f32", "lse")


CODE = r"""
import sys
sys.path[:0] = [%r, %r]
import numpy as np, torch
import paper_2104_05755_amd as tpp
from test_gpu_attention import Paged, Rope, draw, run_backward, up
import oracle

graphs = []


def captured(calls, replays=2):
    s, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    status = None
    with torch.cuda.graph(g, stream=s):
        torch.zeros(1, device="cuda").add_(1)          # no graph is empty
        try:
            calls(s.cuda_stream)
        except tpp.TppError as e:
            status = e.status
    graphs.append(g)
    for _ in range(replays):
        g.replay()
        torch.cuda.synchronize()
    return status


# ---- take all that captures may have: attention with totals, of ever shorter room, never replayed -----------
one = torch.zeros(1 << 12, dtype=torch.int64, device="cuda")
P = one.data_ptr()
for bits in range(29, 6, -1):
    c = tpp.tpp_kv_cache(P, P, tpp.TPP_DT_F32, 8, 1, 1 << 30, 1, 8, 8, 8)
    d = tpp.tpp_attn_desc(1, tpp.TPP_DT_F32, 1.0, 0, 1 << bits)
    take = lambda s: tpp.tpp_paged_attention(d, c, 1, P, 8, P, P, 1, P, 8, None, None, P, 1 << bits, s)
    while (status := captured(take, 0)) is None:
        pass
    assert status == tpp.TPP_ERR_NO_MEMORY, status
print("work space of captures taken by", len(graphs), "captures", flush=True)

# ---- an eviction of one launch needs none ---------------------------------------------------------------------
def evict(lens, budget, max_len, want):
    pc = Paged(lens, 64, 2, 16, "bf16", seed=budget)
    n = len(lens)
    tot = np.random.default_rng(budget).random((n, max_len)).astype(np.float32)
    d_tot, t_out = up(tot), torch.full((n, max_len), -5.0, device="cuda")
    l_out = torch.zeros(n, dtype=torch.int64, device="cuda")
    status = captured(lambda s: tpp.tpp_cache_evict(pc.c(tpp), n, max_len, budget, pc.d_lens, pc.d_pages,
                                                    pc.pages.shape[1], d_tot, None, None, max_len, l_out, t_out,
                                                    None, s), 1 if want is None else 0)
    assert status == want, (lens, budget, status)
    if want is None:
        new, keep = oracle.cache_evict(lens, budget, tot)
        assert l_out.tolist() == new.tolist()
        for b in range(n):
            assert np.array_equal(t_out[b, :new[b]].cpu().numpy(), tot[b, keep[b, :new[b]]])

evict([2049, 2040, 7, 2049], 2048, 2049, None)
print("eviction of one launch: ok", flush=True)
evict([3000, 100], 1000, 3000, tpp.TPP_ERR_NO_MEMORY)
print("eviction of two launches: refused", flush=True)

# ---- the rotation's backward pass has an unsplit form --------------------------------------------------------------
r = Rope((600, 4, 2, 64, 64, "halves", "bf16", 0, 0), 3)
g = [draw(np.random.default_rng(1), (600, h * 64 + 1), "bf16") for h in (4, 2)]
want, want_w = run_backward(tpp, r, g)
dev = [up(x) for x in g]
dx = [torch.zeros(600, h * 64, dtype=torch.int16, device="cuda") for h in (4, 2)]
dw = [torch.zeros(64, device="cuda") for _ in range(2)]
status = captured(lambda s: tpp.tpp_qk_norm_rope_backward(
    r.desc(tpp), 600, r.at[0], r.ld, r.at[1], r.ld, r.dev["w"][0], r.dev["w"][1], r.dev["rot"], r.dev["pos"],
    dev[0], 257, dev[1], 129, dx[0], 256, dx[1], 128, dw[0], dw[1], s))
assert status is None, status
for s, h in enumerate((4, 2)):
    assert torch.equal(dx[s].ravel(), want[s].ravel())
    _, ref = oracle.qk_norm_rope_backward(r.flat[r.off[s]:], r.ld, h, 64, 64, "halves", r.w[s], r.rot, r.pos,
                                          1e-5, "bf16", g[s], h * 64 + 1)
    # (64 + rows) u of the sum of |g xn|, below 600 h * 16 for these normals
    assert np.abs(dw[s].cpu().numpy() - ref).max() < (64 + 600 * h) * 2.0 ** -24 * 600 * h * 16
    assert np.abs(ref).max() > 1
print("backward pass without work space: ok", flush=True)
"""


def test_without_work_space():
    tests = os.path.join(ROOT, "tests")
    r = subprocess.run([sys.executable, "-u", "-c", CODE % (ROOT, tests)], capture_output=True, text=True,
                       timeout=100, cwd=ROOT)
    print(r.stdout, r.stderr[-3000:], flush=True)
    assert r.returncode == 0 and "backward pass without work space: ok" in r.stdout
