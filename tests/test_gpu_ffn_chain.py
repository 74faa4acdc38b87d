"""The feed-forward operators run together as they are used: a serving step in 8 bits and a training step
that keeps its activation in 8 bits, with the BRGEMMs between them, against the oracle.

Each step's output is compared with the oracle's for the step's inputs as the device has them, so that
the bounds are those of one step: a relative distance of 2^-8 in norm is a bf16 output's half unit at most
(each entry is off by 2^-9 of itself to 2^-8), an fp32 output of a product is off by (k + 8) 2^-24 of the
magnitudes at most, 8-bit rows are exact for the stored rows they are made of, and one step of 127 where
they are made of values that are not stored (an activation within 2^-20 of the oracle's can round to its
type, and then to 8 bits, the other way; that moves a scale by up to 2^-8 as well)."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import oracle
import workloads as wk
from helpers import rel_fro, run_call_oracle, values

pytestmark = pytest.mark.gpu
HALF = 2.0 ** -8


@pytest.fixture(scope="module", autouse=True)
def gpu():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"


def run(wl, graph=False):
    """Every step on the device; host copies of all arrays behind each step."""
    from paper_2104_05755_amd import torch_io
    dev = torch_io.upload(wl)
    steps = [torch_io.prepare_step(s, dev) for s in wl.steps]
    host = lambda: {k: torch_io.to_host(dev[k], wl.arrays[k]).copy() for k in wl.arrays}
    got = []
    for s in steps:
        torch_io.launch_step(s, dev)
        torch.cuda.synchronize()
        got.append(host())
    if graph:   # the whole chain captured, replayed three times from cleared outputs
        first = {k: dev[k].clone() for k in dev}
        st = torch.cuda.Stream()
        with torch.cuda.stream(st):
            for s in steps:
                torch_io.launch_step(s, dev, st.cuda_stream)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            for s in steps:
                torch_io.launch_step(s, dev, st.cuda_stream)
        for _ in range(3):
            for k in graph:
                dev[k].zero_()
            g.replay()
            for s in steps:   # the program's own eager work between
                torch_io.launch_step(s, dev, st.cuda_stream)
            g.replay()
            torch.cuda.synchronize()
            for k in dev:
                assert torch.equal(dev[k].view(torch.int8), first[k].view(torch.int8)), k
    return got


def residual_reference(st, a):
    b = oracle.norm(a[st.b], st.features, "bf16", "rms", st.eps, a[st.w_after])
    r = values(a[st.x], "bf16") + st.scale * b
    y = oracle.norm(a[st.r], st.features, "bf16", "rms", st.eps, a[st.w_before])
    return r, y


def test_serving_step():
    wl = wk.ffn_step()
    s1, up, act, down, s2 = wl.steps
    got = run(wl, graph=("r1", "q1", "t1", "z", "q2", "t2", "o", "r2", "y"))
    a = got[0]
    r, y = residual_reference(s1, a)
    assert rel_fro(values(a["r1"], "bf16"), r) <= HALF
    back = a["q1"] * a["t1"].astype(np.float64)[:, None]
    assert (np.abs(back - y) <= a["t1"][:, None] * 0.5 + np.abs(y).max(1, keepdims=True) * 2 * HALF).all()
    a = got[1]
    z = oracle.q8_product(a["w1"], a["q1"], up.k) * a["t1"].astype(np.float64)[:, None] * a["s1"]
    assert rel_fro(values(a["z"], "bf16"), z) <= HALF
    a = got[2]
    zv = values(a["z"], "bf16")
    h = oracle.act(zv[:, :act.features], "silu")[0] * zv[:, act.features:]
    back = a["q2"] * a["t2"].astype(np.float64)[:, None]
    assert (np.abs(back - h) <= a["t2"][:, None] * 0.5 + np.abs(h).max(1, keepdims=True) * 2 * HALF).all()
    a = got[3]
    o = oracle.q8_product(a["w2"], a["q2"], down.k) * a["t2"].astype(np.float64)[:, None] * a["s2"]
    assert rel_fro(values(a["o"], "bf16"), o) <= HALF
    a = got[4]
    r, y = residual_reference(s2, a)
    assert rel_fro(values(a["r2"], "bf16"), r) <= HALF and rel_fro(values(a["y"], "bf16"), y) <= HALF


def test_training_step():
    """And its gradients against those of the network without rounding: the 8 bits move z by a half step of its
    group at most, 1 / 254 of an entry that is below 4 root mean squares in 64, and three roundings to bf16
    are on the way: 4 / 254 + 3 * 2^-8 < 0.03."""
    wl = wk.mlp_kept()
    got = run(wl, graph=("z", "h", "q", "qs", "y", "dh", "dz", "h2", "db1", "dw2", "dx", "dw1"))
    for st, a in zip(wl.steps, got):
        if isinstance(st, wk.Call):
            c = np.array(a[st.c])
            ref = run_call_oracle(st, dict(a, **{st.c: c}), want_ref64=True)
            out = values(a[st.c], st.c_type).reshape(-1)
            assert rel_fro(out, np.asarray(ref).reshape(-1)) <= (HALF if st.c_type == "bf16" else
                                                                 (st.k + 8) * 2.0 ** -24), st.c
        elif isinstance(st, wk.KeepStep):
            z = values(a["z"], "bf16")
            assert rel_fro(values(a["h"], "bf16"), oracle.act(z, "gelu_tanh")[0]) <= HALF
            q, s = oracle.q8_rows(z, st.keep_group)
            assert np.array_equal(a["q"], q) and np.array_equal(a["qs"], s)
        else:
            z = a["q"] * np.repeat(a["qs"].astype(np.float64), st.kept_group, 1)
            value, slope = oracle.act(z, "gelu_tanh")
            dz = values(a["dh"], "bf16") * slope
            assert rel_fro(values(a["dz"], "bf16"), dz) <= HALF
            assert rel_fro(values(a["h2"], "bf16"), value) <= HALF
            assert np.linalg.norm(a["db1"] - dz.sum(0)) <= (len(dz) + 128) * 2.0 ** -24 * np.linalg.norm(
                np.abs(dz).sum(0))
    a, f = got[-1], lambda k: values(wl.arrays[k], "bf16")
    x, w1, w2, dy = f("x"), f("w1"), f("w2"), f("dy")   # w1: [hidden][inter], w2: [inter][hidden]
    value, slope = oracle.act(x @ w1 + wl.arrays["b1"], "gelu_tanh")
    dz = (dy @ w2.T) * slope
    for k, ref in (("dx", dz @ w1.T), ("dw1", x.T @ dz), ("dw2", value.T @ dy), ("db1", dz.sum(0))):
        out = values(a[k], "bf16") if a[k].dtype == np.uint16 else a[k]
        assert rel_fro(out, ref) <= 0.03, k
