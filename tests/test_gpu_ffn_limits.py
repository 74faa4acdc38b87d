"""The feed-forward operators at the ends of what they take: groups without a scale behind every
activation, activations far from zero, norms of rows far below 1.

Bounds (u = 2^-24) beside each test; a bf16 output adds half a unit of its own."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from ffn_common import U, blank, close, code, down, draw, untouched, up
from helpers import values
from test_gpu_q8 import act_code

pytestmark = pytest.mark.gpu
ACTS = ("none", "relu", "gelu_tanh", "silu")


@pytest.fixture(scope="module", autouse=True)
def gpu():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"


@pytest.fixture(scope="module")
def tpp():
    import paper_2104_05755_amd as tpp
    return tpp


def act_backward(tpp, q, scale, group, gh, act, gated, dtype):
    """(dz, h2, dbias) of rows q with their scales, as float64."""
    T, W = q.shape
    F = W >> gated
    d = tpp.tpp_q8_desc(F, group, code(tpp, dtype), act_code(tpp, act), gated)
    dz, h2, db = blank(T, W + 1, dtype), blank(T, F + 1, dtype), blank(1, W, "f32")
    tpp.tpp_q8_act_backward(d, T, up(q), W, up(scale), scale.shape[1], up(gh), gh.shape[1], dz, W + 1, h2, F + 1, db,
                            tpp.current_stream())
    dz, h2 = down(dz), down(h2)
    assert untouched(dz, W) and untouched(h2, F)
    return values(dz, dtype)[:, :W], values(h2, dtype)[:, :F], down(db)[0].astype(np.float64)


# ---- groups without a scale -------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("features,group", [(96, 32), (100, 16), (96, 0), (5, 0)])   # the last: a row below 8 entries
@pytest.mark.parametrize("act", ACTS)
def test_gradients_of_groups_without_a_scale(tpp, act, features, group, dtype):
    """A scale of NaN makes NaN of all that the backward pass makes of its group, whatever the activation, and of
    nothing else."""
    rng = np.random.default_rng(features + group)
    for gated in (0, 1):
        W, T = features << gated, 6
        g = group or W
        q = rng.integers(-127, 128, (T, W)).astype(np.int8)
        scale = rng.uniform(0.5, 2, (T, -(-W // g))).astype(np.float32) / 64
        gh = draw(rng, T, features, features, dtype)
        bad = np.zeros(scale.shape, bool)
        bad[1, 0] = bad[3, -1] = bad[4, scale.shape[1] // 2] = True
        scale[bad] = np.nan
        entry = np.repeat(bad, g, 1)[:, :W]
        q[entry] = 0
        dz, h2, db = act_backward(tpp, q, scale, group, gh, act, gated, dtype)
        a, u = entry[:, :features], entry[:, features:]
        want_h = a | u if gated else a
        want_dz = np.concatenate([a | u, a], 1) if gated else a
        if act == "none" and not gated:   # the slope is 1 whatever the entry: dz = gh
            want_dz = np.zeros_like(a)
        elif act == "none":               # dz of the first half: gh u
            want_dz = np.concatenate([u, a], 1)
        assert np.array_equal(np.isnan(h2), want_h)
        assert np.array_equal(np.isnan(dz), want_dz)
        assert np.array_equal(np.isnan(db), want_dz.any(0))


@pytest.mark.parametrize("group", [0, 32])
def test_an_infinity_is_seen_behind_relu(tpp, group):
    """From an infinity in z to the gradients: the forward call's h keeps it, and the backward pass, which has
    lost the group's entries, gives NaN."""
    rng = np.random.default_rng(1)
    z = draw(rng, 3, 64, 64, "f32")
    z[1, 40] = np.inf
    d = tpp.tpp_q8_desc(64, group, tpp.TPP_DT_F32, tpp.TPP_ACT_RELU, 0)
    q, s = torch.zeros((3, 64), dtype=torch.int8, device="cuda"), torch.zeros((3, 64 // group if group else 1), device="cuda")
    h = blank(3, 64, "f32")
    tpp.tpp_q8_act(d, 3, up(z), 64, h, 64, q, 64, s, s.shape[1], tpp.current_stream())
    assert np.array_equal(down(h), np.where(z > 0, z, 0))
    dz, h2, db = act_backward(tpp, down(q), down(s), group, draw(rng, 3, 64, 64, "f32"), "relu", 0, "f32")
    lost = np.zeros((3, 64), bool)
    lost[1, 32 if group else 0:] = True
    assert np.array_equal(np.isnan(h2), lost) and np.array_equal(np.isnan(dz), lost)
    assert np.array_equal(np.isnan(db), lost.any(0))


@pytest.mark.parametrize("n", [3, 70, 2100])
def test_products_of_tokens_without_a_scale(tpp, n):
    """Their columns are NaN behind no activation and GELU; TPP_EPI_RELU is x > 0 ? x : +0 here as in every other
    product, so 0 behind it."""
    rng = np.random.default_rng(n)
    a, b = (rng.integers(-127, 128, (r, 64)).astype(np.int8) for r in (300, n))
    sa, sb = np.full(300, 0.01, np.float32), rng.uniform(0.5, 1, n).astype(np.float32)
    b[1], sb[1] = 0, np.nan
    for flags in (0, tpp.TPP_EPI_GELU_TANH, tpp.TPP_EPI_RELU):
        d = tpp.tpp_q8_gemm_desc(300, n, 64, 64, 64, 300, tpp.TPP_DT_F32, tpp.TPP_DT_F32, flags)
        c = blank(n, 300, "f32")
        tpp.tpp_q8_gemm(d, up(a), up(sa), up(b), up(sb), c, None, tpp.current_stream())
        c = down(c)
        assert (c[1] == 0).all() if flags == tpp.TPP_EPI_RELU else np.isnan(c[1]).all()
        assert np.isfinite(np.delete(c, 1, 0)).all()


# ---- activations far from zero ------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("gated", [0, 1])
@pytest.mark.parametrize("features", [320, 5])
@pytest.mark.parametrize("act", ["relu", "gelu_tanh", "silu"])
def test_gradients_far_from_zero(tpp, act, gated, features, dtype):
    """|z'| from 90 to 3e38.  To the right act(z) = z and act' = 1 to far below u (1 - s < exp(-90)); z' rounds
    once, s once, their product once, products with gh and u once each: 6 u of the magnitude.  To the left both are 0
    to within 90 exp(-90) < 1e-37."""
    rng = np.random.default_rng(features)
    tops = [90.0, 1e3, 1e6, 1e10, 1e18, 1e19, 1e20, 1e27, 1e30, 1e33, 1e36, 1e38, 3e38]
    T = len(tops)
    q = rng.choice(np.r_[-127, np.arange(-127, -99), np.arange(100, 128), 127], (T, features)).astype(np.int8)
    scale = np.float32(tops)[:, None] / np.float32(100)   # |z'| >= top
    scale = np.minimum(scale, np.float32(3e38) / 127)
    q[:, 0], q[:, 1] = -127, 127
    gh = draw(rng, T, features, features, dtype)
    if dtype == "f32":
        gh = np.clip(gh, -1, 1)        # (gh act stays finite)
    else:
        gh = draw(rng, T, features, features, dtype, std=0.03)
    a = q.astype(np.float64) * scale
    if gated:
        # the second half: one group of its own, of values about 1
        group = 0 if features == 5 else 64
        u8 = rng.integers(1, 128, (T, features)).astype(np.int8)
        if group:
            s_u = np.full((T, features // group), np.float32(1 / 64))
            qq, ss = np.concatenate([q, u8], 1), np.concatenate([np.repeat(scale, features // group, 1), s_u], 1)
            u = u8 / 64.0
        else:                          # one scale for the row: u is as large as a; keep it to the tops that fit
            qq, ss = np.concatenate([q, np.ones_like(u8)], 1), scale
            u = np.ones_like(a) * scale
    else:
        group, qq, ss, u = 0, q, scale, 1.0
    dz, h2, _ = act_backward(tpp, qq, ss, group, gh, act, gated, dtype)
    g = values(gh, dtype)[:, :features]
    right = a > 0
    big = np.float64(np.finfo(np.float32).max) * (1 - 2.0 ** -6)

    def check(got, ref, what):
        ref = np.broadcast_to(ref, got.shape)
        fits = right & (np.abs(ref) < big)
        half = 2.0 ** -8 if dtype == "bf16" else U
        off = np.abs(got - ref)[fits]
        assert (off <= (6 * U + half) * np.abs(ref[fits]) + 1e-37).all(), what
        return got[~right]

    factor = np.abs(np.broadcast_to(u, a.shape))[~right]
    gm = np.abs(g)[~right]
    left = check(h2, a * u, "h2")
    assert (np.abs(left) <= 1e-37 * factor).all(), f"h2 left of zero: {np.abs(left).max()}"
    left = check(dz[:, :features], g * u, "dz")
    assert (np.abs(left) <= 1e-37 * (1 + gm * factor)).all(), f"dz left of zero: {np.abs(left).max()}"
    if gated:
        left = check(dz[:, features:], g * a, "dz of the factor")
        assert (np.abs(left) <= 1e-37 * gm).all(), f"dz of the factor left of zero: {np.abs(left).max()}"


# ---- norms of rows far below 1 -----------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("features", [5, 600, 1001, 6000, 20001])
@pytest.mark.parametrize("after,before", [("rms", "none"), ("none", "rms"), ("layer", "rms"), ("none", "layer")])
@pytest.mark.parametrize("k", [-40, -56])
def test_norms_of_small_rows(tpp, monkeypatch, k, after, before, features, dtype):
    """Rows of 2^k with eps = 0 and nothing beside them in the stream: the norms do not see the factor, down to mean
    squares below 2^-100.  Bounds: those of test_gpu_residual with eps = 0."""
    import test_gpu_residual as res
    monkeypatch.setattr(res, "EPS", 0.0)
    c = res.Case((2, features, after, before, "none", 0, dtype, "f32", 0, 0), 7, mean=0.0)
    small = np.float32(2.0 ** k)
    tiny = lambda a: a * small if dtype == "f32" else _bits(values(a, "bf16") * float(small))
    c.b = tiny(c.b)
    c.x = np.zeros_like(c.x)
    r, y, q, qs = res.forward(tpp, c)
    res.check_forward(c, r, y, q, qs)
    if after == "none":   # (the bound there is that of values about 1; r = scale b: scale's rounding and the product's)
        close(r, c.scale * values(c.b, dtype), 2 * U * np.abs(values(c.b, dtype)), "r")
    assert np.isfinite(values(r, dtype)[:, :features]).all() and (y is None or np.isfinite(values(y, dtype)[:, :features]).all())
    # backward: the small row is the one that is normed
    if after != "none" and before != "none":
        return
    r = draw(np.random.default_rng(9), 2, features, features, dtype)
    if before != "none":
        r = tiny(r)
    got = res.backward(tpp, c, r)
    res.check_backward(c, r, got)


def _bits(v):
    import workloads as wk
    return wk.bf16_bits(v.astype(np.float32)).reshape(v.shape)
