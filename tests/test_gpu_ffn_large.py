"""The feed-forward operators at the sizes that training and serving have: products whose k refills every
place in LDS several times, in each tile and each few-token form; rows past each size from which loads and stores
go past the caches' replacement; row teams and columns of tokens that go round their loops often.

The bounds are those of test_gpu_q8 and test_gpu_residual, whose cases stay below all of that."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import oracle
import test_gpu_q8 as q8
import test_gpu_residual as res
from ffn_common import blank, close, down, draw, untouched, up
from helpers import values

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"


@pytest.fixture(scope="module")
def tpp():
    import paper_2104_05755_amd as tpp
    return tpp


# ---- products ---------------------------------------------------------------------------------------
# m, n, k, extra lda, ldb, ldc, first bytes, c type, flags; stages of 128 bytes of k, places that they go round
LONG = [
    (4100, 3900, 1024, 0, 0, 0, 0, "f32", ()),                        # 256 x 256: 8 stages, 2 places
    (4100, 3900, 1001, 7, 7, 0, 0, "bf16", ("bias", "gelu_tanh")),    # with a tail of k
    (3840, 3840, 2048, 0, 0, 0, 0, "bf16", ("bias", "relu")),         # whole tiles
    (2050, 2048, 1024, 0, 0, 2, 0, "f32", ("bias", "relu")),          # 128 x 128: 8 stages, 2 places
    (2050, 2048, 1000, 8, 8, 0, 0, "bf16", ()),
    (1533, 777, 2048, 0, 0, 0, 0, "f32", ("gelu_tanh",)),             # 64 x 64: 16 stages, 4 places
    (1533, 777, 1001, 7, 7, 0, 0, "f32", ("bias",)),
    (581, 4200, 768, 0, 0, 3, 0, "bf16", ("bias",)),                  # 64 x 64: 6 stages, 2 places
    (581, 4200, 700, 4, 4, 0, 0, "f32", ()),
    (520, 500, 5000, 8, 8, 0, 0, "f32", ("bias",)),                   # shares of k: 5 stages to a wavefront
] + [(m, n, k, pad, pad, 0, 0, ct, fl)                                # up to 64 tokens, 16 and 32 channels to a workgroup
     for m in (1000, 6200)
     for n, k, pad, ct, fl in ((1, 4096, 0, "f32", ()), (16, 3001, 7, "bf16", ("bias",)), (17, 2000, 0, "f32", ("relu",)),
                               (32, 4096, 0, "bf16", ()), (33, 3001, 7, "f32", ("bias",)),
                               (48, 4096, 0, "bf16", ("gelu_tanh",)), (49, 5000, 8, "f32", ()), (64, 2048, 0, "bf16", ()))]


@pytest.mark.parametrize("case", LONG, ids=str)
def test_long_products(tpp, case):
    p = q8.Product(case)
    # exact in fp64 (below 2^31), by rows of the tokens; the oracle's own sums for some rows
    a = p.a[:, :p.k].astype(np.float64).T.copy()
    total = np.concatenate([p.b[j:j + 512, :p.k].astype(np.float64) @ a for j in range(0, p.n, 512)])
    some = np.unique(np.linspace(0, p.n - 1, 5).astype(int))
    assert np.array_equal(oracle.q8_product(p.a, np.ascontiguousarray(p.b[some]), p.k), total[some])
    c = p.run(tpp)
    close(c[:, :p.m], *p.finish(total, p.sb), "c")
    assert untouched(c, p.m)
    # scales of 1 and no epilogue: the sums themselves, and the same ones each time
    p.flags, p.sa[:], p.sb[:], p.ctype = (), 1, 1, "f32"
    first = p.run(tpp)
    assert np.array_equal(first[:, :p.m], total.astype(np.float32))
    assert np.array_equal(p.run(tpp)[:, :p.m], first[:, :p.m])


@pytest.mark.parametrize("n,k", [(1, 4096), (3, 4000), (4, 1001), (16, 768), (130, 4096), (2000, 1024)])
def test_layers_of_wide_inputs(tpp, n, k):
    """tpp_q8_linear: 8-bit rows made beside the product and before it, to the bit of rows made apart."""
    p = q8.Product((6200, n, k, -k % 16, 0, 0, 0, "f32", ("bias",)), 1)
    x = draw(np.random.default_rng(n), n, k, k, "bf16")
    a, sa, bias, c = up(p.a), up(p.sa), up(p.bias), blank(n, 6200, "f32")
    st = tpp.current_stream()
    tpp.tpp_q8_linear(p.desc(tpp, "bf16"), a, sa, up(x), c, bias, st)
    q, s = oracle.q8_rows(values(x, "bf16"))
    b = np.zeros((n, k + -k % 16), np.int8)
    b[:, :k] = q
    apart = blank(n, 6200, "f32")
    tpp.tpp_q8_gemm(p.desc(tpp, ldb=b.shape[1]), a, sa, up(b), up(s[:, 0]), apart, bias, st)
    total = q.astype(np.float64) @ p.a[:, :k].astype(np.float64).T
    close(down(c), *p.finish(total, s[:, 0]), "c")
    close(down(apart), *p.finish(total, s[:, 0]), "c of rows made apart")


# ---- 8-bit rows ---------------------------------------------------------------------------------------
# tokens, features, group, dtype, act, gated, extra ld, first entry
ROWS = [
    (1500, 2048, 128, "bf16", "gelu_tanh", 0, 0, 0),    # outputs above 8 MB
    (1700, 1001, 64, "f32", "silu", 0, 1, 1),
    (1500, 1001, 64, "f32", "silu", 1, 1, 0),           # halves that lie otherwise
    (1500, 1024, 64, "bf16", "silu", 1, 0, 0),          # both halves together
    (6600, 4096, 128, "bf16", "gelu_tanh", 0, 0, 0),    # all above 128 MB
    (2450, 4096, 0, "f32", "silu", 1, 0, 0),
    (2450, 4099, 32, "f32", "gelu_tanh", 1, 0, 0),
]


@pytest.mark.parametrize("case", ROWS, ids=str)
def test_large_act_and_backward(tpp, case):
    q8.test_act_and_backward(tpp, case)


@pytest.mark.parametrize("case", [
    (28100, 1600, 0, "bf16", "none", 0, 0, 0), (7000, 1000, 64, "f32", "relu", 0, 0, 0),
    (30000, 999, 0, "f32", "none", 0, 1, 0), (6000, 8192, 64, "bf16", "relu", 0, 0, 0)], ids=str)
def test_large_quantize(tpp, case):
    """Rows of values as they are: exact."""
    T, F, group, dtype, act, _, pad, _ = case
    rng = np.random.default_rng(T)
    z = np.tile(draw(rng, 500, F, F + pad, dtype), (T // 500 + 1, 1))[:T].copy()   # (of which the oracle does 500)
    c = q8.Rows((3, F, group, dtype, act, 0, pad, 0))
    q, s = torch.full((T, F + 5), 77, dtype=torch.int8, device="cuda"), torch.full((T, c.groups(F) + 1), 55.0, device="cuda")
    tpp.tpp_q8_quantize(c.desc(tpp), T, up(z), F + pad, q, F + 5, s, s.shape[1], tpp.current_stream())
    v = values(z[:500], dtype)[:, :F]
    want, scale = oracle.q8_rows(np.where(v > 0, v, 0) if act == "relu" else v, group)
    q, s = down(q), down(s)
    for t in range(0, T, 500):
        n = min(500, T - t)
        assert np.array_equal(q[t:t + n, :F], want[:n]) and np.array_equal(s[t:t + n, :-1], scale[:n])
    assert (q[:, F:] == 77).all() and (s[:, -1] == 55.0).all()


# ---- norms ----------------------------------------------------------------------------------------------
# tokens, features, after, before, gate, gate_every, dtype, gate type, extra ld, first entry
NORMS = [
    (9001, 500, "layer", "layer", "tanh", 7, "bf16", "bf16", 4, 0),       # a wavefront to a row
    (9001, 504, "rms", "rms", "identity", 0, "bf16", "f32", 0, 0),
    (6000, 1024, "rms", "layer", "identity", 1000, "bf16", "bf16", 0, 0),  # two
    (3000, 2047, "layer", "rms", "sigmoid", 700, "f32", "bf16", 0, 1),     # four
    (1100, 4096, "rms", "rms", "identity", 0, "bf16", "f32", 0, 0),        # eight
    (1100, 4095, "layer", "layer", "tanh", 100, "f32", "f32", 1, 0),
    (1100, 5000, "layer", "rms", "identity", 0, "f32", "f32", 0, 0),       # eight, two chunks to a lane
    (1100, 8192, "rms", "rms", "none", 0, "bf16", "f32", 0, 0),
    (900, 9000, "rms", "layer", "identity", 256, "bf16", "bf16", 0, 0),    # sums by a kernel of their own
    (520, 16384, "rms", "rms", "tanh", 130, "f32", "f32", 0, 0),
    (5500, 2048, "layer", "rms", "sigmoid", 0, "f32", "bf16", 0, 0),       # all above 256 MB
    (5500, 4096, "rms", "rms", "identity", 0, "bf16", "f32", 0, 0),
]


@pytest.mark.parametrize("case", NORMS, ids=str)
def test_large_norms(tpp, case):
    c = res.Case(case)
    r, y, q, qs = res.forward(tpp, c)
    res.check_forward(c, r, y, q, qs)
    r2, y2, _, _ = res.forward(tpp, c, in_place=True, q=False)
    assert np.array_equal(r2[:, :c.F], r[:, :c.F]) and np.array_equal(y2[:, :c.F], y[:, :c.F])


@pytest.mark.parametrize("case", NORMS, ids=str)
def test_large_norms_backward(tpp, case):
    c = res.Case(case, 1)
    r = draw(np.random.default_rng(5), c.T, c.F, c.ld, c.dtype, 1.5, 0.2)
    got = res.backward(tpp, c, r)
    res.check_backward(c, r, got)
    again = res.backward(tpp, c, r, want={"dx", "dw_after", "dgate"})
    for k in ("dx", "dw_after", "dgate"):
        assert got[k] is None or np.array_equal(got[k], again[k], equal_nan=True), k
