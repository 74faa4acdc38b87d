"""The feed-forward operators at the sizes that training and serving have: products whose k refills every
place in LDS several times, in each tile and each few-token form.

The bounds are those of test_gpu_q8, whose cases stay below all of that."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import oracle
import test_gpu_q8 as q8
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
