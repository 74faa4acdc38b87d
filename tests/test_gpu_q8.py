"""GPU parity of the 8-bit rows, through the C ABI, against the fp64 oracle.

Bounds (u = 2^-24): rows of values as they are, and sums of products, are exact.  exp2 of an argument a
is off by (2 + 1.5 |a|) u of itself, a reciprocal by 2 u; with a at most 2 |z| for SILU and up to
2.4 |z| (1 + 0.05 z^2) for GELU:
  act(z)    |z| s with s = 1 / (1 + e): the error of e changes s by a factor e s <= 1 of it, and where the
            argument is large and positive e s^2 falls as exp(-a): |z| u (8 + 2 max(a e^-a)) < 16 u |z|
  act'(z)   s and z e s^2 (..): the same terms, below 64 u (1 + |z| e^-|z| ..) < 128 u
  z' = q scale is one rounding of fp32 in the call and none in the oracle: it moves act by 2 u |z|
  gated and times gh: products of these, 4 roundings
  dbias     over T tokens in any order: (T + 16) u of the sum of magnitudes, and the terms' errors
  a product rounds the sum once, two products with scales, a sum with the bias: 4 u of the magnitudes;
            GELU has a slope below 1.13
A bf16 output adds half a unit of its own."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import oracle
from ffn_common import U, blank, close, code, down, draw, untouched, up
from helpers import values

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"


@pytest.fixture(scope="module")
def tpp():
    import paper_2104_05755_amd as tpp
    return tpp


def act_code(tpp, act):
    return dict(none=tpp.TPP_ACT_NONE, relu=tpp.TPP_ACT_RELU, gelu_tanh=tpp.TPP_ACT_GELU_TANH,
                silu=tpp.TPP_ACT_SILU)[act]


# tokens, features, group, dtype, act, gated, extra ld, first entry
ROWS = [
    (1, 1, 0, "f32", "none", 0, 0, 0),
    (3, 7, 0, "bf16", "silu", 1, 0, 0),
    (3, 8, 16, "bf16", "relu", 0, 0, 0),
    (5, 9, 16, "f32", "gelu_tanh", 1, 1, 1),
    (1, 1024, 0, "bf16", "none", 0, 0, 0),
    (9, 64, 32, "bf16", "gelu_tanh", 1, 0, 0),
    (9, 100, 32, "bf16", "silu", 1, 4, 0),
    (9, 104, 64, "f32", "silu", 1, 0, 0),
    (33, 1001, 64, "f32", "silu", 1, 1, 0),
    (33, 1001, 0, "bf16", "gelu_tanh", 0, 0, 1),
    (33, 1000, 512, "bf16", "relu", 1, 0, 0),
    (17, 2048, 128, "bf16", "gelu_tanh", 0, 0, 0),
    (17, 2056, 256, "f32", "none", 0, 8, 0),
    (7, 4096, 128, "bf16", "silu", 1, 0, 0),
    (7, 4096, 0, "f32", "silu", 1, 0, 0),
    (5, 8192, 0, "bf16", "silu", 1, 0, 0),
    (5, 8184, 128, "f32", "gelu_tanh", 0, 0, 0),
    (3, 16384, 0, "bf16", "gelu_tanh", 1, 0, 0),
    (3, 16384, 0, "f32", "silu", 1, 0, 0),
    (2, 40000, 0, "bf16", "silu", 1, 0, 0),
    (2, 30000, 0, "f32", "gelu_tanh", 0, 0, 0),
    (2, 16001, 32, "bf16", "silu", 1, 0, 0),
    (2, 15000, 512, "f32", "silu", 1, 0, 1),
    (2, 33000, 32, "f32", "relu", 1, 0, 0),
    (1500, 72, 0, "bf16", "silu", 0, 0, 0),
    (1500, 40, 16, "f32", "gelu_tanh", 1, 0, 0),
    (600, 640, 64, "bf16", "silu", 1, 0, 0),
]
IDS = ["-".join(map(str, c)) for c in ROWS]


class Rows:
    def __init__(self, case, seed=0):
        self.T, self.F, self.group, self.dtype, self.act, self.gated, self.pad, self.first = case
        rng = np.random.default_rng(seed + self.T * 17 + self.F)
        self.W = self.F << self.gated
        self.z = draw(rng, self.T, self.W, self.W + self.pad, self.dtype)
        self.z[2::6, :self.W] = 0
        self.gh = draw(rng, self.T, self.F, self.F + self.pad, self.dtype)

    def desc(self, tpp):
        return tpp.tpp_q8_desc(self.F, self.group, code(tpp, self.dtype), act_code(tpp, self.act), self.gated)

    def groups(self, width):
        return -(-width // self.group) if self.group else 1

    def room(self, width):
        return (torch.full((self.T, width + 5), 77, dtype=torch.int8, device="cuda"),
                torch.full((self.T, self.groups(width) + 1), 55.0, device="cuda"))

    def h(self, z):
        """h and the bound of its error, from values z of the whole row."""
        if not self.gated:
            return oracle.act(z, self.act)[0], 16 * U * np.abs(z)
        a, u = z[:, :self.F], z[:, self.F:]
        return oracle.act(a, self.act)[0] * u, 20 * U * np.abs(a * u)


def check_rows(q, s, v, group, width):
    want, scale = oracle.q8_rows(v, group)
    assert np.array_equal(q[:, :width], want), f"{(q[:, :width] != want).sum()} entries differ"
    assert np.array_equal(s[:, :scale.shape[1]], scale, equal_nan=True)
    assert (q[:, width:] == 77).all() and (s[:, scale.shape[1]:] == 55.0).all()


@pytest.mark.parametrize("case", ROWS, ids=IDS)
def test_act_and_backward(tpp, case):
    c = Rows(case)
    z, h = up(c.z, c.first), blank(c.T, c.F + c.pad, c.dtype, c.first)
    q, s = c.room(c.W)
    st = tpp.current_stream()
    tpp.tpp_q8_act(c.desc(tpp), c.T, z, c.W + c.pad, h, c.F + c.pad, q, c.W + 5, s, s.shape[1], st)
    q2, s2 = c.room(c.W)
    tpp.tpp_q8_act(c.desc(tpp), c.T, z, c.W + c.pad, None, 0, q2, c.W + 5, s2, s.shape[1], st)
    qh, sh, hh = down(q), down(s), down(h)
    zv = values(c.z, c.dtype)[:, :c.W]
    check_rows(qh, sh, zv, c.group, c.W)
    assert torch.equal(q, q2) and torch.equal(s, s2)
    ref, err = c.h(zv)
    close(hh[:, :c.F], ref, err, "h")
    assert untouched(hh, c.F)

    outs = lambda: (blank(c.T, c.W + c.pad, c.dtype, c.first), blank(c.T, c.F + c.pad, c.dtype, c.first),
                    blank(1, c.W, "f32"))
    gh = up(c.gh, c.first)
    back = lambda dz, h2, db, g=None: tpp.tpp_q8_act_backward(
        c.desc(tpp), c.T, q, c.W + 5, s, s.shape[1], gh if g is None else g, c.F + c.pad, dz, c.W + c.pad, h2,
        c.F + c.pad, db, st)
    dz, h2, db = outs()
    back(dz, h2, db)
    got = [down(t) for t in (dz, h2, db)]
    scale = np.repeat(sh[:, :c.groups(c.W)].astype(np.float64), c.group or c.W, 1)[:, :c.W]
    zq = qh[:, :c.W] * scale
    g = values(c.gh, c.dtype)[:, :c.F]
    ref, err = c.h(zq)
    close(got[1][:, :c.F], ref, err + 4 * U * np.abs(ref) + 4 * U * np.abs(zq[:, :c.F]) * (
        np.abs(zq[:, c.F:]) if c.gated else 1), "h2")
    value, slope = oracle.act(zq[:, :c.F], c.act)
    A = np.abs
    if c.gated:
        u = zq[:, c.F:]
        ref = np.concatenate([g * u * slope, g * value], 1)
        err = np.concatenate([A(g * u) * 136 * U, A(g * zq[:, :c.F]) * 24 * U], 1)
    else:
        ref, err = g * slope, A(g) * 132 * U
    close(got[0][:, :c.W], ref, err, "dz")
    close(got[2][:, :c.W], ref.sum(0)[None], ((c.T + 16) * U * A(ref).sum(0) + err.sum(0))[None], "dbias")
    assert untouched(got[0], c.W) and untouched(got[1], c.F)
    # one by one, and h2 over gh
    for k in range(3):
        one = list(outs())
        back(*[t if i == k else None for i, t in enumerate(one)])
        assert np.array_equal(down(one[k]), got[k], equal_nan=True)
    g2, dz2 = up(c.gh, c.first), outs()[0]
    back(dz2, g2, None, g2)
    assert np.array_equal(down(g2)[:, :c.F], got[1][:, :c.F]) and np.array_equal(down(dz2), got[0], equal_nan=True)


@pytest.mark.parametrize("case", ROWS, ids=IDS)
def test_quantize(tpp, case):
    c = Rows(case, 3)
    z, (q, s) = up(c.z, c.first), c.room(c.F)
    tpp.tpp_q8_quantize(c.desc(tpp), c.T, z, c.W + c.pad, q, c.F + 5, s, s.shape[1], tpp.current_stream())
    qh, sh = down(q), down(s)
    zv = values(c.z, c.dtype)[:, :c.W]
    ref, err = c.h(zv)
    if c.act in ("none", "relu") and (c.dtype == "f32" or not c.gated):
        exact = ref.astype(np.float32).astype(np.float64)   # one product of fp32 at most, rounded once
        check_rows(qh, sh, exact, c.group, c.F)
        return
    # scales and values within the error of h and half a step
    if c.dtype == "bf16":
        err = err + (np.abs(ref) + err) * 2.0 ** -8
    else:
        err = err + np.abs(ref) * U
    g = c.group or c.F
    for j in range(c.groups(c.F)):
        part = slice(j * g, min(c.F, (j + 1) * g))
        top, e = np.abs(ref[:, part]).max(1), err[:, part].max(1)
        sc = sh[:, j].astype(np.float64)
        assert (np.abs(sc - top / 127) <= e / 127 + 2 * U * top / 127).all()
        back = qh[:, part] * sc[:, None]
        assert (np.abs(back - ref[:, part]) <= err[:, part] + sc[:, None] * (0.5 + 130 * U) + 1e-37).all()
        assert ((np.abs(qh[:, part]).max(1) == 127) | (top == 0)).all()
    assert (qh[:, c.F:] == 77).all() and (sh[:, c.groups(c.F):] == 55.0).all()


def test_rows_at_the_borders(tpp):
    """Ties, groups far out in fp32's range, and groups with infinities and NaN."""
    rng = np.random.default_rng(5)
    v = np.zeros((10, 256), np.float32)
    v[0] = np.arange(256) * 0.5 - 64                       # halves: ties to even
    v[0, 0] = 127
    v[1] = rng.standard_normal(256) * 1e-42                # below the normal numbers
    v[2] = rng.standard_normal(256) * 1e38
    v[2, 9] = 3.4028235e38
    v[3, 5] = 1e-45                                        # alone
    v[4], v[5] = rng.standard_normal((2, 256))
    v[4, 40], v[5, 200] = np.inf, np.nan
    v[6] = -0.0
    k = np.arange(256) - 128                               # just beside (k + 1/2) / 127 of the largest
    v[7] = np.nextafter(((k + 0.5) * np.float32(0.7) / 127).astype(np.float32), np.float32(np.inf))
    v[7, 0] = 0.7
    v[8] = np.nextafter(((k + 0.5) * np.float32(1.9e-30) / 127).astype(np.float32), np.float32(-np.inf))
    v[8, :128] = 0
    v[8, 0] = 1.9e-30
    v[9, 3] = -np.inf
    v[7] = np.clip(v[7], -0.7, 0.7)
    v[8] = np.clip(v[8], -1.9e-30, 1.9e-30)
    for group in (0, 16, 64):
        d = tpp.tpp_q8_desc(256, group, tpp.TPP_DT_F32, tpp.TPP_ACT_NONE, 0)
        q = torch.full((10, 261), 77, dtype=torch.int8, device="cuda")
        s = torch.full((10, (256 // group if group else 1) + 1), 55.0, device="cuda")
        tpp.tpp_q8_quantize(d, 10, up(v), 256, q, 261, s, s.shape[1], tpp.current_stream())
        check_rows(down(q), down(s), v.astype(np.float64), group, 256)


# m, n, k, extra lda, ldb, ldc, first bytes of a and b, c type, flags
PRODUCTS = [
    (1, 1, 1, 0, 0, 0, 0, "f32", ()),
    (4, 1, 16, 0, 0, 0, 0, "bf16", ("bias",)),
    (5, 3, 15, 1, 1, 1, 0, "f32", ("bias", "relu")),
    (64, 1, 1024, 0, 0, 0, 0, "bf16", ()),
    (100, 2, 1000, 8, 8, 0, 0, "bf16", ("gelu_tanh",)),
    (257, 5, 300, 4, 4, 3, 0, "f32", ("bias", "gelu_tanh")),
    (300, 16, 129, 15, 15, 1, 0, "bf16", ("bias",)),
    (16, 17, 64, 0, 0, 0, 0, "f32", ()),
    (130, 33, 96, 0, 0, 0, 0, "f32", ("relu",)),
    (192, 48, 2000, 0, 0, 0, 0, "bf16", ()),
    (1000, 64, 512, 0, 0, 8, 0, "bf16", ("bias",)),
    (129, 65, 272, 0, 0, 0, 0, "f32", ("bias",)),
    (256, 100, 4096, 0, 0, 0, 0, "bf16", ("bias", "relu")),
    (777, 153, 1001, 7, 7, 0, 0, "f32", ("bias", "relu")),
    (512, 512, 256, 0, 0, 0, 0, "bf16", ("gelu_tanh", "bias")),
    (520, 300, 1040, 16, 32, 6, 0, "bf16", ()),
    (1032, 1100, 384, 0, 0, 0, 0, "bf16", ("bias",)),
    (1031, 1090, 400, 0, 16, 1, 0, "f32", ("bias", "gelu_tanh")),
    (2048, 2300, 128, 0, 0, 0, 0, "bf16", ()),
    (2050, 2048, 144, 0, 0, 2, 0, "f32", ("relu",)),
    (192, 600, 1300, 12, 12, 0, 0, "bf16", ("gelu_tanh",)),   # few tiles: shares of k
    (16, 900, 2283, 5, 5, 0, 0, "f32", ("bias",)),
    (581, 4200, 200, 8, 8, 3, 0, "bf16", ("bias",)),          # many small tiles
    (4100, 3900, 130, 14, 14, 0, 0, "bf16", ("bias", "relu")),  # large tiles with tails each way
    (130, 70, 333, 0, 0, 0, 3, "f32", ("bias",)),     # bases and rows at any byte
    (40, 9, 4100, 1, 2, 0, 1, "bf16", ()),
    (33, 200, 64, 0, 0, 0, 4, "f32", ()),
    (3, 2, 131071, 1, 1, 0, 0, "f32", ()),
]


class Product:
    def __init__(self, case, seed=0):
        self.m, self.n, self.k, pa, pb, pc, self.first, self.ctype, self.flags = case
        rng = np.random.default_rng(seed + self.m + self.n * 7)
        self.a = rng.integers(-128, 128, (self.m, self.k + pa)).astype(np.int8)   # behind k too
        self.b = rng.integers(-127, 128, (self.n, self.k + pb)).astype(np.int8)
        self.sa = rng.uniform(0.5, 2, self.m).astype(np.float32) / 4096
        self.sb = rng.uniform(0.5, 2, self.n).astype(np.float32)
        self.sb[3::5] = 0
        self.bias = rng.standard_normal(self.m).astype(np.float32)
        self.ldc = self.m + pc

    def desc(self, tpp, btype="f32", **kw):
        fl = dict(bias=tpp.TPP_EPI_BIAS, relu=tpp.TPP_EPI_RELU, gelu_tanh=tpp.TPP_EPI_GELU_TANH)
        d = dict(m=self.m, n=self.n, k=self.k, lda=self.a.shape[1], ldb=self.b.shape[1], ldc=self.ldc,
                 b_type=code(tpp, btype), c_type=code(tpp, self.ctype), flags=sum(fl[f] for f in self.flags))
        return tpp.tpp_q8_gemm_desc(**dict(d, **kw))

    def run(self, tpp, **kw):
        c = blank(self.n, self.ldc, self.ctype)
        tpp.tpp_q8_gemm(self.desc(tpp, **kw), up(self.a, self.first), up(self.sa), up(self.b, self.first),
                        up(self.sb), c, up(self.bias) if "bias" in self.flags else None, tpp.current_stream())
        return down(c)

    def finish(self, total, sb):
        """C and its error from exact sums [n][m] and the tokens' scales."""
        v = total.astype(np.float64) * sb.astype(np.float64)[:, None] * self.sa.astype(np.float64)
        err = 4 * U * np.abs(v)
        if "bias" in self.flags:
            v = v + self.bias
            err = err + U * np.abs(v)
        if "relu" in self.flags:
            v = np.where(v > 0, v, 0)
        if "gelu_tanh" in self.flags:
            err = 1.13 * err + 16 * U * np.abs(v)
            v = oracle.act(v, "gelu_tanh")[0]
        return v, err


@pytest.mark.parametrize("case", PRODUCTS, ids=str)
def test_product(tpp, case):
    p = Product(case)
    c = p.run(tpp)
    total = oracle.q8_product(p.a, p.b, p.k)
    close(c[:, :p.m], *p.finish(total, p.sb), "c")
    assert untouched(c, p.m)
    if p.ctype == "f32":   # scales of 1 and no epilogue: the sums themselves
        p.flags, p.sa[:], p.sb[:] = (), 1, 1
        assert np.array_equal(p.run(tpp)[:, :p.m], total.astype(np.float32))


LINEAR = [c for c in PRODUCTS if c[2] < 5000]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", LINEAR + [
    (700, 16, 760, 8, 0, 0, 0, "bf16", ("bias",)), (700, 17, 760, 8, 0, 0, 0, "f32", ()),   # one launch, and two
    (6200, 3, 4000, 0, 3, 5, 0, "bf16", ("gelu_tanh",)), (50, 1, 12288, 0, 0, 0, 0, "f32", ())], ids=str)
def test_linear(tpp, case, dtype):
    p = Product(case, 1)
    rng = np.random.default_rng(2)
    ldx = p.b.shape[1]
    x = draw(rng, p.n, p.k, ldx, dtype)
    x[4::7, :p.k] = 0
    first = 1 if p.first else 0
    c = blank(p.n, p.ldc, p.ctype)
    tpp.tpp_q8_linear(p.desc(tpp, dtype), up(p.a, p.first), up(p.sa), up(x, first), c,
                      up(p.bias) if "bias" in p.flags else None, tpp.current_stream())
    c = down(c)
    q, s = oracle.q8_rows(values(x, dtype)[:, :p.k])
    close(c[:, :p.m], *p.finish(oracle.q8_product(p.a, q, p.k), s[:, 0]), "c")
    assert untouched(c, p.m)


def test_tokens_without_a_scale(tpp):
    """An infinity or NaN in a token makes its whole column NaN (0 behind RELU), and no other."""
    rng = np.random.default_rng(7)
    for n in (3, 70):
        x = draw(rng, n, 200, 200, "f32")
        a = rng.integers(-127, 128, (96, 208)).astype(np.int8)
        sa = np.full(96, 0.01, np.float32)
        x[1, 7], x[2, 9] = np.inf, np.nan
        for flags in (0, tpp.TPP_EPI_RELU):
            d = tpp.tpp_q8_gemm_desc(96, n, 200, 208, 200, 96, tpp.TPP_DT_F32, tpp.TPP_DT_F32, flags)
            c = blank(n, 96, "f32")
            tpp.tpp_q8_linear(d, up(a), up(sa), up(x), c, None, tpp.current_stream())
            c = down(c)
            assert (np.isnan(c[1:3]) if not flags else c[1:3] == 0).all()
            assert np.isfinite(np.delete(c, [1, 2], 0)).all()


def test_groups_without_a_scale(tpp):
    c = Rows((4, 96, 32, "bf16", "silu", 1, 0, 0), 9)
    c.z[1, 40], c.z[2, 100] = 0x7F80, 0x7FC0
    q, s = c.room(c.W)
    st = tpp.current_stream()
    tpp.tpp_q8_act(c.desc(tpp), 4, up(c.z), c.W, None, 0, q, c.W + 5, s, s.shape[1], st)
    check_rows(down(q), down(s), values(c.z, "bf16"), 32, c.W)
    for act in ("silu", "gelu_tanh", "none"):
        c.act = act
        dz, h2 = blank(4, c.W, "bf16"), blank(4, c.F, "bf16")
        tpp.tpp_q8_act_backward(c.desc(tpp), 4, q, c.W + 5, s, s.shape[1], up(c.gh), c.F, dz, c.W, h2, c.F, None, st)
        h2, dz = values(down(h2), "bf16"), values(down(dz), "bf16")
        assert np.isnan(h2[1, 32:64]).all() and np.isnan(h2[2, :32]).all()
        assert np.isnan(dz[1, 128:160]).all() and np.isnan(dz[2, :32]).all()
        assert np.isfinite(h2[[0, 3]]).all() and np.isfinite(dz[[0, 3]]).all()
        assert np.isfinite(h2[1, :32]).all() and np.isfinite(h2[2, 32:]).all()


def test_streams_and_graphs(tpp):
    """Captured calls, replayed while the stream's own work buffer grows and is used."""
    p = Product((300, 90, 700, 0, 0, 0, 0, "f32", ()), 3)
    rng = np.random.default_rng(4)
    x = up(draw(rng, 90, 700, 700, "bf16"))
    a, sa, c = up(np.pad(p.a, ((0, 0), (0, 4)))), up(p.sa), blank(90, 300, "f32")
    d = p.desc(tpp, "bf16", lda=704)
    k = Rows((500, 300, 64, "bf16", "silu", 1, 0, 0), 5)
    z, gh, (q, s) = up(k.z), up(k.gh), k.room(k.W)
    dz, db = blank(500, 600, "bf16"), blank(1, 600, "f32")

    def calls(st):
        tpp.tpp_q8_linear(d, a, sa, x, c, None, st)
        tpp.tpp_q8_act(k.desc(tpp), 500, z, 600, None, 0, q, 605, s, s.shape[1], st)
        tpp.tpp_q8_act_backward(k.desc(tpp), 500, q, 605, s, s.shape[1], gh, 300, dz, 600, None, 0, db, st)

    calls(tpp.current_stream())
    torch.cuda.synchronize()
    want = [t.clone() for t in (c, q, s, dz, db)]
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        calls(st.cuda_stream)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=st):
        calls(st.cuda_stream)
    big = up(draw(rng, 900, 704, 704, "bf16"))
    cb = blank(900, 300, "f32")
    for _ in range(3):
        for t in (c, q, s, dz, db):
            t.zero_()
        q.fill_(77)
        s.fill_(55.0)
        g.replay()
        tpp.tpp_q8_linear(p.desc(tpp, "bf16", lda=704, n=900, ldb=704), a, sa, big, cb, None, st.cuda_stream)
        g.replay()
        torch.cuda.synchronize()
        for t, w in zip((c, q, s, dz, db), want):
            assert torch.equal(t.view(torch.int8), w.view(torch.int8))


def test_no_tokens(tpp):
    db = torch.full((128,), 7.0, device="cuda")
    d = tpp.tpp_q8_desc(64, 0, 1, 3, 1)
    tpp.tpp_q8_act_backward(d, 0, None, 128, None, 1, None, 64, None, 128, None, 64, db, tpp.current_stream())
    assert (db == 0).all()


def test_past_32_bits(tpp):
    """Weights, tokens and outputs past 2^32 bytes from their blocks' first entries."""
    ld = (1 << 32) + 16
    p = Product((3, 2, 64, 0, 0, 0, 0, "f32", ()), 6)
    a, b = (torch.zeros(3 * ld, dtype=torch.int8, device="cuda") for _ in range(2))
    for dst, src in ((a, p.a), (b, p.b)):
        for i, row in enumerate(src):
            dst[i * ld:i * ld + 64] = up(row)
    c = torch.zeros((1 << 30) + 64, device="cuda")
    ldc = 1 << 30
    tpp.tpp_q8_gemm(p.desc(tpp, lda=ld, ldb=ld, ldc=ldc), a, up(p.sa), b, up(p.sb), c, None, tpp.current_stream())
    ref, err = p.finish(oracle.q8_product(p.a, p.b, 64), p.sb)
    close(np.stack([down(c[j * ldc:j * ldc + 3]) for j in range(2)]), ref, err, "c")
    del a, b, c
    k = Rows((3, 40, 0, "bf16", "silu", 1, 0, 0), 7)
    ldz = (1 << 31) + 8
    z = torch.zeros(2 * ldz + 80, dtype=torch.bfloat16, device="cuda")
    q = torch.zeros(2 * ld + 80, dtype=torch.int8, device="cuda")
    for t in range(3):
        z[t * ldz:t * ldz + 80] = up(k.z)[t].view(torch.bfloat16)
    s = torch.zeros(3, device="cuda")
    tpp.tpp_q8_act(k.desc(tpp), 3, z, ldz, None, 0, q, ld, s, 1, tpp.current_stream())
    want, scale = oracle.q8_rows(values(k.z, "bf16"))
    assert np.array_equal(down(s), scale[:, 0])
    for t in range(3):
        assert np.array_equal(down(q[t * ld:t * ld + 80]), want[t])
