"""GPU parity of the residual stream's norms, through the C ABI, against the fp64 oracle.

Bounds on the errors, from the arithmetic (u = 2^-24, fp32's half unit; s = (16 + F / 64) u, a sum of F
terms by at least 64 lanes and then pairwise, relative to the sum of their magnitudes):
  a norm     mean: s mean|v| =: m; 1 / sqrt(mean d^2 + eps): relative (s + 2 m rs + 8 u), the change of d by m
             among it; so vn = (v - mean) rs is off by rs (m + u |v|) + |vn| (s + 2 m rs + 8 u), times |w|
  r          scale G n: that of n, of G (8 u (1 + |g|)), 4 roundings, one of the sum
  dx         N'(g) is linear in u = g w, with vn, mean(u vn) and mean(u): each product has the error of vn
             (e) and 8 u; a sum of F terms s: rs (|u| (12 u + s + e) + |vn| c2 + e mean|u vn| + s mean|u|),
             c2 = mean(|u| (|vn| (8 u + s) + e))
  db         the same of its input's error, which passes through N' with a gain of rs |w| and the means
  sums       over T tokens in any order: (T + 16) u of the sum of magnitudes, and the sum of the terms' errors
A bf16 output adds half a unit of its own, 2^-8 of its value at most.  y is compared with the norm of the
r that the call stored, 8-bit rows with the exact rows of the y that it stored."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import oracle
from ffn_common import U, blank, close, code, down, draw, typed, untouched, up
from helpers import values

pytestmark = pytest.mark.gpu
EPS = 1e-5


@pytest.fixture(scope="module", autouse=True)
def gpu():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"


@pytest.fixture(scope="module")
def tpp():
    import paper_2104_05755_amd as tpp
    return tpp


# tokens, features, after, before, gate, gate_every, dtype, gate type, extra ld, first entry
CASES = [
    (1, 1024, "rms", "rms", "none", 0, "bf16", "f32", 0, 0),
    (3, 1, "rms", "layer", "identity", 0, "f32", "f32", 0, 0),
    (5, 2, "layer", "layer", "tanh", 2, "bf16", "bf16", 1, 1),
    (5, 7, "layer", "rms", "sigmoid", 1, "f32", "f32", 0, 0),
    (5, 8, "rms", "rms", "identity", 0, "bf16", "f32", 0, 0),
    (9, 9, "rms", "layer", "identity", 4, "bf16", "bf16", 0, 1),
    (70, 64, "none", "rms", "sigmoid", 7, "bf16", "bf16", 0, 0),
    (70, 64, "rms", "none", "tanh", 0, "f32", "f32", 5, 0),
    (33, 511, "layer", "layer", "identity", 1, "bf16", "bf16", 0, 0),
    (33, 512, "rms", "rms", "identity", 0, "bf16", "f32", 8, 0),
    (33, 513, "rms", "rms", "none", 0, "f32", "f32", 3, 1),
    (300, 520, "layer", "rms", "tanh", 100, "bf16", "bf16", 0, 0),
    (133, 1001, "layer", "layer", "tanh", 100, "f32", "f32", 3, 0),
    (40, 1024, "rms", "rms", "identity", 0, "bf16", "f32", 0, 0),
    (40, 1025, "rms", "layer", "identity", 16, "bf16", "bf16", 0, 0),
    (21, 2047, "none", "layer", "none", 0, "bf16", "f32", 0, 0),
    (21, 2048, "rms", "rms", "sigmoid", 0, "f32", "f32", 0, 0),
    (19, 4096, "rms", "rms", "identity", 0, "bf16", "f32", 0, 0),
    (19, 4104, "layer", "layer", "identity", 6, "f32", "bf16", 0, 0),
    (6, 8192, "layer", "rms", "tanh", 0, "bf16", "f32", 0, 0),
    (6, 8191, "rms", "rms", "identity", 2, "f32", "f32", 5, 0),
    (5, 8200, "rms", "layer", "identity", 2, "bf16", "bf16", 0, 0),
    (4, 16384, "rms", "rms", "identity", 0, "bf16", "f32", 0, 0),
    (4, 16383, "layer", "layer", "sigmoid", 3, "f32", "f32", 1, 0),
    (3, 20001, "layer", "layer", "tanh", 2, "bf16", "f32", 0, 0),
    (2, 70000, "rms", "rms", "identity", 0, "f32", "f32", 0, 0),
    (2600, 72, "rms", "rms", "identity", 0, "bf16", "f32", 0, 0),
    (2600, 72, "layer", "layer", "tanh", 1, "bf16", "bf16", 0, 0),
    (2600, 200, "layer", "rms", "identity", 300, "f32", "f32", 0, 0),
    (1100, 1024, "rms", "layer", "identity", 1000, "bf16", "f32", 0, 0),
]
IDS = ["-".join(map(str, c)) for c in CASES]


class Case:
    def __init__(self, case, seed=0, mean=0.3):
        (self.T, self.F, self.after, self.before, self.gate, self.every, self.dtype, self.gtype, pad,
         self.first) = case
        rng = np.random.default_rng(seed + self.T * 131 + self.F)
        self.ld, self.scale = self.F + pad, 0.7
        rows = lambda std: draw(rng, self.T, self.F, self.ld, self.dtype, std, mean)
        self.x, self.b = rows(1.0), rows(2.0)
        self.x[2::7, :self.F] = 0
        self.b[2::5, :self.F] = 0          # padding tokens
        vec = lambda want, m: (m + 0.2 * rng.standard_normal(self.F)).astype(np.float32) if want else None
        self.wa, self.ca = vec(self.after != "none", 1), vec(self.after == "layer", 0)
        self.wb, self.cb = vec(self.before != "none", 1), vec(self.before == "layer", 0)
        n = -(-self.T // self.every) if self.every else 1
        self.g = None if self.gate == "none" else draw(rng, n, self.F, self.F + 2, self.gtype, 0.5)
        self.gr, self.gy = rows(1.0), rows(1.0)

    def desc(self, tpp):
        norm = dict(none=tpp.TPP_NORM_NONE, rms=tpp.TPP_NORM_RMS, layer=tpp.TPP_NORM_LAYER)
        gate = dict(none=tpp.TPP_GATE_NONE, identity=tpp.TPP_GATE_IDENTITY, sigmoid=tpp.TPP_GATE_SIGMOID,
                    tanh=tpp.TPP_GATE_TANH)
        return tpp.tpp_residual_desc(self.F, code(tpp, self.dtype), norm[self.after], norm[self.before],
                                     gate[self.gate], code(tpp, self.gtype), self.scale, EPS, self.every)

    def gates(self):
        """G(g) and G'(g) of every token, and the gates' own rows of G'."""
        if self.g is None:
            return np.ones((1, self.F)), None, None
        g = values(self.g, self.gtype)[:, :self.F]
        v = dict(identity=lambda: g, sigmoid=lambda: 1 / (1 + np.exp(-g)), tanh=lambda: np.tanh(g))[self.gate]()
        d = dict(identity=lambda: np.ones_like(g), sigmoid=lambda: v * (1 - v),
                 tanh=lambda: 1 / np.cosh(g) ** 2)[self.gate]()
        row = np.arange(self.T) // self.every if self.every else np.zeros(self.T, np.int64)
        return v[row], d, row


def norm_error(v, form, w):
    """(vn, rs, error of vn, error of the norm without its shift) of rows v (float64)."""
    T, F = v.shape
    s = (16 + F / 64) * U
    if form == "none":
        return v, np.ones((T, 1)), 0 * v, 0 * v
    m = s * np.abs(v).mean(1, keepdims=True) if form == "layer" else np.zeros((T, 1))
    d = v - v.mean(1, keepdims=True) if form == "layer" else v
    rs = 1 / np.sqrt((d * d).mean(1, keepdims=True) + EPS)
    vn = d * rs
    e = rs * (m + U * np.abs(v)) + np.abs(vn) * (s + 2 * m * rs + 8 * U)
    return vn, rs, e, e * np.abs(w)


def forward(tpp, c, in_place=False, y=True, q=True, stream=None):
    f, n = c.first, c.T
    x, b = up(c.x, f), up(c.b, f)
    r = x if in_place else blank(n, c.ld, c.dtype, f)
    yy = None if not y else b if in_place else blank(n, c.ld, c.dtype, f)
    qq = torch.full((n, c.F + 3), 77, dtype=torch.int8, device="cuda") if q else None
    qs = torch.full((n + 1,), 55.0, device="cuda") if q else None
    gate, vecs = up(c.g), [up(a) for a in (c.wa, c.ca, c.wb, c.cb)]
    tpp.tpp_residual_norm(c.desc(tpp), n, x, c.ld, b, c.ld, gate, c.F + 2, *vecs, r, c.ld, yy, c.ld, qq,
                          c.F + 3, qs, stream or tpp.current_stream())
    torch.cuda.synchronize()
    return [None if t is None else down(t) for t in (r, yy, qq, qs)]


def check_forward(c, r, y, q, qs):
    x, b = (values(a, c.dtype)[:, :c.F] for a in (c.x, c.b))
    G, _, _ = c.gates()
    n = oracle.norm(c.b, c.F, c.dtype, c.after, EPS, c.wa, c.ca)
    err = norm_error(b, c.after, 1.0 if c.wa is None else c.wa)[3] + 4 * U * (np.abs(n) + 1)
    gin = 0 if c.g is None else np.abs(values(c.g, c.gtype)[:, :c.F]).max()
    add = c.scale * G * n
    close(r[:, :c.F], x + add, c.scale * np.abs(G) * err + np.abs(add) * U * (12 + 8 * gin), "r")
    assert untouched(r, c.F)
    if y is not None:
        rr = values(r, c.dtype)[:, :c.F]
        ref = oracle.norm(r, c.F, c.dtype, c.before, EPS, c.wb, c.cb)
        close(y[:, :c.F], ref, norm_error(rr, c.before, 1.0 if c.wb is None else c.wb)[3] +
              4 * U * (np.abs(ref) + 1), "y")
        assert untouched(y, c.F)
        if q is not None:
            want, scale = oracle.q8_rows(values(y, c.dtype)[:, :c.F])
            assert np.array_equal(q[:, :c.F], want) and np.array_equal(qs[:c.T], scale[:, 0])
            assert (q[:, c.F:] == 77).all() and qs[c.T] == 55.0


@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_forward(tpp, case):
    c = Case(case)
    r, y, q, qs = forward(tpp, c)
    check_forward(c, r, y, q, qs)
    r2, y2, _, _ = forward(tpp, c, in_place=True, q=False)
    assert np.array_equal(r2[:, :c.F], r[:, :c.F]) and np.array_equal(y2[:, :c.F], y[:, :c.F])
    assert untouched(r2, c.F) and untouched(y2, c.F)
    r3, _, q3, qs3 = forward(tpp, c, y=False)
    same = lambda a, b: np.array_equal(a, b, equal_nan=True)
    assert same(r3, r) and same(q3, q) and same(qs3, qs)
    assert same(forward(tpp, c, y=False, q=False)[0], r)


def backward(tpp, c, r, gr=True, gy=True, want=None, stream=None, keep=None):
    """All gradients, or those of `want`; the device tensors in `keep` (a dict) for later calls."""
    f, n, F = c.first, c.T, c.F
    dev = dict(b=up(c.b, f), gate=up(c.g), wa=up(c.wa), ca=up(c.ca), wb=up(c.wb), r=up(r, f),
               gr=up(c.gr, f) if gr else None, gy=up(c.gy, f) if gy else None)
    out = dict(dx=blank(n, c.ld, c.dtype, f), db=blank(n, c.ld, c.dtype, f),
               dgate=None if c.g is None else blank(len(c.g), F + 2, c.gtype))
    for k, a in (("dw_after", c.wa), ("dc_after", c.ca), ("dw_before", c.wb), ("dc_before", c.cb)):
        out[k] = None if a is None else blank(1, F, "f32")
    if want is not None:
        out = {k: v if k in want else None for k, v in out.items()}
    call = lambda s: tpp.tpp_residual_norm_backward(
        c.desc(tpp), n, dev["b"], c.ld, dev["gate"], F + 2, dev["wa"], dev["ca"], dev["wb"], dev["r"], c.ld,
        dev["gr"], c.ld, dev["gy"], c.ld, out["dx"], c.ld, out["db"], c.ld, out["dgate"], F + 2,
        out["dw_after"], out["dc_after"], out["dw_before"], out["dc_before"], s)
    if keep is not None:
        keep.update(call=call, out=out, dev=dev)
    call(stream or tpp.current_stream())
    torch.cuda.synchronize()
    return {k: None if v is None else down(v) for k, v in out.items()}


def norm_backward_error(v, form, w, g, g_err):
    """Error of N'(g), of the sums g vn and g, for gradients g off by g_err."""
    T, F = v.shape
    if form == "none":
        return g_err + U * np.abs(g), None, None
    s, A = (16 + F / 64) * U, np.abs
    vn, rs, e, _ = norm_error(v, form, w)
    u = A(g) * A(w)
    ue = g_err * A(w)
    along = A((g * w * vn).mean(1, keepdims=True))
    c2 = (u * (A(vn) * (8 * U + s) + e) + ue * (A(vn) + e)).mean(1, keepdims=True)
    err = rs * ((u + ue) * (16 * U + s) + ue + u * e + A(vn) * (c2 + along * (s + 16 * U)) + e * (along + c2))
    if form == "layer":
        err = err + rs * (s * u + ue + 8 * U * u).mean(1, keepdims=True)
    total = (T + 16) * U * (A(g) * A(vn)).sum(0) + (A(g) * (e + 4 * U * A(vn)) + g_err * (A(vn) + e)).sum(0)
    return err, total, (T + 16) * U * A(g).sum(0) + g_err.sum(0)


def check_backward(c, r, got, gr=True, gy=True):
    F, T = c.F, c.T
    val = lambda a: values(a, c.dtype)[:, :F]
    zero = np.zeros((T, F))
    y = val(c.gy) if gy else zero
    rv, b = val(r), val(c.b)
    d, dwb, dcb = oracle.norm_backward(r, F, c.dtype, c.before, EPS, c.wb, y)
    wb, wa = (1.0 if a is None else a for a in (c.wb, c.wa))
    e_d, e_w, e_c = norm_backward_error(rv, c.before, wb, y, zero)
    dx = (val(c.gr) if gr else zero) + d
    e_x = e_d + 2 * U * (np.abs(dx) + np.abs(d))
    ref, err = dict(dx=dx, dw_before=dwb, dc_before=dcb), dict(dx=e_x, dw_before=e_w, dc_before=e_c)
    G, slope, row = c.gates()
    gin = 0 if c.g is None else np.abs(values(c.g, c.gtype)[:, :F]).max()
    g_rel = U * (8 + 8 * gin)
    dn = c.scale * dx
    n = oracle.norm(c.b, F, c.dtype, c.after, EPS, c.wa, c.ca)
    if c.g is not None:
        e_n = norm_error(b, c.after, wa)[3] + 4 * U * (np.abs(n) + 1)
        part, e_p = dn * n, c.scale * e_x * (np.abs(n) + e_n) + np.abs(dn) * (e_n + 4 * U * np.abs(n))
        k = len(c.g)
        ref["dgate"], mag, e_g = np.zeros((k, F)), np.zeros((k, F)), np.zeros((k, F))
        np.add.at(ref["dgate"], row, part)
        np.add.at(mag, row, np.abs(part))
        np.add.at(e_g, row, e_p)
        err["dgate"] = (e_g + (T + 16) * U * mag) * np.abs(slope) + np.abs(ref["dgate"]) * np.abs(slope) * U * (
            32 + 32 * gin)
        ref["dgate"] = ref["dgate"] * slope
    db, dwa, dca = oracle.norm_backward(c.b, F, c.dtype, c.after, EPS, c.wa, dn * G)
    e_db, e_wa, e_ca = norm_backward_error(b, c.after, wa, dn * G,
                                           np.abs(c.scale * G) * e_x + np.abs(dn * G) * (g_rel + 4 * U))
    ref.update(db=db, dw_after=dwa, dc_after=dca)
    err.update(db=e_db, dw_after=e_wa, dc_after=e_ca)
    for k, a in got.items():
        if a is None:
            continue
        rows = ref[k].reshape(-1, F)
        close(a[:, :F], rows, np.asarray(err[k]).reshape(-1, F), k)
        assert untouched(a, F), k


@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_backward(tpp, case):
    c = Case(case, 1)
    r = draw(np.random.default_rng(5), c.T, c.F, c.ld, c.dtype, 1.5, 0.2)
    got = backward(tpp, c, r)
    check_backward(c, r, got)
    again = backward(tpp, c, r)
    for k in got:
        assert got[k] is None or np.array_equal(got[k], again[k], equal_nan=True), k
    # outputs one by one, and without one of the gradients
    for want in ({"dx"}, {"db"}, {"dgate", "dw_before"}, {"dw_after", "dc_before"}):
        part = backward(tpp, c, r, want=want)
        for k in want:
            assert got[k] is None or np.array_equal(got[k], part[k], equal_nan=True), k
    check_backward(c, r, backward(tpp, c, r, gr=False), gr=False)
    check_backward(c, r, backward(tpp, c, r, gy=False), gy=False)


def test_gradients_by_differences(tpp):
    """The sum of P * r + Q * y of the forward call, at inputs moved by +-h, against the backward call.
    fp32: a difference is off by the forward's rounding, about 2^-20 of the terms over h, and by h^2."""
    c = Case((6, 40, "layer", "rms", "tanh", 3, "f32", "f32", 0, 0), 3, mean=0.0)
    rng = np.random.default_rng(4)
    c.b[2::5] = rng.standard_normal(c.b[2::5].shape)   # (a row of equal entries is no place for differences)
    P, Q = rng.standard_normal((2, c.T, c.F)).astype(np.float32)
    c.gr, c.gy = P, Q

    def value():
        r, y, _, _ = forward(tpp, c, q=False)
        return (P * r.astype(np.float64)).sum() + (Q * y.astype(np.float64)).sum()

    r0 = forward(tpp, c)[0]
    got = backward(tpp, c, r0)
    h = 2.0 ** -6
    for name, a, grad in (("x", c.x, got["dx"]), ("b", c.b, got["db"]), ("g", c.g, got["dgate"]),
                          ("wa", c.wa, got["dw_after"]), ("ca", c.ca, got["dc_after"]),
                          ("wb", c.wb, got["dw_before"])):
        flat = a.reshape(-1) if a.ndim == 1 else a
        for _ in range(6):
            at = (int(rng.integers(c.F)),) if a.ndim == 1 else (int(rng.integers(len(a))), int(rng.integers(c.F)))
            old = flat[at]
            flat[at] = old + np.float32(h)
            up_, hi = value(), float(flat[at])
            flat[at] = old - np.float32(h)
            lo_, lo = value(), float(flat[at])
            flat[at] = old
            est = (up_ - lo_) / (hi - lo)
            want = float(grad.reshape(-1)[at[0]] if a.ndim == 1 else grad[at])
            # terms: 240 of size ~3 rounded to 2^-24 and read twice, over 2 h = 2^-5; curvature ~ h^2 * 10
            assert abs(est - want) <= 240 * 3 * 2 * 2.0 ** -22 / 2.0 ** -5 + 10 * h * h * max(1, abs(want)), (name, at)


@pytest.mark.parametrize("f", [24, 1024, 9000])
@pytest.mark.parametrize("form", ["rms", "layer"])
def test_values_that_are_not_finite_stay_in_their_token(tpp, f, form):
    c = Case((5, f, form, form, "identity", 0, "bf16", "f32", 0, 0), 6)
    clean = forward(tpp, c)
    c.b[1, 3], c.x[3, 5] = 0x7F80, 0x7FC0          # an infinity, a NaN
    r, y, q, qs = forward(tpp, c)
    for t in (0, 2, 4):
        for a, ref in zip((r, y, q, qs), clean):
            assert np.array_equal(a[t], ref[t])
    assert np.isnan(values(y, "bf16")[[1, 3]]).all() and np.isnan(qs[[1, 3]]).all() and not q[[1, 3], :f].any()


def test_large_and_small_values(tpp):
    """Rows of 2^-40 and of 2^40: far from fp32's limits squared, the norms do not see the factor."""
    for k in (-40, 40):
        c = Case((4, 600, "rms", "rms", "none", 0, "f32", "f32", 0, 0), 7, mean=0.0)
        c.b *= np.float32(2.0 ** k)
        r, y, q, qs = forward(tpp, c)
        if k > 0:
            check_forward(c, r, y, q, qs)
        assert np.isfinite(y).all()


def test_streams_and_graphs(tpp):
    """A side stream; then forward and backward captured, replayed with other calls between."""
    c = Case((700, 1000, "rms", "layer", "identity", 300, "bf16", "bf16", 0, 0), 8)
    r = draw(np.random.default_rng(9), c.T, c.F, c.ld, c.dtype)
    want = backward(tpp, c, r)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    keep = {}
    with torch.cuda.stream(s):
        got = backward(tpp, c, r, stream=s.cuda_stream, keep=keep)
    for k in want:
        assert want[k] is None or np.array_equal(got[k], want[k], equal_nan=True), k
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        keep["call"](s.cuda_stream)
    bigger = Case((900, 3000, "rms", "layer", "identity", 300, "bf16", "bf16", 0, 0), 10)
    rb = draw(np.random.default_rng(11), bigger.T, bigger.F, bigger.ld, bigger.dtype)
    for _ in range(3):
        for t in keep["out"].values():
            if t is not None:
                t.fill_(0)
        g.replay()
        backward(tpp, bigger, rb, stream=s.cuda_stream)    # grows the stream's own work buffer
        g.replay()
        torch.cuda.synchronize()
        for k, t in keep["out"].items():
            if t is not None:
                assert np.array_equal(down(t)[:, :c.F], want[k][:, :c.F], equal_nan=True), k


def test_no_tokens(tpp):
    f = 33
    for every, gone in ((0, True), (4, False)):
        d = tpp.tpp_residual_desc(f, 1, 2, 2, 1, 1, 1.0, EPS, every)
        vecs = [torch.full((f,), 7.0, device="cuda") for _ in range(4)]
        dgate = torch.full((1, f), 7.0, device="cuda", dtype=torch.bfloat16)
        tpp.tpp_residual_norm_backward(d, 0, None, f, None, f, None, None, None, None, f, None, f, None, f,
                                       None, f, None, f, dgate, f, *vecs, tpp.current_stream())
        assert all((v == 0).all() for v in vecs) and bool((dgate == 0).all()) == gone


def test_rows_past_32_bits(tpp):
    """Tokens 2^31 entries apart in one block: rows past 2^32 bytes."""
    ld, f = (1 << 31) + 8, 1000
    x, b, r, y = (torch.empty(2 * ld, dtype=torch.bfloat16, device="cuda") for _ in range(4))
    c = Case((3, f, "rms", "rms", "none", 0, "bf16", "f32", 0, 0), 12)
    for t in range(2):
        for dst, src in ((x, c.x), (b, c.b)):
            dst[t * ld:t * ld + f] = up(src)[t].view(torch.bfloat16)
    wa, wb = up(c.wa), up(c.wb)
    tpp.tpp_residual_norm(c.desc(tpp), 2, x, ld, b, ld, None, 0, wa, None, wb, None, r, ld, y, ld, None, 0,
                          None, tpp.current_stream())
    want = forward(tpp, c)
    for t in range(2):
        for got, ref in ((r, want[0]), (y, want[1])):
            assert np.array_equal(down(got[t * ld:t * ld + f].view(torch.int16)), ref[t])
