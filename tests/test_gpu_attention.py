"""GPU parity of the attention operators, through the C ABI, against the fp64 oracle.

Bounds on the error of each output, from the arithmetic (u = 2^-24, fp32's half unit):
  norm and rotation   a sum of D squares, a square root, a division, three products and a rotation:
                      below 32 u (1 + D / 64) of the head's largest entries a, b; bf16 outputs a rounding more
  its gradients       the same on u and xn, twice: 64 u (1 + D / 64) r (max |u| + max |xn| |mean|);
                      dw: (64 + rows) u of the sum of |g xn|, the bound of a sum in any order
  attention           a score is a sum of D products: |ds| <= (D + 4) u |scale| sum |q k|; a weight is off
                      by exp of twice that and by the exponential's few u; a sum over n positions in any
                      order by (64 + n) u; weights enter the products with the values in two bf16 parts
                      (2^-16) where the cache is bf16
  eviction            whole numbers and moved rows: exact
A bf16 output adds half a unit of its own, 2^-8 of its value at most."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import oracle
import workloads as wk
from helpers import run_call_oracle, values

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
NAN = {"f32": np.float32(np.nan), "bf16": np.uint16(0x7FC0)}


@pytest.fixture(scope="module", autouse=True)
def gpu():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"


@pytest.fixture(scope="module")
def tpp():
    import paper_2104_05755_amd as tpp
    return tpp


def draw(rng, shape, dtype, std=1.0):
    x = (rng.standard_normal(shape) * std).astype(np.float32)
    return x if dtype == "f32" else wk.bf16_bits(x).reshape(shape)


def up(a):
    a = np.ascontiguousarray(a)
    return torch.from_numpy((a.view(np.int16) if a.dtype == np.uint16 else a).copy()).cuda()


def down(t, dtype):
    a = t.cpu().numpy()
    return a.view(np.uint16) if dtype == "bf16" else a


def code(tpp, dtype):
    return tpp.TPP_DT_BF16 if dtype == "bf16" else tpp.TPP_DT_F32


def close(got, ref, bound, dtype, what):
    """|got - ref| <= bound (+ the output's own rounding) everywhere; infinities where ref has them."""
    got = values(got, dtype) if got.dtype != np.float64 else got
    fin = np.isfinite(ref)
    assert np.array_equal(got[~fin], ref[~fin], equal_nan=True), what
    limit = np.broadcast_to(bound, ref.shape) + np.abs(ref) * (2.0 ** -8 if dtype == "bf16" else U) + 1e-37
    off = np.abs(got[fin] - ref[fin])
    assert not np.isnan(off).any() and not (off > limit[fin]).any(), \
        f"{what}: off by {off.max():.3e}, up to {(off / limit[fin]).max():.2f} of what is allowed"


# ---- norms and rotation ------------------------------------------------------------------------
ROPE = [  # tokens, q heads, k heads, D, rot_dim, form, dtype, extra ld, first element
    (1, 16, 16, 64, 64, "halves", "bf16", 0, 0),
    (7, 32, 8, 128, 128, "halves", "bf16", 0, 0),
    (130, 4, 2, 128, 64, "halves", "bf16", 8, 0),
    (33, 3, 1, 96, 96, "pairs", "bf16", 0, 0),
    (33, 3, 1, 80, 16, "pairs", "bf16", 3, 1),       # rows at odd elements
    (19, 5, 5, 256, 256, "halves", "f32", 0, 0),
    (19, 7, 1, 77, 32, "pairs", "f32", 1, 1),        # an odd head
    (19, 2, 3, 77, 76, "halves", "bf16", 0, 0),
    (9, 1, 1, 1, 0, "halves", "f32", 0, 0),
    (9, 1, 2, 2, 2, "pairs", "bf16", 0, 0),
    (9, 3, 2, 512, 512, "halves", "bf16", 0, 0),
    (9, 3, 2, 509, 254, "pairs", "f32", 0, 0),
    (65, 0, 4, 64, 32, "halves", "bf16", 0, 0),      # one side only
    (65, 4, 0, 64, 0, "halves", "f32", 0, 0),        # the norm alone
    (300, 2, 2, 72, 48, "halves", "bf16", 0, 0),
    (300, 2, 2, 112, 56, "pairs", "bf16", 0, 0),
    # parts that are no whole chunks: the halves, the rest, both; a rest below a chunk; odd rows
    (70, 3, 2, 80, 40, "halves", "bf16", 0, 0),
    (70, 3, 2, 72, 72, "halves", "bf16", 1, 1),
    (70, 3, 2, 72, 36, "halves", "f32", 0, 0),
    (70, 3, 2, 77, 38, "halves", "bf16", 0, 1),
    (70, 3, 2, 77, 76, "halves", "f32", 1, 0),
    (70, 3, 2, 77, 0, "halves", "bf16", 0, 0),
    (70, 3, 2, 77, 76, "pairs", "f32", 0, 0),
    (70, 3, 2, 77, 68, "pairs", "bf16", 0, 0),
    (70, 3, 2, 78, 78, "pairs", "bf16", 0, 1),
    (70, 3, 2, 9, 0, "pairs", "bf16", 0, 0),
    (70, 3, 2, 17, 16, "halves", "bf16", 0, 0),
    (9, 2, 1, 511, 10, "halves", "f32", 0, 0),           # one lane too many for a wavefront
    (9, 2, 1, 511, 8, "halves", "f32", 0, 0),
    (9, 2, 1, 511, 500, "halves", "bf16", 0, 0),
]
ROPE_IDS = [f"T{c[0]}-{c[1]}x{c[2]}-D{c[3]}-R{c[4]}-{c[5]}-{c[6]}-{c[7]}-{c[8]}" for c in ROPE]
EPS = 1e-5


class Rope:
    """Inputs of one case, on the host and on the device, queries, keys and values in one block."""

    def __init__(self, case, seed=0):
        self.case = case
        T, hq, hk, D, R, form, dtype, pad, first = case
        rng = np.random.default_rng(seed + T * 1000 + D)
        self.ld = (hq + 2 * hk) * D + pad
        self.flat = draw(rng, T * self.ld + first, dtype)
        n_pos = 50
        ang = rng.uniform(-4, 4, (n_pos, R // 2))
        self.rot = np.concatenate([np.cos(ang), np.sin(ang)], 1).astype(np.float32)
        self.w = [rng.uniform(0.5, 1.5, D).astype(np.float32) for _ in range(2)]
        self.pos = rng.integers(0, n_pos, T)
        self.pos[3::7] = rng.choice([-1, n_pos, 1 << 40], len(self.pos[3::7]))   # padding tokens
        self.heads = (hq, hk)
        self.off = (first, first + hq * D, first + (hq + hk) * D)
        self.dev = dict(flat=up(self.flat), rot=up(self.rot) if R else None,
                        w=[up(x) for x in self.w], pos=up(self.pos))
        es = self.flat.itemsize
        self.at = [self.dev["flat"].data_ptr() + o * es for o in self.off]

    def desc(self, tpp):
        T, hq, hk, D, R, form, dtype = self.case[:7]
        return tpp.tpp_qk_desc(D, R, tpp.TPP_ROT_HALVES if form == "halves" else tpp.TPP_ROT_PAIRS,
                               hq, hk, code(tpp, dtype), EPS, len(self.rot))

    def ref(self, side):
        T, _, _, D, R, form, dtype = self.case[:7]
        return oracle.qk_norm_rope(self.flat[self.off[side]:], self.ld, self.heads[side], D, R, form,
                                   self.w[side], self.rot, self.pos, EPS, dtype)

    def bound(self, ref):
        D = self.case[3]
        return 32 * U * (1 + D / 64) * 2 * np.abs(ref).max(-1, keepdims=True)


@pytest.mark.parametrize("case", ROPE, ids=ROPE_IDS)
def test_norm_rope(tpp, case):
    T, hq, hk, D, R, form, dtype, pad, first = case
    r = Rope(case)
    outs = [up(np.full(T * (h * D + pad) + first, NAN[dtype])) for h in (hq, hk)]
    es = r.flat.itemsize
    ptr = [o.data_ptr() + first * es for o in outs]
    s = tpp.current_stream()
    tpp.tpp_qk_norm_rope(r.desc(tpp), T, r.at[0], r.ld, r.at[1], r.ld, r.dev["w"][0], r.dev["w"][1],
                         r.dev["rot"], r.dev["pos"], ptr[0], hq * D + pad, ptr[1], hk * D + pad, s)
    torch.cuda.synchronize()
    for side, h in enumerate((hq, hk)):
        got = down(outs[side], dtype)
        rows = got[first:].reshape(T, h * D + pad)
        ref = r.ref(side)
        close(rows[:, :h * D].reshape(T, h, D), ref, r.bound(ref) if h else 0, dtype, f"side {side}")
        gap = np.concatenate([got[:first], rows[:, h * D:].ravel()])   # nothing beside the rows is written
        assert np.array_equal(gap.view(np.uint16 if dtype == "bf16" else np.uint32),
                              np.full(gap.shape, NAN[dtype]).view(np.uint16 if dtype == "bf16" else np.uint32))
    # in place, with the values' part of the block untouched
    tpp.tpp_qk_norm_rope(r.desc(tpp), T, r.at[0], r.ld, r.at[1], r.ld, r.dev["w"][0], r.dev["w"][1],
                         r.dev["rot"], r.dev["pos"], r.at[0], r.ld, r.at[1], r.ld, s)
    torch.cuda.synchronize()
    block = down(r.dev["flat"], dtype)[first:].reshape(T, r.ld)
    for side, h in enumerate((hq, hk)):
        a = (0, hq * D)[side]
        want = down(outs[side], dtype)[first:].reshape(T, h * D + pad)[:, :h * D]
        assert block[:, a:a + h * D].tobytes() == want.tobytes()
    assert block[:, (hq + hk) * D:].tobytes() == r.flat[first:].reshape(T, r.ld)[:, (hq + hk) * D:].tobytes()


@pytest.mark.parametrize("case", ROPE, ids=ROPE_IDS)
@pytest.mark.parametrize("heads_first", [False, True])
def test_append(tpp, case, heads_first):
    T, hq, hk, D, R, form, dtype, pad, first = case
    if hk == 0:
        pytest.skip("a cache needs a key head")
    r = Rope(case, 1)
    page, es = 5, r.flat.itemsize
    n_pages = -(-T // page) + 2
    rng = np.random.default_rng(T)
    slot = rng.permutation(n_pages * page)[:T]
    slot[2::9] = rng.choice([-1, n_pages * page, 1 << 40], len(slot[2::9]))   # not cached
    # [page][head][place][D] or [page][place][head][D], rows `pad` apart
    hs, ps = ((D + pad) * page, D + pad) if heads_first else (D + pad, (D + pad) * hk)
    pg = (D + pad) * hk * page + 3
    pools = [up(np.full(n_pages * pg + first, NAN[dtype])) for _ in range(2)]
    c = tpp.tpp_kv_cache(pools[0].data_ptr() + first * es, pools[1].data_ptr() + first * es,
                         code(tpp, dtype), D, hk, page, n_pages, pg, ps, hs)
    q_out = up(np.full(T * hq * D + 1, NAN[dtype]))
    d_slot = up(slot)
    tpp.tpp_qk_norm_rope_append(r.desc(tpp), T, r.at[0], r.ld, r.at[1], r.ld, r.at[2], r.ld,
                                r.dev["w"][0], r.dev["w"][1], r.dev["rot"], r.dev["pos"], q_out,
                                hq * D, c, d_slot, tpp.current_stream())
    torch.cuda.synchronize()
    ref = r.ref(0)
    close(down(q_out, dtype)[:T * hq * D].reshape(T, hq, D), ref, r.bound(ref) if hq else 0, dtype, "q")
    k, v = (down(p, dtype) for p in pools)
    ref = r.ref(1)
    bound = r.bound(ref)
    held = np.zeros(k.shape, bool)
    for t in range(T):
        if not (0 <= slot[t] < n_pages * page and 0 <= r.pos[t] < len(r.rot)):
            continue
        for h in range(hk):
            at = first + slot[t] // page * pg + slot[t] % page * ps + h * hs
            close(k[at:at + D], ref[t, h], bound[t, h], dtype, f"key of token {t}, head {h}")
            src = r.off[2] + t * r.ld + h * D
            assert v[at:at + D].tobytes() == r.flat[src:src + D].tobytes()
            held[at:at + D] = True
    for x in (k, v):   # everything else is as it was
        assert x[~held].tobytes() == np.full((~held).sum(), NAN[dtype]).tobytes()


def run_backward(tpp, r, g, stream=None):
    T, hq, hk, D, R, form, dtype, pad, first = r.case
    dev_g = [up(x) for x in g]
    outs = [up(np.full(T * (h * D + pad), NAN[dtype])) for h in (hq, hk)]
    dw = [up(np.full(D + 1, np.float32(np.nan))) for _ in range(2)]
    tpp.tpp_qk_norm_rope_backward(
        r.desc(tpp), T, r.at[0], r.ld, r.at[1], r.ld, r.dev["w"][0], r.dev["w"][1], r.dev["rot"],
        r.dev["pos"], dev_g[0], hq * D + 1, dev_g[1], hk * D + 1, outs[0], hq * D + pad, outs[1],
        hk * D + pad, dw[0], dw[1], tpp.current_stream() if stream is None else stream)
    torch.cuda.synchronize()
    return outs, dw


def gradient_bounds(r, side, g, dx):
    """The head's scale r (max |u| + max |xn| |mean|) from the oracle's own pieces, as arrays."""
    T, _, _, D, R, form, dtype = r.case[:7]
    h = r.heads[side]
    x = values(r.flat, dtype)[r.off[side]:]
    x = np.stack([x[t * r.ld:t * r.ld + h * D].reshape(h, D) for t in range(T)])
    rstd = 1 / np.sqrt((x ** 2).mean(-1, keepdims=True) + EPS)
    gv = np.abs(values(g, dtype)).reshape(T, -1)[:, :h * D].reshape(T, h, D).max(-1, keepdims=True) * 2 ** 0.5
    um, xm = gv * np.abs(r.w[side]).max(), np.abs(x * rstd).max(-1, keepdims=True)
    return 64 * U * (1 + D / 64) * rstd * (um + xm * um * np.minimum(xm, 1)), (gv * np.abs(x * rstd)).sum((0, 1))


@pytest.mark.parametrize("case", ROPE, ids=ROPE_IDS)
def test_norm_rope_backward(tpp, case):
    T, hq, hk, D, R, form, dtype, pad, first = case
    r = Rope(case, 2)
    rng = np.random.default_rng(3)
    g = [draw(rng, (T, h * D + 1), dtype) for h in (hq, hk)]
    outs, dw = run_backward(tpp, r, g)
    again, dw2 = run_backward(tpp, r, g)
    for side, h in enumerate((hq, hk)):
        if h == 0:
            continue
        dx, ref_w = oracle.qk_norm_rope_backward(r.flat[r.off[side]:], r.ld, h, D, R, form, r.w[side],
                                                 r.rot, r.pos, EPS, dtype, g[side], h * D + 1)
        bx, bw = gradient_bounds(r, side, g[side], dx)
        rows = down(outs[side], dtype).reshape(T, h * D + pad)
        close(rows[:, :h * D].reshape(T, h, D), dx, bx, dtype, f"dx {side}")
        got = dw[side].cpu().numpy()
        close(got[:D], ref_w, (64 + T * h) * U * bw, "f32", f"dw {side}")
        assert np.isnan(got[D])
        assert torch.equal(dw[side][:D], dw2[side][:D])   # the same bits every time
        assert rows.tobytes() == down(again[side], dtype).tobytes()


def test_norm_rope_backward_no_tokens_and_in_place(tpp):
    case = (40, 3, 2, 64, 64, "halves", "bf16", 0, 0)
    r = Rope(case, 5)
    dw = [torch.full((64,), 7.0, device="cuda") for _ in range(2)]
    tpp.tpp_qk_norm_rope_backward(r.desc(tpp), 0, None, 192, None, 128, None, None, None, None, None,
                                  192, None, 128, None, 192, None, 128, dw[0], dw[1],
                                  tpp.current_stream())
    torch.cuda.synchronize()
    assert not dw[0].any() and not dw[1].any()
    g = [draw(np.random.default_rng(4), (40, h * 64 + 1), "bf16") for h in (3, 2)]
    outs, want = run_backward(tpp, r, g)
    dev = [up(x[:, :-1]) for x in g]
    tpp.tpp_qk_norm_rope_backward(r.desc(tpp), 40, r.at[0], r.ld, r.at[1], r.ld, r.dev["w"][0],
                                  r.dev["w"][1], r.dev["rot"], r.dev["pos"], dev[0], 192, dev[1], 128,
                                  dev[0], 192, dev[1], 128, dw[0], dw[1], tpp.current_stream())
    torch.cuda.synchronize()
    for s in range(2):
        assert torch.equal(dev[s].ravel(), outs[s]) and torch.equal(dw[s], want[s][:64])


@pytest.mark.parametrize("form", ["halves", "pairs"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_norm_rope_without_a_table(tpp, form, dtype):
    """A table of no rows: every token is padding, the table may be NULL."""
    T, D = 9, 64
    rot = tpp.TPP_ROT_HALVES if form == "halves" else tpp.TPP_ROT_PAIRS
    d = tpp.tpp_qk_desc(D, D, rot, 2, 1, code(tpp, dtype), EPS, 0)
    rng = np.random.default_rng(1)
    q, k, g = (up(draw(rng, (T, h * D), dtype)) for h in (2, 1, 2))
    w, pos = torch.ones(D, device="cuda"), torch.zeros(T, dtype=torch.int64, device="cuda")
    dw = [torch.full((D,), 7.0, device="cuda") for _ in range(2)]
    out = [torch.full_like(x, 3) for x in (q, k, q, k)]
    s = tpp.current_stream()
    tpp.tpp_qk_norm_rope(d, T, q, 2 * D, k, D, w, w, None, pos, out[0], 2 * D, out[1], D, s)
    tpp.tpp_qk_norm_rope_backward(d, T, q, 2 * D, k, D, w, w, None, pos, g, 2 * D, k, D, out[2], 2 * D,
                                  out[3], D, dw[0], dw[1], s)
    torch.cuda.synchronize()
    assert not any(x.any() for x in out + dw)


@pytest.mark.parametrize("dtype,D,form,T", [("bf16", 128, "halves", 8300), ("bf16", 80, "pairs", 7001),
                                            ("f32", 64, "halves", 5000), ("bf16", 128, "pairs", 4000)])
def test_norm_rope_large(tpp, dtype, D, form, T):
    """Passes large enough to go past the caches give the bits that the same tokens give in small ones."""
    hq, hk, part = 32, 8, 100
    g = torch.Generator(device="cuda")
    g.manual_seed(D)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    x, gy = (torch.randn(T, (hq + hk) * D, generator=g, device="cuda").to(dt) for _ in range(2))
    ang = torch.rand(64, D // 2, generator=g, device="cuda") * 6
    rot = torch.cat([ang.cos(), ang.sin()], 1).contiguous()
    pos = torch.arange(T, device="cuda") % 66 - 1        # padding tokens among them
    w = [1 + 0.1 * torch.randn(D, generator=g, device="cuda") for _ in range(2)]
    desc = tpp.tpp_qk_desc(D, D, tpp.TPP_ROT_HALVES if form == "halves" else tpp.TPP_ROT_PAIRS, hq, hk,
                           code(tpp, dtype), EPS, 64)
    ld, s, es = (hq + hk) * D, tpp.current_stream(), x.element_size()

    def run(t0, n):
        at = lambda a: (a.data_ptr() + t0 * ld * es, a.data_ptr() + (t0 * ld + hq * D) * es)
        y, dx = torch.zeros(n, ld, dtype=dt, device="cuda"), torch.zeros(n, ld, dtype=dt, device="cuda")
        o = lambda a: (a.data_ptr(), a.data_ptr() + hq * D * es)
        dw = [torch.zeros(D, device="cuda") for _ in range(2)]
        p = pos[t0:t0 + n].contiguous()
        (q, k), (gq, gk), (yq, yk), (dq, dk) = at(x), at(gy), o(y), o(dx)
        tpp.tpp_qk_norm_rope(desc, n, q, ld, k, ld, w[0], w[1], rot, p, yq, ld, yk, ld, s)
        tpp.tpp_qk_norm_rope_backward(desc, n, q, ld, k, ld, w[0], w[1], rot, p, gq, ld, gk, ld, dq, ld, dk,
                                      ld, dw[0], dw[1], s)
        torch.cuda.synchronize()
        return y, dx, dw

    y, dx, dw = run(0, T)
    for t0 in (0, 1234, T - part):
        yp, dxp, _ = run(t0, part)
        assert torch.equal(y[t0:t0 + part], yp) and torch.equal(dx[t0:t0 + part], dxp)
    halves = [run(0, T // 2), run(T // 2, T - T // 2)]
    for side in range(2):
        # both are within (64 + rows) u of the sum of |g xn|, below rows * 64 for these normals
        both = halves[0][2][side].double() + halves[1][2][side].double()
        rows = T * (hq, hk)[side]
        assert (dw[side].double() - both).abs().max() <= 2 * (64 + rows ** 0.5) * U * rows * 2
        assert dw[side].abs().max() > 0


def test_norm_rope_past_32_bits(tpp):
    """Tokens more than 2^32 bytes apart."""
    D, ld, T = 64, (1 << 31) + 72, 3
    big = torch.zeros(ld * (T - 1) + 3 * D, dtype=torch.bfloat16, device="cuda")
    small = torch.randn(T, 3 * D, device="cuda").bfloat16()
    for t in range(T):
        big[t * ld:t * ld + 3 * D] = small[t]
    rot = torch.rand(8, D, device="cuda")
    pos, w = torch.tensor([1, 7, 3], device="cuda"), torch.ones(D, device="cuda")
    desc, s, res = tpp.tpp_qk_desc(D, D, tpp.TPP_ROT_HALVES, 2, 1, tpp.TPP_DT_BF16, EPS, 8), tpp.current_stream(), []
    for x, l in ((small.clone(), 3 * D), (big, ld)):
        p = x.data_ptr()
        dw = torch.zeros(2, D, device="cuda")
        g = small.flip(0).contiguous()
        dx = torch.zeros_like(g)
        tpp.tpp_qk_norm_rope_backward(desc, T, p, l, p + 4 * D, l, w, w, rot, pos, g, 3 * D, g.data_ptr() + 4 * D,
                                      3 * D, dx, 3 * D, dx.data_ptr() + 4 * D, 3 * D, dw[0], dw[1], s)
        tpp.tpp_qk_norm_rope(desc, T, p, l, p + 4 * D, l, w, w, rot, pos, p, l, p + 4 * D, l, s)   # in place
        torch.cuda.synchronize()
        y = torch.stack([x.reshape(-1)[t * l:t * l + 3 * D] for t in range(T)])
        res.append((y, dx, dw))
    for a, b in zip(*res):
        assert torch.equal(a, b) and a.any()


def test_backward_against_differences(tpp):
    """fp32 gradients against central differences of the GPU's own forward pass, all entries of one
    head moved along a random direction: the sum's curvature bounds the rest."""
    case = (6, 2, 1, 64, 64, "pairs", "f32", 0, 0)
    r = Rope(case, 6)
    rng = np.random.default_rng(7)
    g = [draw(rng, (6, h * 64 + 1), "f32") for h in (2, 1)]
    outs, _ = run_backward(tpp, r, g)
    step, base = 2.0 ** -6, r.flat.copy()
    way = rng.standard_normal(base.shape).astype(np.float32)

    def forward(x):
        dev, res = up(x), 0.0
        o = [up(np.zeros(6 * h * 64, np.float32)) for h in (2, 1)]
        at = [dev.data_ptr() + k * 4 for k in r.off]
        tpp.tpp_qk_norm_rope(r.desc(tpp), 6, at[0], r.ld, at[1], r.ld, r.dev["w"][0], r.dev["w"][1],
                             r.dev["rot"], r.dev["pos"], o[0], 128, o[1], 64, tpp.current_stream())
        torch.cuda.synchronize()
        for s, h in enumerate((2, 1)):
            res += float((o[s].cpu().numpy().astype(np.float64) * g[s][:, :h * 64].ravel()).sum())
        return res

    slope = (forward(base + step * way) - forward(base - step * way)) / (2 * step)
    want = 0.0
    for s, h in enumerate((2, 1)):
        w = way.reshape(6, r.ld)[:, (0, 128)[s]:(0, 128)[s] + h * 64]
        want += float((outs[s].cpu().numpy().astype(np.float64) * w.ravel()).sum())
    # third derivative over six, times step^2: |g| |way|^3 per head; 18 heads of |g| = |way| = 8
    assert abs(slope - want) < 18 * 8 * step ** 2 * 4 + 1e-3


# ---- attention ------------------------------------------------------------------------------------
class Paged:
    """A cache of given lengths whose unused places are NaN, in either layout, at any alignment."""

    def __init__(self, lens, D, hk, page, dtype, seed=0, heads_first=False, pad=0, first=0, holes=(),
                 room=0):
        rng = self.rng = np.random.default_rng(seed)
        self.lens, self.D, self.hk, self.page, self.dtype = np.array(lens), D, hk, page, dtype
        per = max(1, -(-max(lens) // page)) + 1          # a column more than needed
        self.n_pages = len(lens) * per + 1
        self.pages = rng.permutation(self.n_pages)[:len(lens) * per].reshape(len(lens), per)
        for b, j in holes:
            self.pages[b, j % per] = [-1, self.n_pages, 1 << 40][j % 3]
        # a table for longer sequences: columns that name no page yet
        self.pages = np.pad(self.pages, ((0, 0), (0, -(-room // page))), constant_values=-1)
        d = D + pad
        self.strides = (d * hk * page + 5 * pad, d, d * page) if heads_first else \
            (d * hk * page + 5 * pad, d * hk, d)
        self.first = first
        self.pool = [np.full(self.n_pages * self.strides[0] + first, NAN[dtype]) for _ in range(2)]
        for b, n in enumerate(self.lens):
            for t in range(n):
                at = self.row(b, t)
                if at is None:
                    continue
                for h in range(hk):
                    for p in self.pool:
                        p[at + h * self.strides[2]:][:D] = draw(rng, D, dtype)
        self.dev = [up(p) for p in self.pool]
        self.d_pages, self.d_lens = up(self.pages), up(self.lens.astype(np.int64))

    def row(self, b, t):
        page = self.pages[b, t // self.page]
        if not 0 <= page < self.n_pages:
            return None
        return self.first + page * self.strides[0] + t % self.page * self.strides[1]

    def c(self, tpp):
        es = self.pool[0].itemsize
        return tpp.tpp_kv_cache(self.dev[0].data_ptr() + self.first * es,
                                self.dev[1].data_ptr() + self.first * es, code(tpp, self.dtype),
                                self.D, self.hk, self.page, self.n_pages, *self.strides)

    def host(self):
        return [p[self.first:] for p in self.pool]


def attend(tpp, pc, q, hq, out_type, scale, window=0, max_len=None, totals=None, pad=0, stream=None):
    n, f = len(pc.lens), hq * pc.D
    max_len = int(max(pc.lens)) if max_len is None else max_len
    out = up(np.full((n, f + pad), NAN[out_type]))
    lse = torch.full((n, hq), 7.0, device="cuda")
    qd = up(q)
    tot = None if totals is None else up(totals)
    tot_out = None if totals is None else torch.full_like(tot, -5.0)
    tpp.tpp_paged_attention(tpp.tpp_attn_desc(hq, code(tpp, out_type), scale, window, max_len),
                            pc.c(tpp), n, qd, q.shape[1], pc.d_lens, pc.d_pages, pc.pages.shape[1],
                            out, f + pad, lse, tot, tot_out, 0 if tot is None else tot.shape[1],
                            tpp.current_stream() if stream is None else stream)
    torch.cuda.synchronize()
    return down(out, out_type), lse.cpu().numpy(), None if tot is None else tot_out.cpu().numpy()


def check_attention(tpp, pc, hq, out_type, window=0, with_totals=False, max_len=None, pad=0, std=1.0,
                    scale=None):
    n, D, dt = len(pc.lens), pc.D, pc.dtype
    q = draw(pc.rng, (n, hq * D + pad), dt, std)
    scale = D ** -0.5 if scale is None else scale
    cut = np.clip(pc.lens, 0, max_len) if max_len is not None else np.clip(pc.lens, 0, None)
    ldt = int(max(1, cut.max(initial=0), max_len or 0)) + 3
    totals = pc.rng.random((n, ldt)).astype(np.float32) if with_totals else None
    k, v = pc.host()
    args = (dt, D, pc.hk, pc.page, pc.n_pages, pc.strides, pc.pages, q, q.shape[1], hq, cut)
    ref, lse, tot = oracle.paged_attention(k, v, *args, scale, window, totals)
    # sum p |v| and the scores' scale, for the bounds
    mag = {"f32": np.abs, "bf16": lambda x: x & 0x7FFF}[dt]
    big, _, _ = oracle.paged_attention(k, mag(v), *args, scale, window)
    qn = np.abs(values(q, dt))[:, :hq * D].reshape(n, hq, D).sum(-1)
    kmax = np.nanmax(np.abs(values(k, dt)), initial=0.0)
    ds = (D + 4) * U * abs(scale) * qn * kmax
    got, got_lse, got_tot = attend(tpp, pc, q, hq, out_type, scale, window, max_len, totals, pad)
    again = attend(tpp, pc, q, hq, out_type, scale, window, max_len, totals, pad)
    assert got.tobytes() == again[0].tobytes() and got_lse.tobytes() == again[1].tobytes()
    top = int(cut.max(initial=0))
    rel = 2 * ds + (64 + top) * U + 2.0 ** -20 + (2.0 ** -16 if dt == "bf16" else 0)
    close(got[:, :hq * D].reshape(n, hq, D), ref, rel[..., None] * big, out_type, "out")
    close(got_lse.astype(np.float64), lse, 2 * ds + (64 + top) * U + 2.0 ** -20, "f32", "lse")
    if pad:
        assert np.array_equal(got[:, hq * D:].view(np.uint8), np.full((n, pad), NAN[out_type]).view(np.uint8))
    if with_totals:
        assert got_tot.tobytes() == again[2].tobytes()
        for b in range(n):
            close(got_tot[b, :cut[b]].astype(np.float64), tot[b, :cut[b]],
                  rel[b].max() * (tot[b, :cut[b]] - totals[b, :cut[b]]) + 1e-30, "f32", f"totals {b}")
            assert (got_tot[b, cut[b]:] == -5.0).all()     # nothing is written behind the length


EDGES = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 100]
MORE = [0, 127, 128, 129, 200, 255, 256, 257, 500, 511, 512, 513, 700]
ATTN = [  # lens, D, q heads, k heads, page, dtype, out, heads first, pad, first
    (EDGES, 64, 16, 16, 16, "bf16", "bf16", False, 0, 0),
    (EDGES, 128, 32, 8, 16, "bf16", "bf16", False, 0, 0),
    (MORE, 128, 8, 2, 16, "bf16", "f32", True, 0, 0),
    (MORE, 128, 8, 2, 64, "f32", "f32", False, 0, 0),
    (EDGES, 8, 3, 1, 1, "bf16", "f32", False, 0, 0),
    (EDGES, 8, 3, 1, 5, "f32", "f32", False, 0, 0),
    (MORE, 32, 7, 1, 7, "bf16", "bf16", True, 0, 0),
    (MORE, 77, 21, 7, 7, "f32", "f32", False, 3, 1),
    (MORE, 77, 6, 3, 7, "bf16", "f32", False, 3, 1),     # rows at odd elements, a tail of 5
    (EDGES, 9, 2, 2, 32, "bf16", "bf16", False, 0, 1),
    (MORE, 80, 10, 2, 128, "bf16", "f32", True, 5, 3),
    (EDGES, 96, 4, 1, 256, "bf16", "f32", False, 0, 0),
    (EDGES, 100, 4, 1, 3, "f32", "bf16", True, 1, 0),
    (EDGES, 192, 8, 2, 16, "bf16", "f32", False, 0, 0),
    (MORE, 256, 8, 1, 16, "bf16", "bf16", False, 0, 0),
    (MORE, 256, 4, 2, 16, "f32", "f32", False, 0, 0),
    (EDGES, 250, 4, 2, 16, "f32", "f32", False, 0, 1),
    (EDGES, 64, 24, 1, 16, "bf16", "f32", False, 0, 0),  # more queries to a key head than a tile holds
    (EDGES, 64, 35, 1, 16, "f32", "f32", False, 0, 0),
    (MORE, 128, 64, 1, 16, "bf16", "f32", False, 0, 0),
    (EDGES, 40, 17, 1, 6, "bf16", "f32", False, 0, 0),
]
ATTN_IDS = [f"L{max(c[0])}-D{c[1]}-{c[2]}x{c[3]}-P{c[4]}-{c[5]}-{c[6]}-{int(c[7])}{c[8]}{c[9]}" for c in ATTN]


@pytest.mark.parametrize("case", ATTN, ids=ATTN_IDS)
@pytest.mark.parametrize("with_totals", [False, True])
def test_attention(tpp, case, with_totals):
    lens, D, hq, hk, page, dtype, out, hf, pad, first = case
    pc = Paged(lens, D, hk, page, dtype, seed=D, heads_first=hf, pad=pad, first=first)
    check_attention(tpp, pc, hq, out, with_totals=with_totals, pad=pad)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window", [1, 31, 32, 100, 513, 10 ** 12])
def test_attention_window(tpp, dtype, window):
    pc = Paged(MORE, 64, 2, 16, dtype, seed=window % 97)
    check_attention(tpp, pc, 8, "f32", window=window, with_totals=window == 100)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [1, 7, 64])
def test_attention_pages_that_hold_nothing(tpp, dtype, page):
    """Whole tiles, single positions and whole sequences masked; whatever lies there is never read."""
    lens = [5, 64, 300, 600, 33]
    holes = [(0, j) for j in range(6)] + [(3, j) for j in range(0, 600, 2)] + [(2, 0), (2, 1), (4, 0)]
    pc = Paged(lens, 64, 2, page, dtype, seed=page, holes=holes)
    check_attention(tpp, pc, 6, "f32", with_totals=True)
    check_attention(tpp, pc, 6, "f32", window=40)


def test_attention_empty_and_cut_lengths(tpp):
    pc = Paged([50, 60, 0, 1], 64, 2, 16, "bf16")
    pc.d_lens = up(np.array([50, 60, -3, 0], np.int64))
    pc.lens = np.array([50, 60, -3, 0])
    check_attention(tpp, pc, 4, "f32", max_len=55, with_totals=True)
    check_attention(tpp, pc, 4, "f32", max_len=0, with_totals=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_large_scores(tpp, dtype):
    """Scores in the thousands: one position takes nearly all the weight, nothing overflows."""
    pc = Paged([1, 40, 300], 64, 2, 16, dtype)
    check_attention(tpp, pc, 4, "f32", std=400.0, with_totals=True)
    check_attention(tpp, pc, 4, "f32", scale=-1.0)
    check_attention(tpp, pc, 4, "f32", scale=0.0, with_totals=True)


@pytest.mark.parametrize("n,L,D,hq,hk,dtype", [(1, 9000, 128, 8, 2, "bf16"), (2, 5001, 64, 4, 4, "f32"),
                                               (3, 4000, 80, 20, 1, "bf16"), (40, 700, 64, 2, 1, "bf16")])
def test_attention_long(tpp, n, L, D, hq, hk, dtype):
    rng = np.random.default_rng(L)
    lens = [L] + rng.integers(1, L, n - 1).tolist()
    pc = Paged(lens, D, hk, 16, dtype, seed=L, room=3000)
    check_attention(tpp, pc, hq, "f32", with_totals=True)
    check_attention(tpp, pc, hq, "bf16", max_len=L + 3000)


@pytest.mark.parametrize("D,hq,hk,page,dtype", [(128, 24, 1, 16, "bf16"), (128, 64, 1, 64, "f32"),
                                                (77, 70, 2, 7, "bf16"), (64, 35, 1, 16, "f32")])
def test_attention_two_head_tiles(tpp, D, hq, hk, page, dtype):
    """Room for 8192 positions in 40 sequences: two tiles of query heads to a workgroup, whose span is of
    more positions than it looks up at a time; some of those blocks hold nothing, some a single page."""
    lens = [2700, 1500, 1025, 0, 1024, 2100] + list(range(34))
    holes = [(0, j) for j in range(1030 // page, 2100 // page)] + [(5, j) for j in range(1024 // page + 1)]
    pc = Paged(lens, D, hk, page, dtype, seed=hq, holes=holes, room=8192)
    check_attention(tpp, pc, hq, "f32", max_len=8192, with_totals=True)
    check_attention(tpp, pc, hq, "bf16", max_len=8192, window=5000)


def test_attention_nan_in_what_is_held_shows(tpp):
    """A NaN among the held keys reaches the heads that read it, one among the values its entry alone."""
    pc = Paged([70, 300], 64, 2, 16, "bf16", seed=4)
    hold = lambda b, t, h: pc.row(b, t) + h * pc.strides[2]
    pc.dev[0][hold(0, 33, 1)] = int(NAN["bf16"])
    pc.dev[1][hold(1, 299, 0) + 5] = int(NAN["bf16"])
    out, lse, _ = attend(tpp, pc, draw(pc.rng, (2, 4 * 64), "bf16"), 4, "f32", 0.125)
    bad = np.isnan(out.reshape(2, 4, 64))
    assert bad[0, 2:].all() and not bad[0, :2].any() and np.isnan(lse[0, 2:]).all()
    assert bad[1, :2, 5].all() and bad[1].sum() == 2 and not np.isnan(lse[1]).any()


def test_attention_past_32_bits(tpp):
    """Pages more than 2^32 bytes apart."""
    D, page, stride = 64, 16, (1 << 31) + 64
    pool = torch.full((2 * stride + page * D,), float("nan"), dtype=torch.bfloat16, device="cuda")
    small = torch.randn(3, page, D, device="cuda").bfloat16()
    for j in range(3):
        pool[j * stride:j * stride + page * D] = small[j].ravel()
    table, lens = torch.tensor([[2, 0, 1]], device="cuda"), torch.tensor([41], device="cuda")
    q = torch.randn(1, 4 * D, device="cuda").bfloat16()
    outs = []
    for k, st in ((pool, stride), (small, page * D)):
        out = torch.zeros(1, 4 * D, device="cuda")
        tpp.tpp_paged_attention(tpp.tpp_attn_desc(4, tpp.TPP_DT_F32, 0.125, 0, 41),
                                tpp.tpp_kv_cache(k.data_ptr(), k.data_ptr(), tpp.TPP_DT_BF16, D, 1,
                                                 page, 3, st, D, D), 1, q, 4 * D, lens, table, 3, out,
                                4 * D, None, None, None, 0, tpp.current_stream())
        torch.cuda.synchronize()
        outs.append(out)
    assert torch.equal(*outs) and not outs[0].isnan().any() and outs[0].any()
    # and an eviction that moves the last page's last row to the first place of a page below it
    totals = torch.ones(1, 41, device="cuda")
    totals[0, 3] = 0
    n_out = torch.zeros(1, dtype=torch.int64, device="cuda")
    tpp.tpp_cache_evict(tpp.tpp_kv_cache(pool.data_ptr(), pool.data_ptr(), tpp.TPP_DT_BF16, D, 1, page, 3,
                                         stride, D, D), 1, 41, 40, lens, table, 3, totals, None, None, 41,
                        n_out, totals, None, tpp.current_stream())
    torch.cuda.synchronize()
    assert n_out.item() == 40
    assert torch.equal(pool[2 * stride + 3 * D:2 * stride + 4 * D], small[1, 8])


# ---- eviction ---------------------------------------------------------------------------------------
def run_evict(tpp, pc, budget, totals, pos, horizon, max_len, in_place):
    n, ldt = totals.shape
    d_tot, d_pos = up(totals), None if pos is None else up(pos)
    d_hor = None if pos is None else up(np.asarray(horizon, np.int64))
    lens = pc.d_lens.clone()
    if in_place:
        t_out, p_out, l_out = d_tot, d_pos, lens
    else:
        t_out = torch.full_like(d_tot, -5.0)
        p_out = None if pos is None else torch.full_like(d_pos, -5)
        l_out = torch.full_like(lens, -5)
    tpp.tpp_cache_evict(pc.c(tpp), n, max_len, budget, lens, pc.d_pages, pc.pages.shape[1], d_tot, d_pos,
                        d_hor, ldt, l_out, t_out, p_out, tpp.current_stream())
    torch.cuda.synchronize()
    return l_out.cpu().numpy(), t_out.cpu().numpy(), None if pos is None else p_out.cpu().numpy()


EVICT = [  # lens, budget, D, heads, page, dtype, kind of totals, positions
    ([0, 1, 63, 64, 65, 66, 130], 64, 64, 2, 16, "bf16", "random", None),
    ([0, 1, 63, 64, 65, 66, 130], 64, 77, 3, 7, "f32", "ties", 16),
    ([129, 128, 127], 128, 128, 8, 16, "bf16", "random", 5),
    ([1000, 1024, 1025, 17, 400], 100, 32, 1, 1, "bf16", "ties", 30),
    ([1000, 1024, 1025, 17, 400], 0, 9, 2, 64, "bf16", "random", None),
    ([300, 5], 1, 64, 2, 16, "f32", "equal", None),
    ([300, 299], 40, 64, 2, 16, "bf16", "odd", 3),
    ([3000, 1], 2999, 40, 1, 16, "bf16", "odd", None),
    ([5000, 4097, 2222], 1111, 16, 2, 32, "f32", "ties", 700),
    ([70, 80], 10, 64, 1, 16, "bf16", "random", 75),       # more protected than the budget holds
    ([20000, 4097], 19999, 8, 1, 64, "bf16", "ties", 50),  # one leaves of more than 16 positions a thread
    ([32768, 20001], 19000, 8, 1, 64, "bf16", "random", 50),
    ([70000, 32769], 69990, 8, 1, 64, "bf16", "ties", 500),    # several parts
    ([33000, 40000], 30000, 8, 1, 64, "f32", "odd", 3000),
    ([2000, 1999], 1996, 64, 8, 16, "bf16", "equal", 100),     # a few leave, one by one
    ([2000, 1999], 1997, 64, 8, 16, "bf16", "odd", None),
    ([30, 29, 28], 26, 32, 2, 16, "bf16", "odd", 28),          # fewer candidates than have to leave
    ([8192, 4097, 20, 8191], 8189, 64, 2, 16, "bf16", "random", 90),   # one launch of several positions a thread
    ([6000, 5901, 4500], 5900, 8, 2, 7, "f32", "ties", 300),
]


@pytest.mark.parametrize("case", EVICT, ids=lambda c: f"L{max(c[0])}-B{c[1]}-D{c[2]}-{c[5]}-{c[6]}-{c[7]}")
@pytest.mark.parametrize("in_place", [False, True])
def test_evict(tpp, case, in_place):
    lens, budget, D, hk, page, dtype, kind, recent = case
    pc = Paged(lens, D, hk, page, dtype, seed=budget, pad=1, first=1,
               holes=[(0, 1), (len(lens) - 1, 2)] if kind == "random" else ())
    rng = np.random.default_rng(budget + D)
    n, ldt = len(lens), max(lens) + 4
    totals = rng.standard_normal((n, ldt)).astype(np.float32) if kind != "ties" else \
        rng.integers(0, 4, (n, ldt)).astype(np.float32)
    if kind == "equal":
        totals[:] = 0.25
    if kind == "odd":
        at = rng.random((n, ldt))
        for lo, x in ((0.5, 0.0), (0.6, -0.0), (0.7, np.nan), (0.8, np.inf), (0.9, -np.inf), (0.95, 1e-42)):
            totals[at > lo] = x
    pos = horizon = None
    if recent is not None:
        pos = np.stack([rng.permutation(ldt) for _ in range(n)]).astype(np.int64)
        horizon = ldt - recent - np.arange(n)
    new, keep = oracle.cache_evict(lens, budget, totals, pos, horizon)
    got_n, got_t, got_p = run_evict(tpp, pc, budget, totals, pos, horizon, max(lens) + 1, in_place)
    assert got_n.tolist() == new.tolist()
    pools = [np.array(p) for p in pc.pool]
    for b in range(n):
        k = keep[b, :new[b]]
        assert got_t[b, :new[b]].tobytes() == totals[b, k].tobytes()
        tail = totals[b, new[b]:] if in_place else np.full(ldt - new[b], np.float32(-5))
        assert got_t[b, new[b]:].tobytes() == tail.tobytes()
        if pos is not None:
            assert np.array_equal(got_p[b, :new[b]], pos[b, k])
            assert np.array_equal(got_p[b, new[b]:], pos[b, new[b]:] if in_place else np.full(ldt - new[b], -5))
        for t in np.nonzero(k != np.arange(new[b]))[0]:
            a, s = pc.row(b, t), pc.row(b, k[t])
            if a is None or s is None:
                continue
            for h in range(hk):
                o = h * pc.strides[2]
                for p, was in zip(pools, pc.pool):
                    p[a + o:a + o + D] = was[s + o:s + o + D]
    for p, d in zip(pools, pc.dev):     # every element of both pools
        assert p.tobytes() == down(d, dtype).tobytes()


def test_evict_nothing(tpp):
    """A budget above every length only hands the totals on."""
    pc = Paged([5, 0, 30], 16, 1, 4, "bf16")
    totals = np.random.default_rng(0).random((3, 30)).astype(np.float32)
    n, t, _ = run_evict(tpp, pc, 30, totals, None, None, 30, False)
    assert n.tolist() == [5, 0, 30]
    for b, x in enumerate((5, 0, 30)):
        assert np.array_equal(t[b, :x], totals[b, :x]) and (t[b, x:] == -5).all()
    run_evict(tpp, pc, 0, np.zeros((3, 1), np.float32), None, None, 0, False)


# ---- the chain, streams and graphs --------------------------------------------------------------------
def chain_reference(wl):
    """Every step of the decode step through the oracle, on copies of its arrays; each output rounded
    to bf16 where the device stores bf16."""
    a = {k: np.array(v, copy=True) for k, v in wl.arrays.items()}
    qkv, ap, at, out, ev = wl.steps
    run_call_oracle(qkv, a)
    d, hq, hk = ap.dim, ap.q_heads, ap.k_heads
    flat, ld = a["qkv"].ravel(), (hq + 2 * hk) * d
    norm = lambda off, h, w: oracle.qk_norm_rope(flat[off:], ld, h, d, ap.rot_dim, ap.rot_form, a[w],
                                                 a["rot"], a["pos"], ap.eps, "bf16")
    bits = lambda x: wk.bf16_bits(x.astype(np.float32))
    a["q"][:] = bits(norm(0, hq, "wq")).reshape(a["q"].shape)
    rows = (-1, hk, d)
    a["kc"].reshape(rows)[a["slot"]] = bits(norm(hq * d, hk, "wk"))
    a["vc"].reshape(rows)[a["slot"]] = a["qkv"][:, (hq + hk) * d:].reshape(-1, hk, d)
    o, _, a["totals64"] = oracle.paged_attention(
        a["kc"], a["vc"], "bf16", d, hk, at.page, len(a["kc"]), (at.page * hk * d, hk * d, d), a["pages"],
        a["q"], hq * d, hq, a["lens"], at.scale, 0, a["totals"])
    a["o"][:] = bits(o).reshape(a["o"].shape)
    run_call_oracle(out, a)
    return a


def test_decode_step(tpp):
    """The chain as a server runs it: projections by the BRGEMM, cache, attention, eviction.  Up to the
    eviction against the oracle; the eviction exactly, by the device's own totals."""
    from paper_2104_05755_amd import torch_io
    wl = wk.decode_step()
    dev = torch_io.upload(wl)
    steps = [torch_io.prepare_step(s, dev) for s in wl.steps]
    for s in steps[:-1]:
        torch_io.launch_step(s, dev)
    torch.cuda.synchronize()
    ref = chain_reference(wl)
    for name, bar in (("qkv", 5e-3), ("q", 5e-3), ("kc", 5e-3), ("vc", 5e-3), ("o", 1e-2), ("y", 1e-2)):
        got, want = values(torch_io.to_host(dev[name], wl.arrays[name]), "bf16"), values(ref[name], "bf16")
        assert np.linalg.norm(got - want) <= bar * np.linalg.norm(want), name
    totals = dev["totals"].cpu().numpy()
    # what enters is rounded to bf16 before the scores: a weight is off by 2^-8 of |score| <= 8
    assert np.abs(totals - ref["totals64"]).max() <= 16 * 2.0 ** -8 * 8
    for b, n in enumerate(wl.arrays["lens"]):   # every head's weights add up to one
        assert abs((totals[b, :n] - wl.arrays["totals"][b, :n]).sum() - 16) < 1e-3
    before = {k: dev[k].cpu().numpy() for k in ("kc", "vc", "cached_pos")}
    torch_io.launch_step(steps[-1], dev)
    torch.cuda.synchronize()
    ev = wl.steps[-1]
    new, keep = oracle.cache_evict(wl.arrays["lens"], ev.budget, totals, wl.arrays["cached_pos"],
                                   wl.arrays["horizon"])
    assert np.array_equal(dev["lens"].cpu().numpy(), new) and (new <= ev.budget).all()
    for b in range(ev.seqs):
        k, at = keep[b, :new[b]], np.arange(new[b])
        assert np.array_equal(dev["totals"].cpu().numpy()[b, :new[b]], totals[b, k])
        assert np.array_equal(dev["cached_pos"].cpu().numpy()[b, :new[b]], before["cached_pos"][b, k])
        pg = wl.arrays["pages"][b]
        for x in ("kc", "vc"):
            got = dev[x].cpu().numpy()[pg[at // ev.page], at % ev.page]
            assert np.array_equal(got, before[x][pg[k // ev.page], k % ev.page])


def test_current_stream_is_torchs(tpp):
    assert tpp.current_stream() == torch.cuda.current_stream().cuda_stream
    with torch.cuda.stream(torch.cuda.Stream()):
        assert tpp.current_stream() == torch.cuda.current_stream().cuda_stream != 0
    assert tpp.current_stream() == torch.cuda.current_stream().cuda_stream


def test_side_stream(tpp):
    """All calls on a stream that is not torch's current one, beside work on that one."""
    pc = Paged([3000, 700], 128, 2, 16, "bf16", seed=1)
    q = draw(pc.rng, (2, 8 * 128), "bf16")
    totals = pc.rng.random((2, 3000)).astype(np.float32)
    want = attend(tpp, pc, q, 8, "f32", 0.1, totals=totals)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = attend(tpp, pc, q, 8, "f32", 0.1, totals=totals, stream=side.cuda_stream)
    for x, y in zip(want, got):
        assert x.tobytes() == y.tobytes()
    r = Rope((600, 4, 2, 64, 64, "halves", "bf16", 0, 0), 3)
    g = [draw(np.random.default_rng(1), (600, h * 64 + 1), "bf16") for h in (4, 2)]
    want = run_backward(tpp, r, g)
    got = run_backward(tpp, r, g, side.cuda_stream)
    for x, y in zip(want[0] + want[1], got[0] + got[1]):
        assert torch.equal(x.nan_to_num(9) if x.is_floating_point() else x,
                           y.nan_to_num(9) if y.is_floating_point() else y)


def test_graph_replays(tpp):
    """The attention, the backward pass and the eviction captured in one graph, replayed between eager
    calls that use and grow the same streams' work buffers; every replay gives the eager results."""
    pc = Paged([4000, 900, 1], 64, 2, 16, "bf16", seed=2)
    q = draw(pc.rng, (3, 8 * 64), "bf16")
    totals = pc.rng.random((3, 4000)).astype(np.float32)
    out, lse = torch.zeros(3, 512, device="cuda"), torch.zeros(3, 8, device="cuda")
    d_q, d_tot = up(q), up(totals)
    t_out, t_ev = torch.zeros_like(d_tot), torch.zeros_like(d_tot)
    l_ev = torch.zeros(3, dtype=torch.int64, device="cuda")
    r = Rope((500, 4, 2, 64, 64, "halves", "bf16", 0, 0), 3)
    g = [up(draw(np.random.default_rng(1), (500, h * 64), "bf16")) for h in (4, 2)]
    dx = [torch.zeros_like(x) for x in g]
    dw = [torch.zeros(64, device="cuda") for _ in range(2)]
    pools = [d.clone() for d in pc.dev]

    def all_calls(s):
        tpp.tpp_paged_attention(tpp.tpp_attn_desc(8, tpp.TPP_DT_F32, 0.125, 0, 4000), pc.c(tpp), 3, d_q,
                                512, pc.d_lens, pc.d_pages, pc.pages.shape[1], out, 512, lse, d_tot,
                                t_out, 4000, s)
        tpp.tpp_qk_norm_rope_backward(r.desc(tpp), 500, r.at[0], r.ld, r.at[1], r.ld, r.dev["w"][0],
                                      r.dev["w"][1], r.dev["rot"], r.dev["pos"], g[0], 256, g[1], 128,
                                      dx[0], 256, dx[1], 128, dw[0], dw[1], s)
        tpp.tpp_cache_evict(pc.c(tpp), 3, 4000, 500, pc.d_lens, pc.d_pages, pc.pages.shape[1], t_out,
                            None, None, 4000, l_ev, t_ev, None, s)

    results = [out, lse, t_out, t_ev, l_ev, *dx, *dw]

    def reset():
        for x in results:
            x.zero_()
        for d, p in zip(pc.dev, pools):
            d.copy_(p)

    all_calls(tpp.current_stream())
    torch.cuda.synchronize()
    want = [x.clone() for x in results + pc.dev]
    assert l_ev.tolist() == [500, 500, 1]
    reset()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        all_calls(tpp.current_stream())
    big = Paged([6000] * 4, 64, 2, 16, "bf16", seed=3)
    for _ in range(4):
        reset()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(results + pc.dev, want):
            assert torch.equal(x, y)
        attend(tpp, big, draw(big.rng, (4, 512), "bf16"), 8, "f32", 0.1,
               totals=np.zeros((4, 6000), np.float32))


# ---- weights in 32 bits -------------------------------------------------------------------------------
@pytest.mark.parametrize("D,hq", [(64, 16), (128, 16), (256, 16), (128, 64)])
def test_attention_weights_in_32_bits(tpp, D, hq):
    """A bf16 cache, an fp32 output: the softmax weights keep their 32 bits.  Two positions, scores 0 and
    s = q k exactly (one entry each), -4 <= s < 0; values 0 and 1, so that out = p = e^s / (1 + e^s).  In
    u = 2^-24: the scaled score (its factor and its product) is off by 2 u |s| log2 e, e^s by 8 u for that,
    by 2 u in the exponential; the sum of weights by half that; the sums and the quotient by 2 u each: below
    20 u in all.  64 heads to one key head with room for 65536 positions are two head tiles a workgroup."""
    n, room = 32, (65536 if hq == 64 else 0)
    pc = Paged([2] * n, D, 1, 16, "bf16", room=room)
    rng = np.random.default_rng(D + hq)
    one = wk.bf16_bits(np.ones(1, np.float32))[0]
    for b in range(n):
        a = pc.row(b, 0)
        k, v = (p[a:a + 2 * D].reshape(2, D) for p in pc.pool)
        k[:], v[0], v[1] = 0, 0, one
        k[1, b % D] = one
    pc.dev = [up(p) for p in pc.pool]
    s = wk.bf16_bits(-rng.uniform(2.0 ** -8, 4, (n, hq)).astype(np.float32)).reshape(n, hq)
    q = np.zeros((n, hq, D), np.uint16)
    q[np.arange(n), :, np.arange(n) % D] = s
    out, _, _ = attend(tpp, pc, q.reshape(n, hq * D), hq, "f32", 1.0, max_len=room or 2)
    p = 1 / (1 + np.exp(-values(s, "bf16").astype(np.float64)))
    off = np.abs(out.reshape(n, hq, D) - p[..., None]) / p[..., None]
    assert off.max() <= 20 * U, f"off by {off.max() / U:.0f} u"


# ---- infinities -----------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,hq,hk,page,lens,window,room,std", [
    (64, 4, 2, 16, [1, 2, 33, 100, 31], 0, 0, 1.0),
    (77, 6, 3, 7, [300, 45, 513, 700], 40, 0, 1.0),
    (128, 8, 2, 16, [3000, 2049, 17], 0, 0, 20.0),       # several spans, weights that 32 bits cannot hold
    (64, 2, 1, 64, [20000], 0, 0, 1.0),
    (256, 4, 1, 16, [600, 64], 0, 0, 20.0),
    (64, 24, 1, 16, [1500, 33], 0, 65536, 1.0)], ids=str)   # (spans of several blocks, two head tiles)
def test_attention_infinite_values(tpp, dtype, D, hq, hk, page, lens, window, room, std):
    """sum p_t v_t with p_t > 0: one infinity among the held values is the entry's result, two signs or a NaN
    are NaN; no other entry changes, and what lies outside the window or in unused places (NaN) counts nothing."""
    holes = [(len(lens) - 1, 1)] if page < 64 else []
    n, pad = len(lens), max(0, 40 - len(lens)) if room else 0
    pc = Paged(list(lens) + [0] * pad, D, hk, page, dtype, seed=D, holes=holes, room=room)
    inf = {"f32": np.float32(np.inf), "bf16": np.uint16(0x7F80)}[dtype]
    neg = {"f32": np.float32(-np.inf), "bf16": np.uint16(0xFF80)}[dtype]
    rng = np.random.default_rng(D)
    for b in range(n):
        lo = max(0, lens[b] - window) if window else 0
        held = [t for t in range(lo, lens[b]) if pc.row(b, t) is not None]
        first, last, some = held[0], held[-1], int(rng.choice(held))
        for t, e, x in ((last, 1, inf), (last, 3, neg), (first, 5, inf), (some, 7, neg), (first, 2, inf),
                        (last, 2, inf)):
            pc.pool[1][pc.row(b, t) + e] = x
        if lo > 0 and pc.row(b, lo - 1) is not None:   # outside the window
            pc.pool[1][pc.row(b, lo - 1) + 8] = inf
        if first != last:   # both signs, and a NaN beside an infinity
            pc.pool[1][pc.row(b, first) + 4], pc.pool[1][pc.row(b, last) + 4] = inf, neg
            pc.pool[1][pc.row(b, first) + 6], pc.pool[1][pc.row(b, last) + 6] = NAN[dtype], inf
    pc.dev = [up(p) for p in pc.pool]
    max_len = room or None
    check_attention(tpp, pc, hq, "f32", window=window, with_totals=True, std=std, max_len=max_len)
    check_attention(tpp, pc, hq, "bf16", window=window, std=std, max_len=max_len)


ROPE_INF = [  # q heads, k heads, D, rot_dim, form, dtype: by whole chunks, by others, by units
    (2, 1, 128, 64, "halves", "bf16"), (2, 1, 128, 0, "halves", "bf16"), (2, 1, 64, 32, "pairs", "bf16"),
    (2, 1, 64, 32, "halves", "f32"), (2, 1, 64, 6, "pairs", "f32"), (2, 1, 77, 38, "halves", "bf16"),
    (2, 1, 77, 32, "pairs", "f32"), (2, 1, 77, 0, "halves", "f32"), (2, 1, 77, 76, "pairs", "f32"),
    (2, 1, 72, 36, "halves", "f32"), (2, 1, 9, 4, "halves", "f32"), (2, 1, 6, 2, "pairs", "bf16"),
    (2, 1, 511, 10, "halves", "f32")]


@pytest.mark.parametrize("case", ROPE_INF, ids=str)
def test_norm_rope_infinities_behind_the_rotated_part(tpp, case):
    """An entry that is not rotated meets no other: an infinite weight shows in that entry's outputs alone, an
    infinite gradient in its own dw and, by the mean, in its head's dx."""
    hq, hk, D, R, form, dtype = case
    T, inf = 5, {"f32": np.float32(np.inf), "bf16": np.uint16(0x7F80)}[dtype]
    for e in sorted({R, R + 1, (R + D) // 2, D - 1} - {D}):
        r = Rope((T, hq, hk, D, R, form, dtype, 0, 0), e)
        r.pos[:] = np.arange(T) % 4
        r.dev["pos"] = up(r.pos)
        w = r.w[0].copy()
        r.w[0][e] = np.float32(np.inf)
        r.dev["w"] = [up(x) for x in r.w]
        outs = [up(np.full(T * h * D, NAN[dtype])) for h in (hq, hk)]
        tpp.tpp_qk_norm_rope(r.desc(tpp), T, r.at[0], r.ld, r.at[1], r.ld, r.dev["w"][0], r.dev["w"][1],
                             r.dev["rot"], r.dev["pos"], outs[0], hq * D, outs[1], hk * D, tpp.current_stream())
        torch.cuda.synchronize()
        ref = r.ref(0)
        assert np.isinf(ref[..., e]).all() and np.isfinite(np.delete(ref, e, -1)).all()
        rest = np.abs(np.delete(ref, e, -1)).max(-1, keepdims=True)
        close(down(outs[0], dtype).reshape(T, hq, D), ref, 64 * U * (1 + D / 64) * rest, dtype, f"entry {e}")
        r.w[0] = w
        r.dev["w"] = [up(x) for x in r.w]
        g = [draw(np.random.default_rng(e), (T, h * D + 1), dtype) for h in (hq, hk)]
        g[0][3, D + e] = inf           # token 3, head 1
        outs, dw = run_backward(tpp, r, g)
        with np.errstate(invalid="ignore"):
            dx, ref_w = oracle.qk_norm_rope_backward(r.flat[r.off[0]:], r.ld, hq, D, R, form, r.w[0], r.rot,
                                                     r.pos, EPS, dtype, g[0], hq * D + 1)
            bx, bw = gradient_bounds(r, 0, g[0], dx)
        assert np.isinf(ref_w[e]) and np.isfinite(np.delete(ref_w, e)).all()
        gf = g[0].copy()
        gf[3, D + e] = 0
        _, bw = gradient_bounds(r, 0, gf, dx)
        close(dw[0].cpu().numpy()[:D], ref_w, (64 + T * hq) * U * bw, "f32", f"dw, entry {e}")
        close(down(outs[0], dtype).reshape(T, hq, D), dx, bx, dtype, f"dx, entry {e}")


def test_norm_rope_more_rows_than_a_grid(tpp):
    """Heads of one entry go 16 to a workgroup: more than 2^28 of them would pass a grid's 2^32 threads.  In
    place; the bound of this file's head with two u more for the reference in fp32."""
    T, heads = (1 << 18) + 5, 1024
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    x = torch.randn(T, heads, generator=g, device="cuda").bfloat16()
    pos = torch.zeros(T, dtype=torch.int64, device="cuda")
    pos[7::1000] = -1
    pos[-2] = -1
    w = torch.tensor([1.25], device="cuda")
    ref = x.float()
    ref = ref / torch.sqrt(ref * ref + EPS) * w
    ref[pos < 0] = 0
    desc = tpp.tpp_qk_desc(1, 0, tpp.TPP_ROT_HALVES, heads, 0, tpp.TPP_DT_BF16, EPS, 1)
    print(f"norm of {T} x {heads} heads of one entry", flush=True)
    tpp.tpp_qk_norm_rope(desc, T, x, heads, None, 0, w, None, None, pos, x, heads, None, 0, tpp.current_stream())
    torch.cuda.synchronize()
    off = (x.float() - ref).abs()
    assert bool((off <= ref.abs() * (2.0 ** -8 + 70 * U)).all()) and bool((ref[-1] != 0).any())


def test_decode_step_totals(tpp):
    """The totals of the chain, position by position: against the oracle's weights for the queries, keys and
    values that the device itself has after its first two steps, with the bounds of check_attention.  Uniform
    weights, weights one position on and totals that nothing was added to are past those bounds."""
    from paper_2104_05755_amd import torch_io
    wl = wk.decode_step()
    dev = torch_io.upload(wl)
    for s in wl.steps[:3]:
        torch_io.launch_step(torch_io.prepare_step(s, dev), dev)
    torch.cuda.synchronize()
    at, a = wl.steps[2], {k: torch_io.to_host(dev[k], wl.arrays[k]) for k in ("q", "kc", "vc", "totals")}
    d, hq, hk, lens, was = at.dim, at.q_heads, at.k_heads, wl.arrays["lens"], wl.arrays["totals"].astype(np.float64)
    _, _, ref = oracle.paged_attention(a["kc"], a["vc"], "bf16", d, hk, at.page, len(a["kc"]),
                                       (at.page * hk * d, hk * d, d), wl.arrays["pages"], a["q"], hq * d, hq, lens,
                                       at.scale, 0, was)
    qn = np.abs(values(a["q"], "bf16")).reshape(len(lens), hq, d).sum(-1)
    rel = 2 * (d + 4) * U * at.scale * qn.max(-1) * np.abs(values(a["kc"], "bf16")).max() + \
        (64 + lens.max()) * U + 2.0 ** -20
    for b, n in enumerate(lens):
        more = ref[b, :n] - was[b, :n]
        bound = rel[b] * more + 1e-30
        close(a["totals"][b, :n].astype(np.float64), ref[b, :n], bound, "f32", f"totals of sequence {b}")
        limit = bound + U * np.abs(ref[b, :n])
        assert (more > limit).any()
        if n >= 8:
            assert (np.abs(hq / n - more) > limit).any() and (np.abs(np.roll(more, 1) - more) > limit).any()
        assert np.array_equal(a["totals"][b, n:], wl.arrays["totals"][b, n:])
