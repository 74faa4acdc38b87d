"""The measured work of the library's feed-forward operators: what a program that trains and serves a
transformer on it asks of ``include/tpp_residual.h`` and ``include/tpp_q8.h``.

Five families:

  norm      the residual stream between two blocks, r = x + scale * G(gate) * N_after(b) and the next
            block's input y = N_before(r), in one pass
  norm_bwd  its gradients: of x, of b, of the gate and of the norms' weights
  linear    a layer in 8-bit integers: each token quantised by its largest entry, multiplied with 8-bit
            weights that have a scale for each channel, bias and activation
  keep      an activation of training, its input kept in 8 bits, and the backward pass from what was kept
  ffn       the feed-forward half of a layer that serves tokens: norm to 8 bits, product, gated activation
            to 8 bits, product, norm

``own`` False: elementary torch operations in 32 bits (64 where a quotient is rounded to 8 bits), rounded
once at the end.  ``own`` True: the library's entry points.  ``exact`` is each definition in 64 bits,
written separately.

Layouts: activations are column-major 2D blocks, a column per token, so a torch tensor
``[tokens][features]``; weights are ``[channels][features]``.
"""
from __future__ import annotations

import math

import torch

own = False

_DT = {"f32": torch.float32, "bf16": torch.bfloat16}
_SIZE = {"f32": 4, "bf16": 2}
EPS = 1e-5
DEV = "cuda"


def listed():
    return [
        # One new token on its way through the residual stream, hidden size 1024: latency.
        dict(name="norm_one", family="norm", tokens=1, features=1024, after="rms", before="rms",
             gate="none", gate_every=0, dtype="bf16", pad=0),
        # The forward pass of training, 8192 tokens, a learned gate for each feature.
        dict(name="norm_train", family="norm", tokens=8192, features=4096, after="rms", before="rms",
             gate="identity", gate_every=0, dtype="bf16", pad=0),
        # Its backward pass.
        dict(name="norm_train_bwd", family="norm_bwd", tokens=8192, features=4096, after="rms",
             before="rms", gate="identity", gate_every=0, dtype="bf16", pad=0),
        # Odd everything: fp32, layer norms, gates made for each sequence of 100 tokens, rows that no
        # vector divides.
        dict(name="norm_odd_bwd", family="norm_bwd", tokens=1533, features=1001, after="layer",
             before="layer", gate="tanh", gate_every=100, dtype="f32", pad=3),
        # One token through one layer: latency.
        dict(name="linear_one", family="linear", tokens=1, k=1024, m=4096, act="none", bias=True,
             dtype="bf16", pad=0),
        # The first layer of the MLP block, 8192 tokens.
        dict(name="linear_mlp", family="linear", tokens=8192, k=1024, m=4096, act="gelu_tanh",
             bias=True, dtype="bf16", pad=0),
        # A wide layer over a long prompt.
        dict(name="linear_large", family="linear", tokens=8192, k=4096, m=16384, act="none",
             bias=False, dtype="bf16", pad=0),
        # fp32 in and out, sizes that no tile and no vector divides.
        dict(name="linear_odd", family="linear", tokens=1533, k=1001, m=777, act="relu", bias=True,
             dtype="f32", pad=0),
        # The MLP block's activation in training, 8192 tokens of 4096.
        dict(name="keep_train", family="keep", tokens=8192, features=4096, act="gelu_tanh",
             gated=False, group=128, dtype="bf16", pad=0),
        # A gated activation of odd length, fp32.
        dict(name="keep_odd", family="keep", tokens=1533, features=1001, act="silu", gated=True,
             group=64, dtype="f32", pad=1),
        # A server's step of one sequence: five calls, latency.
        dict(name="ffn_one", family="ffn", tokens=1, hidden=1024, inter=4096, act="silu", dtype="bf16"),
        # A step of 48 sequences, one token each, through a wide layer: the weights' bytes.
        dict(name="ffn_serve", family="ffn", tokens=48, hidden=4096, inter=8192, act="silu",
             dtype="bf16"),
    ]


# ---- draws -----------------------------------------------------------------------------------
def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """A size of a network: mostly a multiple of 64, sometimes of 8 or of nothing."""
    n = _logint(rng, lo, hi)
    by = rng.choice([64, 64, 64, 8, 1])
    return max(lo, n // by * by)


def draw(rng):
    family = rng.choice(["norm", "norm_bwd", "norm_bwd", "linear", "linear", "linear", "keep", "keep",
                         "ffn"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    pad = rng.choice([0, 0, 0, 8, 5])
    if family in ("norm", "norm_bwd"):
        f = _size(rng, 8, 16384)
        tokens = _logint(rng, 1, max(2, min(16384, 8192 * 4096 * 2 // (f * _SIZE[dtype]))))
        after, before = rng.choice([("rms", "rms"), ("rms", "rms"), ("layer", "layer"),
                                    ("none", "rms"), ("none", "layer"), ("rms", "none")])
        gate = rng.choice(["none", "identity", "identity", "sigmoid", "tanh"])
        every = rng.choice([0, 0, 1, 7, 256, 1024]) if gate != "none" else 0
        return dict(family=family, tokens=tokens, features=f, after=after, before=before, gate=gate,
                    gate_every=every, dtype=dtype, pad=pad)
    if family == "linear":
        k, m = _size(rng, 16, 8192), _size(rng, 16, 16384)
        most = 8192 * 4096 * 16384 // (k * m)
        return dict(family=family, tokens=_logint(rng, 1, max(2, min(16384, most))), k=k, m=m,
                    act=rng.choice(["none", "none", "relu", "gelu_tanh"]), bias=rng.random() < 0.5,
                    dtype=dtype, pad=pad)
    if family == "keep":
        f, gated = _size(rng, 16, 16384), rng.random() < 0.5
        most = 8192 * 4096 * 2 // (f * _SIZE[dtype] * (2 if gated else 1))
        return dict(family=family, tokens=_logint(rng, 1, max(2, min(16384, most))), features=f,
                    act=rng.choice(["relu", "gelu_tanh", "silu"]), gated=gated,
                    group=rng.choice([0, 32, 64, 128]), dtype=dtype, pad=pad)
    return dict(family=family, tokens=_logint(rng, 1, 512), hidden=_size(rng, 64, 4096),
                inter=_size(rng, 64, 8192), act=rng.choice(["silu", "gelu_tanh"]), dtype="bf16")


# ---- inputs ----------------------------------------------------------------------------------
class _Draws:
    def __init__(self, seed):
        self.g = torch.Generator(device=DEV)
        self.g.manual_seed(seed)

    def normal(self, shape, dtype=torch.float32, std=1.0):
        return (torch.randn(shape, generator=self.g, device=DEV) * std).to(dtype)

    def rows(self, n, f, pad, dtype, std=1.0):
        """n columns of f entries, f + pad apart; a few features are large, a few tokens are padding."""
        big = 1 + 7 * (torch.rand((f,), generator=self.g, device=DEV) < 0.01)
        x = torch.zeros((n, f + pad), dtype=dtype, device=DEV)[:, :f]
        x.copy_(torch.randn((n, f), generator=self.g, device=DEV) * std * big)
        x[96::97] = 0
        return x

    def weights8(self, m, k):
        """8-bit weights of m channels, their rows at multiples of 16, and the channels' scales."""
        w = torch.zeros((m, -(-k // 16) * 16), dtype=torch.int8, device=DEV)[:, :k]
        w.copy_((torch.randn((m, k), generator=self.g, device=DEV) * 36).round().clamp(-127, 127))
        s = (0.5 + torch.rand((m,), generator=self.g, device=DEV)) * (4 / 127 * k ** -0.5)
        return w, s


def _empty(n, f, pad, dtype):
    return torch.zeros((n, f + pad), dtype=dtype, device=DEV)[:, :f]


def _norm_prepare(c, seed):
    r, dt, n, f, p = _Draws(seed), _DT[c["dtype"]], c["tokens"], c["features"], c["pad"]
    st = dict(case=c, x=r.rows(n, f, p, dt), b=r.rows(n, f, p, dt, 2.0))
    for side in ("after", "before"):
        st["w_" + side] = 1 + r.normal((f,), std=0.1) if c[side] != "none" else None
        st["c_" + side] = r.normal((f,), std=0.1) if c[side] == "layer" else None
    if c["gate"] == "none":
        st["gate"] = None
    elif c["gate_every"]:   # made by a layer from each sequence
        st["gate"] = r.normal((-(-n // c["gate_every"]), f), dt, 0.5)
    else:                   # a parameter
        st["gate"] = r.normal((1, f), std=0.5)
    new = lambda: _empty(n, f, p, dt)
    vec = lambda want: torch.zeros((f,), device=DEV) if want is not None else None
    if c["family"] == "norm":
        st.update(r=new(), y=new() if c["before"] != "none" else None)
    else:
        st["r"] = st.pop("x")
        st.update(gr=r.rows(n, f, p, dt), gy=r.rows(n, f, p, dt) if c["before"] != "none" else None,
                  dx=new(), db=new(),
                  dgate=None if st["gate"] is None else torch.zeros_like(st["gate"]),
                  **{"d" + k: vec(st[k]) for k in ("w_after", "c_after", "w_before", "c_before")})
    return st


def _linear_prepare(c, seed):
    r, dt = _Draws(seed), _DT[c["dtype"]]
    st = dict(case=c, x=r.rows(c["tokens"], c["k"], c["pad"], dt))
    st["w"], st["ws"] = r.weights8(c["m"], c["k"])
    st["bias"] = r.normal((c["m"],), std=0.5) if c["bias"] else None
    st["y"] = _empty(c["tokens"], c["m"], c["pad"], dt)
    return st


def _keep_prepare(c, seed):
    r, dt, n, f, p = _Draws(seed), _DT[c["dtype"]], c["tokens"], c["features"], c["pad"]
    wide = 2 * f if c["gated"] else f
    return dict(case=c, z=r.rows(n, wide, p, dt), gh=r.rows(n, f, p, dt), h=_empty(n, f, p, dt),
                dz=_empty(n, wide, p, dt), h2=_empty(n, f, p, dt),
                dbias=torch.zeros((wide,), device=DEV),
                q=torch.zeros((n, -(-wide // 16) * 16), dtype=torch.int8, device=DEV),
                s=torch.zeros((n, -(-wide // c["group"]) if c["group"] else 1), device=DEV))


def _ffn_prepare(c, seed):
    r, dt, n, d, f = _Draws(seed), _DT[c["dtype"]], c["tokens"], c["hidden"], c["inter"]
    st = dict(case=c, x=r.rows(n, d, 0, dt), b=r.rows(n, d, 0, dt, 2.0))
    st["w1"], st["s1"] = r.weights8(2 * f, d)
    st["w2"], st["s2"] = r.weights8(d, f)
    for k in ("wa1", "wb1", "wa2", "wb2"):
        st[k] = 1 + r.normal((d,), std=0.1)
    q8 = lambda w: torch.zeros((n, -(-w // 16) * 16), dtype=torch.int8, device=DEV)
    st.update(q1=q8(d), t1=torch.zeros((n,), device=DEV), q2=q8(f), t2=torch.zeros((n,), device=DEV),
              r1=_empty(n, d, 0, dt), z=_empty(n, 2 * f, 0, dt), o=_empty(n, d, 0, dt),
              r2=_empty(n, d, 0, dt), y=_empty(n, d, 0, dt))
    return st


# ---- the plain forms -------------------------------------------------------------------------
def _stats(v, kind):
    """v without its mean (where the norm takes it off) and 1 / its root mean square."""
    if kind == "layer":
        v = v - v.sum(-1, keepdim=True) / v.shape[-1]
    return v, torch.rsqrt((v * v).sum(-1, keepdim=True) / v.shape[-1] + EPS)


def _normed(v, kind, w, c):
    if kind == "none":
        return v
    v, rs = _stats(v, kind)
    v = v * rs * w
    return v if c is None else v + c


def _gate_value(g, kind):
    if kind == "sigmoid":
        return 1 / (1 + torch.exp(-g))
    return torch.tanh(g) if kind == "tanh" else g


def _gate_rows(st, g):
    """The gate of each token, or of all."""
    c = st["case"]
    if not c["gate_every"]:
        return g
    return g[torch.arange(c["tokens"], device=DEV) // c["gate_every"]]


def _residual_plain(x, b, gate, after, before, wa, ca, wb, cb, dtype):
    n = _normed(b.float(), after, wa, ca)
    r = (x.float() + SCALE * (n if gate is None else gate * n)).to(dtype)
    return r, None if before == "none" else _normed(r.float(), before, wb, cb).to(dtype)


SCALE = 0.7   # of the residual branch


def _norm_plain(st):
    c = st["case"]
    gate = None
    if st["gate"] is not None:
        gate = _gate_rows(st, _gate_value(st["gate"].float(), c["gate"]))
    r, y = _residual_plain(st["x"], st["b"], gate, c["after"], c["before"], st["w_after"],
                           st["c_after"], st["w_before"], st["c_before"], st["x"].dtype)
    return dict(r=r, y=y)


def _norm_grad(v, g, kind, w):
    """Gradients of v, of the weights and of the shift from the gradient g of the norm."""
    if kind == "none":
        return g, None, None
    vc, rs = _stats(v, kind)
    vn = vc * rs
    u = g * w
    d = u - vn * ((u * vn).sum(-1, keepdim=True) / v.shape[-1])
    if kind == "layer":
        d = d - u.sum(-1, keepdim=True) / v.shape[-1]
    return d * rs, (g * vn).sum(0), g.sum(0) if kind == "layer" else None


def _norm_bwd_plain(st):
    c = st["case"]
    dt, got = st["r"].dtype, {}
    total = st["gr"].float()
    if c["before"] != "none":
        d, got["dw_before"], got["dc_before"] = _norm_grad(st["r"].float(), st["gy"].float(),
                                                           c["before"], st["w_before"])
        total = total + d
    got["dx"] = total.to(dt)
    b, dn = st["b"].float(), SCALE * total
    if st["gate"] is not None:
        v = _gate_value(st["gate"].float(), c["gate"])
        slope = {"identity": torch.ones_like(v), "sigmoid": v * (1 - v), "tanh": 1 - v * v}[c["gate"]]
        part = dn * _normed(b, c["after"], st["w_after"], st["c_after"])
        if c["gate_every"]:
            n, e = c["tokens"], c["gate_every"]
            full = torch.zeros((len(v) * e, c["features"]), device=DEV)
            full[:n] = part
            part = full.reshape(len(v), e, -1).sum(1)
        else:
            part = part.sum(0, keepdim=True)
        got["dgate"] = (part * slope).to(st["gate"].dtype)
        dn = dn * _gate_rows(st, v)
    d, got["dw_after"], got["dc_after"] = _norm_grad(b, dn, c["after"], st["w_after"])
    return dict(got, db=d.to(dt))


def _to8(h, group):
    """8-bit values of the rows of h (as floats) and the scale of each group of `group` entries (0: row)."""
    n, f = h.shape
    g = group or f
    full = torch.zeros((n, -(-f // g) * g), dtype=h.dtype, device=DEV)
    full[:, :f] = h
    full = full.reshape(n, -1, g)
    top = full.abs().amax(-1, keepdim=True)
    some = torch.where(top == 0, 1.0, top)
    if h.dtype == torch.bfloat16:   # 15 bits of the product: the fp32 quotient rounds as the true one
        q = torch.round((full.float() * 127) / some.float())
    else:
        q = torch.round((full.double() * 127) / some.double()).float()
    return q.reshape(n, -1)[:, :f], (top.float() / torch.full_like(top, 127, dtype=torch.float32))[..., 0]


def _act(z, kind):
    if kind == "relu":
        return torch.where(z > 0, z, 0.0)
    if kind == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))
    return z / (1 + torch.exp(-z)) if kind == "silu" else z


def _act_grad(z, kind):
    if kind == "relu":
        return torch.where(z > 0, 1.0, 0.0)
    if kind == "gelu_tanh":
        t = torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * (math.sqrt(2 / math.pi) * (1 + 0.134145 * z * z))
    s = 1 / (1 + torch.exp(-z))
    return s * (1 + z * (1 - s))


def _product_plain(q, s, w, ws, bias, act):
    """Sums below 2^24 are whole in fp32."""
    y = torch.matmul(q, w.float().t()) * s * ws
    return _act(y if bias is None else y + bias, act)


def _linear_plain(st):
    c = st["case"]
    q, s = _to8(st["x"], 0)
    st["y"].copy_(_product_plain(q, s, st["w"], st["ws"], st["bias"], c["act"]))
    return dict(y=st["y"])


def _gated(z, act):
    f = z.shape[1] // 2
    return _act(z[:, :f], act) * z[:, f:]


def _keep_plain(st):
    c = st["case"]
    z, f, act = st["z"].float(), c["features"], c["act"]
    h = _gated(z, act) if c["gated"] else _act(z, act)
    q, s = _to8(st["z"], c["group"])
    g = c["group"] or q.shape[1]
    z = q * s.repeat_interleave(g, 1)[:, :q.shape[1]]
    gh = st["gh"].float()
    if c["gated"]:
        a, u = z[:, :f], z[:, f:]
        dz, h2 = torch.cat([gh * u * _act_grad(a, act), gh * _act(a, act)], 1), _act(a, act) * u
    else:
        dz, h2 = gh * _act_grad(z, act), _act(z, act)
    dt = st["z"].dtype
    return dict(h=h.to(dt), dz=dz.to(dt), h2=h2.to(dt), dbias=dz.sum(0))


def _ffn_plain(st):
    c, dt = st["case"], _DT[st["case"]["dtype"]]
    r1, y1 = _residual_plain(st["x"], st["b"], None, "rms", "rms", st["wa1"], None, st["wb1"], None, dt)
    q, s = _to8(y1, 0)
    z = _product_plain(q, s, st["w1"], st["s1"], None, "none").to(dt)
    q, s = _to8(_gated(z.float(), c["act"]).to(dt), 0)
    o = _product_plain(q, s, st["w2"], st["s2"], None, "none").to(dt)
    r2, y2 = _residual_plain(r1, o, None, "rms", "rms", st["wa2"], None, st["wb2"], None, dt)
    return dict(r=r2, y=y2)


_PLAIN = {"norm": _norm_plain, "norm_bwd": _norm_bwd_plain, "linear": _linear_plain,
          "keep": _keep_plain, "ffn": _ffn_plain}


# ---- the library's entry points -----------------------------------------------------------------
def _code(tpp, dtype):
    return tpp.TPP_DT_BF16 if dtype == torch.bfloat16 else tpp.TPP_DT_F32


def _norm_desc(tpp, st):
    c = st["case"]
    norm = {"none": tpp.TPP_NORM_NONE, "rms": tpp.TPP_NORM_RMS, "layer": tpp.TPP_NORM_LAYER}
    gate = {"none": tpp.TPP_GATE_NONE, "identity": tpp.TPP_GATE_IDENTITY,
            "sigmoid": tpp.TPP_GATE_SIGMOID, "tanh": tpp.TPP_GATE_TANH}
    of = tpp.TPP_DT_F32 if st["gate"] is None else _code(tpp, st["gate"].dtype)
    return tpp.tpp_residual_desc(c["features"], _code(tpp, st["b"].dtype), norm[c["after"]],
                                 norm[c["before"]], gate[c["gate"]], of, SCALE, EPS, c["gate_every"])


def _norm_own(tpp, st):
    c, s = st["case"], tpp.current_stream()
    if "desc" not in st:
        st["desc"] = _norm_desc(tpp, st)
    ld = c["features"] + c["pad"]
    tpp.tpp_residual_norm(st["desc"], c["tokens"], st["x"], ld, st["b"], ld, st["gate"], c["features"],
                          st["w_after"], st["c_after"], st["w_before"], st["c_before"], st["r"], ld,
                          st["y"], ld, None, 0, None, s)
    return dict(r=st["r"], y=st["y"])


def _norm_bwd_own(tpp, st):
    c, s = st["case"], tpp.current_stream()
    if "desc" not in st:
        st["desc"] = _norm_desc(tpp, st)
    ld = c["features"] + c["pad"]
    tpp.tpp_residual_norm_backward(
        st["desc"], c["tokens"], st["b"], ld, st["gate"], c["features"], st["w_after"], st["c_after"],
        st["w_before"], st["r"], ld, st["gr"], ld, st["gy"], ld, st["dx"], ld, st["db"], ld,
        st["dgate"], c["features"], st["dw_after"], st["dc_after"], st["dw_before"], st["dc_before"], s)
    return {k: st[k] for k in ("dx", "db", "dgate", "dw_after", "dc_after", "dw_before", "dc_before")}


def _flags(tpp, act, bias):
    return {"none": 0, "relu": tpp.TPP_EPI_RELU, "gelu_tanh": tpp.TPP_EPI_GELU_TANH}[act] | (
        tpp.TPP_EPI_BIAS if bias else 0)


def _act_code(tpp, act):
    return {"none": tpp.TPP_ACT_NONE, "relu": tpp.TPP_ACT_RELU, "gelu_tanh": tpp.TPP_ACT_GELU_TANH,
            "silu": tpp.TPP_ACT_SILU}[act]


def _linear_own(tpp, st):
    c, s = st["case"], tpp.current_stream()
    if "desc" not in st:
        t = _code(tpp, st["x"].dtype)
        st["desc"] = tpp.tpp_q8_gemm_desc(c["m"], c["tokens"], c["k"], st["w"].stride(0),
                                          c["k"] + c["pad"], c["m"] + c["pad"], t, t,
                                          _flags(tpp, c["act"], c["bias"]))
    tpp.tpp_q8_linear(st["desc"], st["w"], st["ws"], st["x"], st["y"], st["bias"], s)
    return dict(y=st["y"])


def _keep_own(tpp, st):
    c, s = st["case"], tpp.current_stream()
    if "desc" not in st:
        st["desc"] = tpp.tpp_q8_desc(c["features"], c["group"], _code(tpp, st["z"].dtype),
                                     _act_code(tpp, c["act"]), c["gated"])
    f, wide, ldq, lds = c["features"], st["dbias"].shape[0], st["q"].stride(0), st["s"].stride(0)
    p = c["pad"]
    tpp.tpp_q8_act(st["desc"], c["tokens"], st["z"], wide + p, st["h"], f + p, st["q"], ldq, st["s"],
                   lds, s)
    tpp.tpp_q8_act_backward(st["desc"], c["tokens"], st["q"], ldq, st["s"], lds, st["gh"], f + p,
                            st["dz"], wide + p, st["h2"], f + p, st["dbias"], s)
    return {k: st[k] for k in ("h", "dz", "h2", "dbias")}


def _ffn_own(tpp, st):
    c, s, bf = st["case"], tpp.current_stream(), tpp.TPP_DT_BF16
    n, d, f = c["tokens"], c["hidden"], c["inter"]
    if "norm" not in st:
        st["norm"] = tpp.tpp_residual_desc(d, bf, tpp.TPP_NORM_RMS, tpp.TPP_NORM_RMS,
                                           tpp.TPP_GATE_NONE, tpp.TPP_DT_F32, SCALE, EPS, 0)
        ld1, ld2 = st["q1"].stride(0), st["q2"].stride(0)
        st["up"] = tpp.tpp_q8_gemm_desc(2 * f, n, d, st["w1"].stride(0), ld1, 2 * f, bf, bf, 0)
        st["act"] = tpp.tpp_q8_desc(f, 0, bf, _act_code(tpp, c["act"]), True)
        st["down"] = tpp.tpp_q8_gemm_desc(d, n, f, st["w2"].stride(0), ld2, d, bf, bf, 0)
    tpp.tpp_residual_norm(st["norm"], n, st["x"], d, st["b"], d, None, 0, st["wa1"], None, st["wb1"],
                          None, st["r1"], d, None, 0, st["q1"], st["q1"].stride(0), st["t1"], s)
    tpp.tpp_q8_gemm(st["up"], st["w1"], st["s1"], st["q1"], st["t1"], st["z"], None, s)
    tpp.tpp_q8_quantize(st["act"], n, st["z"], 2 * f, st["q2"], st["q2"].stride(0), st["t2"], 1, s)
    tpp.tpp_q8_gemm(st["down"], st["w2"], st["s2"], st["q2"], st["t2"], st["o"], None, s)
    tpp.tpp_residual_norm(st["norm"], n, st["r1"], d, st["o"], d, None, 0, st["wa2"], None, st["wb2"],
                          None, st["r2"], d, st["y"], d, None, 0, None, s)
    return dict(r=st["r2"], y=st["y"])


_OWN = {"norm": _norm_own, "norm_bwd": _norm_bwd_own, "linear": _linear_own, "keep": _keep_own,
        "ffn": _ffn_own}


# ---- the definitions in 64 bits ---------------------------------------------------------------
def _norm64(v, kind, w, shift):
    if kind == "none":
        return v
    if kind == "rms":
        return v / (v.pow(2).mean(-1, keepdim=True) + EPS).sqrt() * w
    v = (v - v.mean(-1, keepdim=True)) / (v.var(-1, unbiased=False, keepdim=True) + EPS).sqrt()
    return v * w + shift


def _branch64(c, b, gate, wa, ca):
    """What the block adds to the stream."""
    n = _norm64(b, c["after"], wa, ca) * SCALE
    if gate is None:
        return n
    g = {"identity": lambda v: v, "sigmoid": torch.sigmoid, "tanh": torch.tanh}[c["gate"]](gate)
    if c["gate_every"]:
        g = g.repeat_interleave(c["gate_every"], 0)[:c["tokens"]]
    return n * g


def _up64(st, k):
    return None if st[k] is None else st[k].double()


def _norm_exact(c, seed):
    st = _norm_prepare(c, seed)
    r = st["x"].double() + _branch64(c, st["b"].double(), _up64(st, "gate"), _up64(st, "w_after"),
                                     _up64(st, "c_after"))
    y = None
    if c["before"] != "none":
        y = _norm64(r.to(st["x"].dtype).double(), c["before"], st["w_before"].double(),
                    _up64(st, "c_before"))
    return dict(r=r, y=y)


def _norm_bwd_exact(c, seed):
    st = _norm_prepare(c, seed)
    leaf = {}
    for k in ("r", "b", "gate", "w_after", "c_after", "w_before", "c_before"):
        leaf[k] = None if st[k] is None else st[k].double().requires_grad_(True)
    total = st["gr"].double()
    got = dict.fromkeys(("dgate", "dw_after", "dc_after", "dw_before", "dc_before"))
    if c["before"] != "none":
        y = _norm64(leaf["r"], c["before"], leaf["w_before"], leaf["c_before"])
        on = [k for k in ("r", "w_before", "c_before") if leaf[k] is not None]
        g = dict(zip(on, torch.autograd.grad(y, [leaf[k] for k in on], st["gy"].double())))
        total = total + g["r"]
        got.update({"d" + k: g[k] for k in on[1:]})
    out = _branch64(c, leaf["b"], leaf["gate"], leaf["w_after"], leaf["c_after"])
    on = [k for k in ("b", "gate", "w_after", "c_after") if leaf[k] is not None]
    g = torch.autograd.grad(out, [leaf[k] for k in on], total)
    return dict(got, dx=total, **{"d" + k: v for k, v in zip(on, g)})


def _to8_64(h, group):
    """Groups as pieces of the row; whole quotients and halves are what they are in 64 bits."""
    q, s = [], []
    for piece in h.double().split(group or h.shape[1], 1):
        top = piece.abs().amax(1, keepdim=True)
        q.append(torch.round(piece * 127 / torch.where(top > 0, top, torch.ones_like(top))))
        s.append(top / 127)
    return q, s


def _act64(z, kind):
    if kind == "none":
        return z
    if kind == "relu":
        return torch.relu(z)   # its gradient at 0 is 0
    if kind == "silu":
        return z * torch.sigmoid(z)
    u = 2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)
    return z * torch.sigmoid(u)


def _product64(x, w, ws, bias, act):
    q, s = _to8_64(x, 0)
    y = q[0] @ w.double().t() * s[0] * ws.double()
    return _act64(y if bias is None else y + bias.double(), act)


def _linear_exact(c, seed):
    st = _linear_prepare(c, seed)
    return dict(y=_product64(st["x"], st["w"], st["ws"], st["bias"], c["act"]))


def _glu64(z, c):
    if not c.get("gated", True):
        return _act64(z, c["act"])
    a, u = z.chunk(2, 1)
    return _act64(a, c["act"]) * u


def _keep_exact(c, seed):
    st = _keep_prepare(c, seed)
    q, s = _to8_64(st["z"], c["group"])
    z = torch.cat([a * b for a, b in zip(q, s)], 1).requires_grad_(True)
    h2 = _glu64(z, c)
    dz, = torch.autograd.grad(h2, z, st["gh"].double())
    return dict(h=_glu64(st["z"].double(), c), dz=dz, h2=h2.detach(), dbias=dz.sum(0))


def _ffn_exact(c, seed):
    st = _ffn_prepare(c, seed)
    dt = _DT[c["dtype"]]
    form = dict(after="rms", gate="none", gate_every=0)
    r1 = (st["x"].double() + _branch64(form, st["b"].double(), None, st["wa1"].double(), None)).to(dt)
    y1 = _norm64(r1.double(), "rms", st["wb1"].double(), None).to(dt)
    z = _product64(y1, st["w1"], st["s1"], None, "none").to(dt)
    o = _product64(_glu64(z.double(), c).to(dt), st["w2"], st["s2"], None, "none").to(dt)
    r2 = r1.double() + _branch64(form, o.double(), None, st["wa2"].double(), None)
    return dict(r=r2, y=_norm64(r2.to(dt).double(), "rms", st["wb2"].double(), None))


# ---- what a pass has to move and compute ---------------------------------------------------------
def _norm_work(c):
    e, n, f = _SIZE[c["dtype"]], c["tokens"], c["features"]
    after, before = c["after"] != "none", c["before"] != "none"
    vecs = sum({"none": 0, "rms": 1, "layer": 2}[c[k]] for k in ("after", "before"))
    side = vecs * f * 4
    if c["gate"] != "none":
        side += -(-n // c["gate_every"]) * f * e if c["gate_every"] else f * 4
    if c["family"] == "norm":
        return dict(bytes=n * f * e * (3 + before) + side, flops=n * f * (3 + 4 * after + 4 * before))
    rows = 4 + 2 * before                        # b, gr, dx, db; r, gy
    return dict(bytes=n * f * e * rows + 2 * side, flops=n * f * (4 + 12 * after + 12 * before))


def _linear_work(c):
    e, n, k, m = _SIZE[c["dtype"]], c["tokens"], c["k"], c["m"]
    return dict(bytes=n * k * e + m * k + n * m * e + m * 4 * (2 if c["bias"] else 1),
                flops=2 * n * k * m)


def _keep_work(c):
    e, n, f = _SIZE[c["dtype"]], c["tokens"], c["features"]
    wide = 2 * f if c["gated"] else f
    scales = n * (-(-wide // c["group"]) if c["group"] else 1) * 4
    # z read, h and 8 bits written; 8 bits and gh read, dz and h written
    return dict(bytes=n * (wide * e + f * e + wide) + n * (wide + f * e + wide * e + f * e) +
                2 * scales + wide * 4, flops=30 * n * wide)


def _ffn_work(c):
    e, n, d, f = _SIZE[c["dtype"]], c["tokens"], c["hidden"], c["inter"]
    return dict(bytes=3 * d * f + (2 * f + 5 * d) * 4 + 4 * n * d * e, flops=6 * n * d * f)


_KINDS = {"norm": (_norm_prepare, _norm_exact, _norm_work),
          "norm_bwd": (_norm_prepare, _norm_bwd_exact, _norm_work),
          "linear": (_linear_prepare, _linear_exact, _linear_work),
          "keep": (_keep_prepare, _keep_exact, _keep_work),
          "ffn": (_ffn_prepare, _ffn_exact, _ffn_work)}


def prepare(case, seed):
    return _KINDS[case["family"]][0](case, seed)


def run(state):
    family = state["case"]["family"]
    if own:
        import paper_2104_05755_amd as tpp
        return _OWN[family](tpp, state)
    return _PLAIN[family](state)


def exact(case, seed):
    return _KINDS[case["family"]][1](case, seed)


def work(case):
    return _KINDS[case["family"]][2](case)
