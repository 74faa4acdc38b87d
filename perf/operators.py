"""The measured work of the library's attention operators: what a program that trains and serves a
transformer on it asks of ``include/tpp_attention.h``.

Six families over one paged key-value cache:

  rope        norms of every query and key head with the position rotation, in one pass
  rope_bwd    its gradients: dq, dk and the two norm weights'
  append      the same norms and rotation with the keys and values written to their cache slots
  attend      attention of one new token per sequence over the cache
  attend_acc  the same, adding every position's attention weight to a running total
  evict       the positions of least total weight leave the cache, others move into their places

``own`` False: elementary torch operations in 32 bits, rounded once at the end.  ``own`` True: the
library's entry points.  ``exact`` is each definition in 64 bits, written separately.

Layouts: activations are column-major 2D blocks, a column per token, so a torch tensor
``[tokens][heads * D]``; the caches are ``[page][token in page][head][D]``; row b of the page table
lists the pages of sequence b.  A table entry outside the pool is a page that holds nothing.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

_DT = {"f32": torch.float32, "bf16": torch.bfloat16}
_SIZE = {"f32": 4, "bf16": 2}
EPS = 1e-6
DEV = "cuda"


def listed():
    return [
        # The new token of one sequence on its way into the cache, 16 heads of 64 (hidden size 1024):
        # nothing but latency.
        dict(name="append_one", family="append", tokens=1, q_heads=16, k_heads=16, dim=64, rot=64,
             form="halves", dtype="bf16", page=16, pad=0),
        # A prompt of 2048 tokens written to the cache, grouped heads.
        dict(name="append_prompt", family="append", tokens=2048, q_heads=32, k_heads=8, dim=128,
             rot=128, form="halves", dtype="bf16", page=16, pad=0),
        # The forward pass of training, 8192 tokens.
        dict(name="rope_train", family="rope", tokens=8192, q_heads=32, k_heads=8, dim=128, rot=128,
             form="halves", dtype="bf16", pad=0),
        # Its backward pass.
        dict(name="rope_train_bwd", family="rope_bwd", tokens=8192, q_heads=32, k_heads=8, dim=128,
             rot=128, form="halves", dtype="bf16", pad=0),
        # Odd everything: fp32, a head that is only partly rotated, neighbouring pairs, token count
        # of no multiple, padding tokens.
        dict(name="rope_odd_bwd", family="rope_bwd", tokens=1533, q_heads=21, k_heads=7, dim=77,
             rot=32, form="pairs", dtype="f32", pad=16),
        # One short conversation: latency.
        dict(name="attend_one", family="attend", seqs=1, len_min=100, len_max=100, q_heads=16,
             k_heads=16, dim=64, dtype="bf16", page=16, window=0, holes=0),
        # A batch being served: 64 sequences of 1 to 8192 tokens, four queries to a key head.
        dict(name="attend_batch", family="attend", seqs=64, len_min=1, len_max=8192, q_heads=32,
             k_heads=8, dim=128, dtype="bf16", page=16, window=0, holes=0),
        # One long document.
        dict(name="attend_long", family="attend", seqs=1, len_min=131072, len_max=131072,
             q_heads=32, k_heads=8, dim=128, dtype="bf16", page=64, window=0, holes=0),
        # fp32, an odd head, pages of seven tokens, a window, sequences of length zero on, pages that
        # hold nothing.
        dict(name="attend_odd_f32", family="attend", seqs=13, len_min=0, len_max=1533, q_heads=21,
             k_heads=7, dim=77, dtype="f32", page=7, window=1000, holes=9),
        # The batch of a server that prunes its caches: weights totalled beside the output.
        dict(name="attend_totals", family="attend_acc", seqs=32, len_min=2049, len_max=4096,
             q_heads=32, k_heads=8, dim=128, dtype="bf16", page=16, window=0, holes=0),
        # The steady state of such a server: every sequence one token over its budget.
        dict(name="evict_step", family="evict", seqs=32, len_min=2049, len_max=2049, budget=2048,
             recent=128, k_heads=8, dim=128, dtype="bf16", page=16, steady=True),
        # After long prompts: three quarters of each cache go.
        dict(name="evict_prompt", family="evict", seqs=8, len_min=9001, len_max=16384, budget=4096,
             recent=512, k_heads=8, dim=128, dtype="bf16", page=16, steady=False),
    ]


# ---- draws -----------------------------------------------------------------------------------
_LARGEST = 64 * 4096 * 8 * 128 * 2 * 2   # bytes of keys and values that attend_batch reads


def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _heads(rng):
    k = rng.choice([1, 2, 4, 7, 8, 16])
    g = rng.choice([1, 1, 2, 3, 4, 4, 7, 8, 16, 24])
    return min(k * g, 64) // k * k, k


def draw(rng):
    family = rng.choice(["rope", "rope_bwd", "append", "attend", "attend", "attend", "attend_acc",
                         "evict"])
    q_heads, k_heads = _heads(rng)
    dim = rng.choice([32, 64, 64, 72, 77, 80, 96, 128, 128, 128, 192, 256])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    page = rng.choice([1, 7, 16, 16, 32, 64, 128, 256])
    base = dict(family=family, q_heads=q_heads, k_heads=k_heads, dim=dim, dtype=dtype)
    if family in ("rope", "rope_bwd", "append"):
        most = 8192 * 40 * 128 * 2 // ((q_heads + k_heads) * dim * _SIZE[dtype])
        c = dict(base, tokens=_logint(rng, 1, max(2, min(16384, most))),
                 rot=rng.choice([dim // 2 * 2, dim // 2 * 2, dim // 4 * 2, 0]),
                 form=rng.choice(["halves", "halves", "pairs"]), pad=rng.choice([0, 0, 5, 16]))
        return dict(c, page=page) if family == "append" else c
    seqs = _logint(rng, 1, 64)
    most = _LARGEST // 2 // (seqs * k_heads * dim * 2 * _SIZE[dtype])
    len_max = _logint(rng, 1 if family != "evict" else 16, max(32, min(65536, most)))
    len_min = rng.choice([0, len_max // 2, len_max])
    if family == "evict":
        budget = rng.choice([len_max - 1, len_max // 2, len_max // 4])
        return dict(family=family, k_heads=k_heads, dim=dim, dtype=dtype, seqs=seqs, page=page,
                    len_min=len_min, len_max=len_max, budget=budget,
                    recent=rng.choice([0, budget // 8, budget // 2]), steady=rng.random() < 0.5)
    return dict(base, seqs=seqs, len_min=len_min, len_max=len_max, page=page,
                window=rng.choice([0, 0, 0, max(1, len_max // 3)]), holes=rng.choice([0, 0, 0, 9]))


# ---- inputs ----------------------------------------------------------------------------------
class _Draws:
    def __init__(self, seed):
        self.g = torch.Generator(device=DEV)
        self.g.manual_seed(seed)

    def normal(self, shape, dtype=torch.float32):
        return torch.randn(shape, generator=self.g, device=DEV).to(dtype)

    def rand(self, shape):
        return torch.rand(shape, generator=self.g, device=DEV)

    def perm(self, n):
        return torch.randperm(n, generator=self.g, device=DEV)


def _zeros(shape, dtype):
    return torch.zeros(shape, dtype=dtype, device=DEV)


def _lens(c):
    """The lengths of a case's sequences, evenly spread; a seed only decides which has which."""
    n, lo, hi = c["seqs"], c["len_min"], c["len_max"]
    return [hi if n == 1 else lo + (hi - lo) * i // (n - 1) for i in range(n)]


def _rope_prepare(c, seed):
    r = _Draws(seed)
    n, d, dt = c["tokens"], c["dim"], _DT[c["dtype"]]
    hq, hk, rot = c["q_heads"], c["k_heads"], c["rot"]
    n_pos = n + 64
    # the output of a layer's one projection: query, key and value heads side by side in a column
    qkv = r.normal((n, (hq + 2 * hk) * d), dt)
    pos = torch.arange(n, device=DEV) + 7 + seed % 50
    if c["pad"]:
        pos[c["pad"] - 1::c["pad"]] = -1   # padding tokens
    ang = torch.arange(n_pos, device=DEV, dtype=torch.float64)[:, None] * (
        10000.0 ** (-torch.arange(0, rot, 2, device=DEV, dtype=torch.float64) / max(rot, 1)))
    st = dict(case=c, qkv=qkv, q=qkv[:, :hq * d], k=qkv[:, hq * d:(hq + hk) * d],
              v=qkv[:, (hq + hk) * d:], pos=pos,
              rot=torch.cat([ang.cos(), ang.sin()], 1).float().contiguous(), n_pos=n_pos,
              wq=1 + 0.1 * r.normal((d,)), wk=1 + 0.1 * r.normal((d,)),
              q_out=_zeros((n, hq * d), dt))
    if c["family"] == "rope_bwd":
        st.update(gq=r.normal((n, hq * d), dt), gk=r.normal((n, hk * d), dt),
                  dq=_zeros((n, hq * d), dt), dk=_zeros((n, hk * d), dt),
                  dwq=_zeros((d,), torch.float32), dwk=_zeros((d,), torch.float32))
    elif c["family"] == "rope":
        st.update(k_out=_zeros((n, hk * d), dt))
    else:
        pages = -(-n // c["page"]) + 3
        slot = r.perm(pages)[torch.arange(n, device=DEV) // c["page"]] * c["page"] + \
            torch.arange(n, device=DEV) % c["page"]
        if c["pad"]:
            slot[c["pad"] - 1::c["pad"]] = -1
        st.update(slot=slot, kc=r.normal((pages, c["page"], hk, d), dt),
                  vc=r.normal((pages, c["page"], hk, d), dt))
    return st


def _cache_prepare(c, seed):
    r = _Draws(seed)
    d, dt, hk, page = c["dim"], _DT[c["dtype"]], c["k_heads"], c["page"]
    lens = torch.tensor(_lens(c), device=DEV)[r.perm(c["seqs"])]
    per = max(1, -(-c["len_max"] // page))
    n_pages = c["seqs"] * per + 2
    table = r.perm(n_pages)[:c["seqs"] * per].reshape(c["seqs"], per).contiguous()
    if c.get("holes"):
        table[:, c["holes"] - 1::c["holes"]] = -1
    return r, dict(case=c, lens=lens, table=table, per=per, n_pages=n_pages,
                   kc=r.normal((n_pages, page, hk, d), dt), vc=r.normal((n_pages, page, hk, d), dt))


def _attend_prepare(c, seed):
    r, st = _cache_prepare(c, seed)
    n, hq, dt, L = c["seqs"], c["q_heads"], _DT[c["dtype"]], max(1, c["len_max"])
    st.update(q=r.normal((n, hq * c["dim"]), dt), out=_zeros((n, hq * c["dim"]), dt),
              lse=_zeros((n, hq), torch.float32))
    if c["family"] == "attend_acc":
        st.update(tot=r.rand((n, L)), tot_out=_zeros((n, L), torch.float32))
    return st


def _evict_prepare(c, seed):
    r, st = _cache_prepare(c, seed)
    n, L = c["seqs"], c["len_max"]
    tot = r.rand((n, L)) ** 4 * 8       # most positions get little weight, a few much
    tot = torch.where(r.rand((n, L)) < 0.05, torch.zeros_like(tot), tot)   # ties
    pos = torch.arange(L, device=DEV).expand(n, L)
    if c["steady"]:
        # a cache that has been pruned before: what it holds has stayed out of order
        pos = torch.argsort(r.rand((n, L)), dim=1) * 2
    st.update(tot=tot, pos=pos.contiguous(), tot_out=_zeros((n, L), torch.float32),
              pos_out=_zeros((n, L), torch.int64), len_out=_zeros((n,), torch.int64))
    top = 2 * L if c["steady"] else st["lens"]
    scale = 2 if c["steady"] else 1
    st["horizon"] = (top - scale * c["recent"]) + _zeros((n,), torch.int64)
    return st


# ---- the plain forms -------------------------------------------------------------------------
def _rotate(y, c, s, form, rot):
    """The rotation of [tokens][heads][D] by per-token cosines and sines [tokens][1][rot / 2]."""
    if form == "halves":
        a, b = y[..., :rot // 2], y[..., rot // 2:rot]
        return torch.cat([a * c - b * s, b * c + a * s, y[..., rot:]], -1)
    a, b = y[..., 0:rot:2], y[..., 1:rot:2]
    turned = torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2)
    return torch.cat([turned, y[..., rot:]], -1)


def _tokens_plain(st):
    c = st["case"]
    ok = (st["pos"] >= 0) & (st["pos"] < st["n_pos"])
    row = st["rot"][st["pos"].clamp(0, st["n_pos"] - 1)][:, None, :]
    return ok[:, None, None], row[..., :c["rot"] // 2], row[..., c["rot"] // 2:]


def _norm_plain(st, x, w, heads):
    c = st["case"]
    ok, cos, sin = _tokens_plain(st)
    x = x.float().reshape(c["tokens"], heads, c["dim"])
    y = x * torch.rsqrt((x * x).sum(-1, keepdim=True) / c["dim"] + EPS) * w
    return torch.where(ok, _rotate(y, cos, sin, c["form"], c["rot"]), 0.0)


def _rope_plain(st):
    c = st["case"]
    q = _norm_plain(st, st["q"], st["wq"], c["q_heads"])
    k = _norm_plain(st, st["k"], st["wk"], c["k_heads"])
    st["q_out"].copy_(q.reshape(c["tokens"], -1))
    if c["family"] == "rope":
        st["k_out"].copy_(k.reshape(c["tokens"], -1))
        return dict(q=st["q_out"], k=st["k_out"])
    held = st["slot"] >= 0
    rows = (-1, c["k_heads"], c["dim"])
    at = st["slot"][held]
    st["kc"].reshape(rows)[at] = k[held].to(st["kc"].dtype)
    st["vc"].reshape(rows)[at] = st["v"].reshape(rows)[held]
    return dict(q=st["q_out"], k=st["kc"], v=st["vc"])


def _grad_plain(st, x, g, w, heads):
    c = st["case"]
    ok, cos, sin = _tokens_plain(st)
    shape = (c["tokens"], heads, c["dim"])
    x, g = x.float().reshape(shape), g.float().reshape(shape)
    g = torch.where(ok, _rotate(g, cos, -sin, c["form"], c["rot"]), 0.0)
    r = torch.rsqrt((x * x).sum(-1, keepdim=True) / c["dim"] + EPS)
    xn = x * r
    u = g * w
    dx = r * (u - xn * ((u * xn).sum(-1, keepdim=True) / c["dim"]))
    return dx.reshape(c["tokens"], -1), (g * xn).sum((0, 1))


def _rope_bwd_plain(st):
    c = st["case"]
    dq, dwq = _grad_plain(st, st["q"], st["gq"], st["wq"], c["q_heads"])
    dk, dwk = _grad_plain(st, st["k"], st["gk"], st["wk"], c["k_heads"])
    return dict(dq=dq.to(st["dq"].dtype), dk=dk.to(st["dk"].dtype), dwq=dwq, dwk=dwk)


def _rows_of(st, L):
    """Cache row of each position [seqs][L], and whether it holds anything."""
    c = st["case"]
    t = torch.arange(L, device=DEV)
    page = st["table"][:, t // c["page"]]
    ok = (t < st["lens"][:, None]) & (page >= 0) & (page < st["n_pages"])
    return page.clamp(0, st["n_pages"] - 1) * c["page"] + t % c["page"], ok


def _attend_plain(st):
    c = st["case"]
    n, hk, d, L = c["seqs"], c["k_heads"], c["dim"], max(1, c["len_max"])
    rows, ok = _rows_of(st, L)
    t = torch.arange(L, device=DEV)
    if c["window"]:
        ok = ok & (t >= st["lens"][:, None] - c["window"])
    k = st["kc"].reshape(-1, hk, d)[rows].float().permute(0, 2, 3, 1).contiguous()
    v = st["vc"].reshape(-1, hk, d)[rows].float().permute(0, 2, 1, 3).contiguous()
    q = st["q"].float().reshape(n, hk, -1, d)
    s = torch.matmul(q, k) * d ** -0.5                       # [seqs][key heads][queries][L]
    s = s.masked_fill(~ok[:, None, None, :], -math.inf)
    top = s.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    e = torch.exp(s - top)
    total = e.sum(-1, keepdim=True)
    p = e / torch.where(total == 0, 1.0, total)
    out = torch.matmul(p, torch.where(ok[:, None, :, None], v, 0.0))
    st["out"].copy_(out.reshape(n, -1))
    got = dict(out=st["out"], lse=(top + torch.log(total)).reshape(n, -1))
    if c["family"] == "attend_acc":
        tot = st["tot"] + p.sum((1, 2))
        got["tot"] = torch.where(t < st["lens"][:, None], tot, st["tot_out"])
    return got


def _evict_plain(st):
    c = st["case"]
    L, hk, d = c["len_max"], c["k_heads"], c["dim"]
    t = torch.arange(L, device=DEV)
    held = t < st["lens"][:, None]
    may = held & (st["pos"] < st["horizon"][:, None])
    n = torch.minimum((st["lens"] - c["budget"]).clamp(min=0), may.sum(1))
    # the lowest totals first, equal ones by position, what has to stay last
    order = torch.sort(st["tot"], dim=1, stable=True).indices
    order = order.gather(1, torch.sort((~may).gather(1, order).to(torch.int8), dim=1,
                                       stable=True).indices)
    rank = torch.empty_like(order).scatter_(1, order, t.expand_as(order))
    gone = rank < n[:, None]
    left = (st["lens"] - n)[:, None]
    place, mover = (gone & (t < left)).nonzero(), (held & ~gone & (t >= left)).nonzero()
    tot, pos = st["tot"].clone(), st["pos"].clone()
    tot[place[:, 0], place[:, 1]] = st["tot"][mover[:, 0], mover[:, 1]]
    pos[place[:, 0], place[:, 1]] = st["pos"][mover[:, 0], mover[:, 1]]
    rows, _ = _rows_of(st, L)
    to, src = rows[place[:, 0], place[:, 1]], rows[mover[:, 0], mover[:, 1]]
    k, v = st["kc"].reshape(-1, hk, d), st["vc"].reshape(-1, hk, d)
    k[to], v[to] = k[src], v[src]
    return dict(len=left[:, 0], tot=torch.where(t < left, tot, st["tot_out"]),
                pos=torch.where(t < left, pos, st["pos_out"]), k=st["kc"], v=st["vc"])


_PLAIN = {"rope": _rope_plain, "append": _rope_plain, "rope_bwd": _rope_bwd_plain,
          "attend": _attend_plain, "attend_acc": _attend_plain, "evict": _evict_plain}


# ---- the library's entry points -----------------------------------------------------------------
def _code(tpp, c):
    return tpp.TPP_DT_BF16 if c["dtype"] == "bf16" else tpp.TPP_DT_F32


def _qk_desc(tpp, st):
    c = st["case"]
    form = tpp.TPP_ROT_HALVES if c["form"] == "halves" else tpp.TPP_ROT_PAIRS
    return tpp.tpp_qk_desc(c["dim"], c["rot"], form, c["q_heads"], c["k_heads"], _code(tpp, c), EPS,
                           st["n_pos"])


def _kv_cache(tpp, st):
    c, k = st["case"], st["kc"]
    return tpp.tpp_kv_cache(k.data_ptr(), st["vc"].data_ptr(), _code(tpp, c), c["dim"],
                            c["k_heads"], c["page"], k.shape[0], k.stride(0), k.stride(1),
                            k.stride(2))


def _rope_own(tpp, st):
    c, s = st["case"], tpp.current_stream()
    if "desc" not in st:
        st["desc"] = _qk_desc(tpp, st)
    ld = st["qkv"].stride(0)
    tpp.tpp_qk_norm_rope(st["desc"], c["tokens"], st["q"], ld, st["k"], ld, st["wq"], st["wk"],
                         st["rot"], st["pos"], st["q_out"], st["q_out"].stride(0), st["k_out"],
                         st["k_out"].stride(0), s)
    return dict(q=st["q_out"], k=st["k_out"])


def _append_own(tpp, st):
    c, s = st["case"], tpp.current_stream()
    if "desc" not in st:
        st["desc"], st["cache"] = _qk_desc(tpp, st), _kv_cache(tpp, st)
    ld = st["qkv"].stride(0)
    tpp.tpp_qk_norm_rope_append(st["desc"], c["tokens"], st["q"], ld, st["k"], ld, st["v"], ld,
                                st["wq"], st["wk"], st["rot"], st["pos"], st["q_out"],
                                st["q_out"].stride(0), st["cache"], st["slot"], s)
    return dict(q=st["q_out"], k=st["kc"], v=st["vc"])


def _rope_bwd_own(tpp, st):
    c, s = st["case"], tpp.current_stream()
    if "desc" not in st:
        st["desc"] = _qk_desc(tpp, st)
    ld, lq, lk = st["qkv"].stride(0), st["gq"].stride(0), st["gk"].stride(0)
    tpp.tpp_qk_norm_rope_backward(st["desc"], c["tokens"], st["q"], ld, st["k"], ld, st["wq"],
                                  st["wk"], st["rot"], st["pos"], st["gq"], lq, st["gk"], lk,
                                  st["dq"], lq, st["dk"], lk, st["dwq"], st["dwk"], s)
    return dict(dq=st["dq"], dk=st["dk"], dwq=st["dwq"], dwk=st["dwk"])


def _attend_own(tpp, st):
    c, s = st["case"], tpp.current_stream()
    if "desc" not in st:
        st["desc"] = tpp.tpp_attn_desc(c["q_heads"], _code(tpp, c), c["dim"] ** -0.5, c["window"],
                                       c["len_max"])
        st["cache"] = _kv_cache(tpp, st)
    acc = c["family"] == "attend_acc"
    tpp.tpp_paged_attention(st["desc"], st["cache"], c["seqs"], st["q"], st["q"].stride(0),
                            st["lens"], st["table"], st["per"], st["out"], st["out"].stride(0),
                            st["lse"], st["tot"] if acc else None, st["tot_out"] if acc else None,
                            st["tot"].stride(0) if acc else 0, s)
    got = dict(out=st["out"], lse=st["lse"])
    return dict(got, tot=st["tot_out"]) if acc else got


def _evict_own(tpp, st):
    c, s = st["case"], tpp.current_stream()
    if "cache" not in st:
        st["cache"] = _kv_cache(tpp, st)
    tpp.tpp_cache_evict(st["cache"], c["seqs"], c["len_max"], c["budget"], st["lens"], st["table"],
                        st["per"], st["tot"], st["pos"], st["horizon"], st["tot"].stride(0),
                        st["len_out"], st["tot_out"], st["pos_out"], s)
    return dict(len=st["len_out"], tot=st["tot_out"], pos=st["pos_out"], k=st["kc"], v=st["vc"])


_OWN = {"rope": _rope_own, "append": _append_own, "rope_bwd": _rope_bwd_own,
        "attend": _attend_own, "attend_acc": _attend_own, "evict": _evict_own}


# ---- the definitions in 64 bits ---------------------------------------------------------------
def _turn64(y, ang, form, rot):
    """Rotation as a product of complex numbers."""
    n = rot // 2
    a, b = (y[..., :n], y[..., n:rot]) if form == "halves" else (y[..., 0:rot:2], y[..., 1:rot:2])
    z = torch.complex(a, b) * ang
    z = torch.cat([z.real, z.imag], -1) if form == "halves" else torch.view_as_real(z).flatten(-2)
    return torch.cat([z, y[..., rot:]], -1)


def _norm64(st, x, w, heads):
    c = st["case"]
    ok = ((st["pos"] >= 0) & (st["pos"] < st["n_pos"])).double()[:, None, None]
    tab = st["rot"].double()[st["pos"].clamp(0, st["n_pos"] - 1)]
    ang = torch.complex(tab[:, :c["rot"] // 2].contiguous(), tab[:, c["rot"] // 2:].contiguous())
    x = x.unflatten(-1, (heads, c["dim"]))
    y = x / (x.pow(2).mean(-1, keepdim=True) + EPS).sqrt() * w
    return _turn64(y, ang[:, None], c["form"], c["rot"]) * ok


def _rope_exact(c, seed):
    st = _rope_prepare(c, seed)
    q = _norm64(st, st["q"].double(), st["wq"].double(), c["q_heads"]).flatten(1)
    k = _norm64(st, st["k"].double(), st["wk"].double(), c["k_heads"])
    if c["family"] == "rope":
        return dict(q=q, k=k.flatten(1))
    kc, vc = st["kc"].double(), st["vc"].double()
    at = [i for i, x in enumerate(st["slot"].tolist()) if x >= 0]
    to = st["slot"][at]
    kc.flatten(0, 1).index_copy_(0, to, k[at])
    vc.flatten(0, 1).index_copy_(0, to, st["v"].double().unflatten(-1, (c["k_heads"], -1))[at])
    return dict(q=q, k=kc, v=vc)


def _rope_bwd_exact(c, seed):
    st = _rope_prepare(c, seed)
    got = {}
    for name, heads in (("q", c["q_heads"]), ("k", c["k_heads"])):
        x = st[name].double().clone().requires_grad_(True)
        w = st["w" + name].double().requires_grad_(True)
        y = _norm64(st, x, w, heads).flatten(1)
        got["d" + name], got["dw" + name] = torch.autograd.grad(y, (x, w), st["g" + name].double())
    return got


def _seq_rows(st, b, lo, hi):
    """Rows and positions of sequence b's places lo .. hi - 1 that hold anything (host lists)."""
    page, pages = st["case"]["page"], st["table"][b].tolist()
    at = [t for t in range(lo, hi) if 0 <= pages[t // page] < st["n_pages"]]
    return [pages[t // page] * page + t % page for t in at], at


def _attend_exact(c, seed):
    st = _attend_prepare(c, seed)
    hk, d = c["k_heads"], c["dim"]
    out, lse = torch.zeros_like(st["out"], dtype=torch.float64), _zeros((c["seqs"], c["q_heads"]),
                                                                        torch.float64)
    lse.fill_(-math.inf)
    tot = st["tot"].double() if c["family"] == "attend_acc" else None
    for b, n in enumerate(st["lens"].tolist()):
        rows, at = _seq_rows(st, b, max(0, n - c["window"]) if c["window"] else 0, n)
        if tot is not None:
            tot[b, n:] = 0
        if not rows:
            continue
        rows = torch.tensor(rows, device=DEV)
        k = st["kc"].flatten(0, 1)[rows].double().transpose(0, 1).contiguous()
        v = st["vc"].flatten(0, 1)[rows].double().transpose(0, 1).contiguous()
        q = st["q"][b].double().reshape(hk, -1, d).transpose(1, 2).contiguous()
        s = torch.bmm(k, q) / math.sqrt(d)                     # [key heads][positions][queries]
        z = torch.logsumexp(s, 1)
        p = torch.exp(s - z[:, None])
        lse[b] = z.flatten()
        out[b] = torch.bmm(p.transpose(1, 2).contiguous(), v).flatten()
        if tot is not None:
            tot[b].index_add_(0, torch.tensor(at, device=DEV), p.sum((0, 2)))
    got = dict(out=out, lse=lse)
    return got if tot is None else dict(got, tot=tot)


def _evict_exact(c, seed):
    st = _evict_prepare(c, seed)
    k, v = st["kc"].double(), st["vc"].double()
    tot, pos = st["tot"].double().cpu().numpy(), st["pos"].cpu().numpy()
    tot_out, pos_out, len_out = np.zeros_like(tot), np.zeros_like(pos), []
    page, table = c["page"], st["table"].tolist()
    src, dst = [], []
    for b, n in enumerate(st["lens"].tolist()):
        hor = int(st["horizon"][b])
        cand = sorted((tot[b, t], t) for t in range(n) if pos[b, t] < hor)
        gone = {t for _, t in cand[:max(0, n - c["budget"])]}
        left = n - len(gone)
        free = sorted(t for t in gone if t < left)
        move = [t for t in range(left, n) if t not in gone]
        was = list(range(left))
        for to, frm in zip(free, move):
            was[to] = frm
            dst.append(table[b][to // page] * page + to % page)
            src.append(table[b][frm // page] * page + frm % page)
        tot_out[b, :left], pos_out[b, :left] = tot[b, was], pos[b, was]
        len_out.append(left)
    at = lambda x: torch.tensor(x, device=DEV, dtype=torch.int64)
    for x in (k, v):
        x.flatten(0, 1)[at(dst)] = x.flatten(0, 1)[at(src)]
    return dict(len=at(len_out), tot=torch.from_numpy(tot_out), pos=torch.from_numpy(pos_out), k=k,
                v=v)


# ---- what a pass has to move and compute ---------------------------------------------------------
def _rope_work(c):
    e, n, d = _SIZE[c["dtype"]], c["tokens"], c["dim"]
    hq, hk, rows = c["q_heads"], c["k_heads"], c["tokens"] * (c["q_heads"] + c["k_heads"])
    side = n * 8 + n * c["rot"] * 4 + 2 * d * 4          # positions, table rows, norm weights
    if c["family"] == "rope_bwd":
        return dict(bytes=3 * rows * d * e + side + 2 * d * 4, flops=16 * rows * d)
    b, f = 2 * rows * d * e + side, 8 * rows * d
    if c["family"] == "append":
        b += 2 * n * hk * d * e + n * 8
    return dict(bytes=b, flops=f)


def _attend_work(c):
    e, d, hk, hq, n = _SIZE[c["dtype"]], c["dim"], c["k_heads"], c["q_heads"], c["seqs"]
    lens = _lens(c)
    read = 0
    for x in lens:
        lo = max(0, x - c["window"]) if c["window"] else 0
        read += x - lo
        if c["holes"]:
            p = c["page"]
            read -= sum(max(0, min(x, (j + 1) * p) - max(lo, j * p))
                        for j in range(c["holes"] - 1, -(-x // p), c["holes"]))
    b = read * hk * d * e * 2 + sum(-(-x // c["page"]) for x in lens) * 8 + n * 8
    b += n * hq * (d * e * 2 + 4)
    if c["family"] == "attend_acc":
        b += sum(lens) * 8
    return dict(bytes=b, flops=4 * read * hq * d)


def _evict_work(c):
    e, row = _SIZE[c["dtype"]], c["k_heads"] * c["dim"]
    b = 0
    for x in _lens(c):
        may = max(0, x - c["recent"])
        n = min(max(0, x - c["budget"]), may)
        left = x - n
        b += 8 * 3 + 12 * x + 12 * left
        if n:   # the share of the free places that lie below the new length
            share = (left / x) if c["steady"] else min(1.0, left / may)
            b += int(n * share) * row * e * 2 * 2
    return dict(bytes=b, flops=sum(_lens(c)))


_KINDS = {"rope": (_rope_prepare, _rope_own, _rope_exact, _rope_work),
          "append": (_rope_prepare, _append_own, _rope_exact, _rope_work),
          "rope_bwd": (_rope_prepare, _rope_bwd_own, _rope_bwd_exact, _rope_work),
          "attend": (_attend_prepare, _attend_own, _attend_exact, _attend_work),
          "attend_acc": (_attend_prepare, _attend_own, _attend_exact, _attend_work),
          "evict": (_evict_prepare, _evict_own, _evict_exact, _evict_work)}


def prepare(case, seed):
    return _KINDS[case["family"]][0](case, seed)


def run(state):
    family = state["case"]["family"]
    if own:
        import paper_2104_05755_amd as tpp
        return _OWN[family](tpp, state)
    return _PLAIN[family](state)


def exact(case, seed):
    return _KINDS[case["family"]][2](case, seed)


def work(case):
    return _KINDS[case["family"]][3](case)
