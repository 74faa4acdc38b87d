"""Shared by the GPU tests of the residual norms and the 8-bit rows."""
from __future__ import annotations

import numpy as np
import torch

import workloads as wk
from helpers import values

U = 2.0 ** -24
HALF = {"f32": U, "bf16": 2.0 ** -8}   # a rounding, relative to the value


def draw(rng, n, f, ld, dtype, std=1.0, mean=0.0):
    """n rows of f entries, ld apart; what stands behind them is NaN.  A few features are large."""
    big = np.where(rng.random(f) < 0.05, 8.0, 1.0)
    x = np.full((n, ld), np.nan, np.float32)
    x[:, :f] = rng.standard_normal((n, f)) * std * big + mean
    return x if dtype == "f32" else wk.bf16_bits(x).reshape(n, ld)


def up(a, first=0):
    """A device copy whose first entry stands `first` entries into its allocation."""
    if a is None:
        return None
    a = np.ascontiguousarray(a)
    a = a.view(np.int16) if a.dtype == np.uint16 else a
    t = torch.empty(a.size + first, dtype=torch.from_numpy(a[:0].copy()).dtype, device="cuda")
    t[first:] = torch.from_numpy(a.reshape(-1).copy()).cuda()
    return t[first:].view(a.shape)


def blank(n, ld, dtype, first=0):
    a = np.full((n, ld), np.nan, np.float32) if dtype == "f32" else np.full((n, ld), 0x7FC0, np.uint16)
    return up(a, first)


def down(t):
    a = t.cpu().numpy()
    return a.view(np.uint16) if a.dtype == np.int16 else a


def typed(a):
    return "bf16" if a.dtype == np.uint16 else "f32"


def code(tpp, dtype):
    return tpp.TPP_DT_BF16 if dtype == "bf16" else tpp.TPP_DT_F32


def untouched(a, f):
    """Whether the entries behind each row's f are still the NaN they were."""
    return bool(np.isnan(values(a[:, f:], typed(a))).all())


def close(got, ref, bound, what):
    """|got - ref| <= bound and the rounding of got's type, everywhere; NaN and infinities where ref has
    them."""
    half = HALF[typed(got)]
    got = values(got, typed(got))
    fin = np.isfinite(ref)
    assert np.array_equal(got[~fin], ref[~fin], equal_nan=True), f"{what}: not finite elsewhere"
    bound = np.broadcast_to(bound, ref.shape)
    limit = bound + (np.abs(ref) + bound) * half + 1e-37
    off = np.abs(got[fin] - ref[fin])
    assert not np.isnan(off).any() and not (off > limit[fin]).any(), \
        f"{what}: off by {off.max():.3e}, up to {(off / limit[fin]).max():.2f} of what is allowed"
