"""The oracle's norms, activations and 8-bit rows against values worked out in other ways: torch in
float64 (autograd for the gradients), rational arithmetic for the roundings, and small cases by hand;
and planted mistakes in copies of the oracle, which these pins have to catch."""
from __future__ import annotations

import os
import subprocess
import sys
from fractions import Fraction

import numpy as np
import pytest
import torch

import oracle

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
EPS = 0.25


def _torch_norm(v, form, w, c):
    if form == "none":
        return v
    if form == "layer":
        return torch.nn.functional.layer_norm(v, v.shape[1:], w, c, EPS)
    return v / torch.sqrt((v * v).mean(1, keepdim=True) + EPS) * w


@pytest.mark.parametrize("form", ["none", "rms", "layer"])
def test_norm_and_gradients(form):
    rng = np.random.default_rng(1)
    f, v = 9, (rng.standard_normal((5, 11)) + 0.5).astype(np.float32)
    w, c = (rng.uniform(0.5, 1.5, f).astype(np.float32) for _ in range(2))
    g = rng.standard_normal((5, f))
    tv, tw, tc = (torch.from_numpy(a).double().requires_grad_(True) for a in (v[:, :f].copy(), w, c))
    ref = _torch_norm(tv, form, tw, tc)
    got = oracle.norm(v, f, "f32", form, EPS, w, c if form == "layer" else None)
    assert np.allclose(got, ref.detach().numpy(), rtol=1e-12, atol=1e-14)
    ref.backward(torch.from_numpy(g))
    dv, dw, dc = oracle.norm_backward(v, f, "f32", form, EPS, w, g)
    assert np.allclose(dv, tv.grad.numpy(), rtol=1e-11, atol=1e-13)
    if form != "none":
        assert np.allclose(dw, tw.grad.numpy(), rtol=1e-11, atol=1e-13)
    assert np.allclose(dc, g.sum(0), rtol=1e-12)


@pytest.mark.parametrize("form", ["none", "relu", "gelu_tanh", "silu"])
def test_activations(form):
    z = np.concatenate([np.linspace(-9, 9, 41), [0.0]])
    t = torch.from_numpy(z).requires_grad_(True)
    fn = {"none": lambda x: x * 1, "relu": torch.relu, "silu": torch.nn.functional.silu,
          "gelu_tanh": lambda x: torch.nn.functional.gelu(x, approximate="tanh")}[form]
    ref = fn(t)
    ref.sum().backward()
    value, slope = oracle.act(z, form)
    assert np.allclose(value, ref.detach().numpy(), rtol=1e-12, atol=1e-15)
    assert np.allclose(slope, t.grad.numpy(), rtol=1e-10, atol=1e-13)


def test_rows_are_the_nearest():
    rng = np.random.default_rng(2)
    v = rng.standard_normal((6, 50)).astype(np.float32)
    v[1] = np.arange(50) * 0.5 - 12                    # ties: 127 v / 127 below
    v[1, 7] = 127
    v[2] = 0
    v[3, 5], v[4, 9] = np.inf, np.nan
    for group in (0, 16):
        q, s = oracle.q8_rows(v.astype(np.float64), group)
        for t in range(6):
            for j in range(0, 50, group or 50):
                part = v[t, j:j + (group or 50)]
                sc = s[t, j // (group or 50)]
                if not np.isfinite(part).all():
                    assert np.isnan(sc) and not q[t, j:j + (group or 50)].any()
                    continue
                top = np.abs(part).max()
                assert sc == np.float32(top) / np.float32(127)
                for e, x in enumerate(part):
                    k = round(Fraction(127) * Fraction(float(x)) / Fraction(float(top))) if top else 0
                    assert q[t, j + e] == k
    assert oracle.q8_rows(v[1:2].astype(np.float64))[0][0, :8].tolist() == [-12, -12, -11, -10, -10, -10, -9, 127]


def test_product():
    rng = np.random.default_rng(3)
    a, b = (rng.integers(-128, 128, s).astype(np.int8) for s in ((5, 23), (4, 21)))
    ref = b[:, :20].astype(np.int64) @ a[:, :20].astype(np.int64).T
    assert np.array_equal(oracle.q8_product(a, b, 20), ref)


MUTANTS = {
    "stats_without_eps": ("1.0 / sqrt(s / f + eps)", "1.0 / sqrt(s / f)"),
    "rms_with_mean": ("if (form == 2)\n    for (int32_t i = 0; i < f; ++i) m +=",
                      "if (form >= 1)\n    for (int32_t i = 0; i < f; ++i) m +="),
    "layer_without_shift": ("if (form == 2 && c) n += c[i];", ""),
    "gradient_without_level": ("if (form == 2) level += u / f;", ""),
    "gradient_without_along": ("along += u * n / f;", ""),
    "vector_gradient_with_w": ("dw[i] += gi * n;", "dw[i] += u * n;"),
    "relu_slope_at_zero": ("form == 1 ? (z[i] > 0 ? 1.0 : 0.0)", "form == 1 ? (z[i] >= 0 ? 1.0 : 0.0)"),
    "silu_slope": ("s + z[i] * s * (1.0 / (1.0 + exp(z[i])))", "s"),
    "ties_away": ("(k + 0.5) * top == a && (k & 1)) ++k;", "(k + 0.5) * top == a) ++k;"),
    "scale_of_128": ("(float)top / 127.0f", "(float)top / 128.0f"),
    "nan_not_marked": ("if (!isfinite(a)) bad = 1;", ""),
    "sign_dropped": ("(int8_t)(v[t * f + i] < 0 ? -k : k)", "(int8_t)k"),
    "product_of_unsigned": ("s += (int64_t)a[i * lda + p] * b", "s += (int64_t)(uint8_t)a[i * lda + p] * b"),
}


@pytest.mark.parametrize("name", sorted(MUTANTS))
def test_pins_catch_planted_mistakes(name, tmp_path):
    old, new = MUTANTS[name]
    src = open(os.path.join(ROOT, "oracle", "oracle.c")).read()
    assert src.count(old) == 1, f"mutant {name} no longer applies"
    path = tmp_path / "oracle.c"
    path.write_text(src.replace(old, new))
    lib = tmp_path / "liboracle_mutant.so"
    subprocess.run(["gcc", "-O1", "-fPIC", "-shared", "-std=c11", "-I", os.path.join(ROOT, "oracle"),
                    "-o", str(lib), str(path), "-lm"], check=True)
    r = subprocess.run([sys.executable, "-m", "pytest", "-x", "-q", "-p", "no:cacheprovider", __file__,
                        "-k", "not planted"], cwd=ROOT, capture_output=True, text=True,
                       env=dict(os.environ, ORACLE_LIB_OVERRIDE=str(lib)))
    assert r.returncode == 1, f"mutant {name} survived:\n{r.stdout[-800:]}"
