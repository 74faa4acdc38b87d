"""The oracle's attention functions against values worked out in other ways: torch in float64
(autograd for the gradients, its softmax and sorting), differences of the forward function, and small
cases by hand; and planted mistakes in copies of the oracle, which these pins have to catch."""
from __future__ import annotations

import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import oracle
import workloads as wk

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
EPS = 1e-5


def _rope_case(seed, tokens=5, heads=3, D=10, rot_dim=6, ld=41):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal(tokens * ld).astype(np.float32)
    ang = rng.uniform(-3, 3, (7, rot_dim // 2))
    rot = np.concatenate([np.cos(ang), np.sin(ang)], 1).astype(np.float32)
    w = rng.uniform(0.5, 1.5, D).astype(np.float32)
    pos = np.array([3, 0, -1, 6, 7][:tokens])   # -1 and 7 are outside the table
    return x, ld, rot, w, pos


def _torch_norm_rope(x, ld, heads, D, rot_dim, form, w, rot, pos):
    t = len(pos)
    v = x.reshape(t, ld)[:, :heads * D].reshape(t, heads, D)
    y = v / torch.sqrt((v ** 2).mean(-1, keepdim=True) + EPS) * w
    inside = torch.tensor([0 <= p < rot.shape[0] for p in pos])[:, None, None]
    row = torch.from_numpy(rot).double()[torch.tensor(pos).clamp(0, rot.shape[0] - 1)][:, None]
    h = rot_dim // 2
    c, s = row[..., :h], row[..., h:]
    a, b = (y[..., :h], y[..., h:rot_dim]) if form == "halves" else \
        (y[..., 0:rot_dim:2], y[..., 1:rot_dim:2])
    ra, rb = a * c - b * s, b * c + a * s
    turned = torch.cat([ra, rb], -1) if form == "halves" else torch.stack([ra, rb], -1).flatten(-2)
    return torch.where(inside, torch.cat([turned, y[..., rot_dim:]], -1), torch.zeros(()).double())


@pytest.mark.parametrize("form", ["halves", "pairs"])
@pytest.mark.parametrize("rot_dim", [0, 6, 10])
def test_norm_rope_and_gradients(form, rot_dim):
    heads, D = 3, 10
    x, ld, rot, w, pos = _rope_case(1, rot_dim=rot_dim)
    got = oracle.qk_norm_rope(x, ld, heads, D, rot_dim, form, w, rot, pos, EPS, "f32")
    tx = torch.from_numpy(x).double().requires_grad_(True)
    tw = torch.from_numpy(w).double().requires_grad_(True)
    ref = _torch_norm_rope(tx, ld, heads, D, rot_dim, form, tw, rot, pos)
    assert np.allclose(got, ref.detach().numpy(), rtol=1e-12, atol=1e-14)
    g = np.random.default_rng(2).standard_normal(len(pos) * heads * D).astype(np.float32)
    ref.backward(torch.from_numpy(g).double().reshape(ref.shape))
    dx, dw = oracle.qk_norm_rope_backward(x, ld, heads, D, rot_dim, form, w, rot, pos, EPS, "f32", g,
                                          heads * D)
    want = tx.grad.numpy().reshape(len(pos), ld)[:, :heads * D].reshape(dx.shape)
    assert np.allclose(dx, want, rtol=1e-11, atol=1e-13)
    assert np.allclose(dw, tw.grad.numpy(), rtol=1e-11, atol=1e-13)


def test_gradient_by_differences():
    """Central differences of the forward function in float32 inputs that hold x +- h exactly."""
    heads, D, rot_dim, h = 1, 6, 4, 2.0 ** -8
    x, ld, rot, w, pos = _rope_case(4, tokens=2, heads=1, D=6, rot_dim=4, ld=6)
    x = (np.round(x * 64) / 64).astype(np.float32)
    g = np.random.default_rng(3).standard_normal(12).astype(np.float32)
    f = lambda v: float((oracle.qk_norm_rope(v, ld, heads, D, rot_dim, "pairs", w, rot, pos, EPS, "f32")
                         .ravel() * g).sum())
    dx, _ = oracle.qk_norm_rope_backward(x, ld, heads, D, rot_dim, "pairs", w, rot, pos, EPS, "f32", g,
                                         6)
    for i in range(12):
        up, down = x.copy(), x.copy()
        up[i] += h
        down[i] -= h
        # the truncation error is h^2 / 6 of the third derivative, below 1e-3 here
        assert abs((f(up) - f(down)) / (2 * h) - dx.ravel()[i]) < 2e-3


def _cache(rng, lens, D, hk, page, holes=()):
    per = -(-max(lens) // page) if max(lens) else 1
    n_pages = len(lens) * per + 1
    pages = rng.permutation(n_pages)[:len(lens) * per].reshape(len(lens), per)
    for b, j in holes:
        pages[b, j] = -1 if j % 2 else n_pages
    k, v = (rng.standard_normal((n_pages, page, hk, D)).astype(np.float32) for _ in range(2))
    return k, v, pages, n_pages


@pytest.mark.parametrize("window", [0, 5])
def test_paged_attention(window):
    rng = np.random.default_rng(5)
    lens, D, hk, hq, page = [0, 1, 7, 20], 8, 2, 6, 3
    k, v, pages, n_pages = _cache(rng, lens, D, hk, page, holes=[(3, 1), (3, 6), (1, 0)])
    q = rng.standard_normal((4, hq * D)).astype(np.float32)
    tot = rng.random((4, 20))
    out, lse, got = oracle.paged_attention(k, v, "f32", D, hk, page, n_pages,
                                           (page * hk * D, hk * D, D), pages, q, hq * D, hq, lens,
                                           0.37, window, tot)
    for b, n in enumerate(lens):
        at = [(t, pages[b, t // page], t % page) for t in range(n)
              if 0 <= pages[b, t // page] < n_pages and (not window or t >= n - window)]
        for h in range(hq):
            if not at:
                assert lse[b, h] == -np.inf and not out[b, h].any()
                continue
            kk = torch.tensor(np.array([k[p, s, h // 3] for _, p, s in at])).double()
            vv = torch.tensor(np.array([v[p, s, h // 3] for _, p, s in at])).double()
            sc = 0.37 * (kk @ torch.from_numpy(q[b, h * D:(h + 1) * D]).double())
            pr = torch.softmax(sc, 0)
            assert np.allclose(out[b, h], (pr @ vv).numpy(), rtol=1e-10, atol=1e-12)
            assert np.isclose(lse[b, h], torch.logsumexp(sc, 0).item(), rtol=1e-12)
            for (t, _, _), x in zip(at, pr.tolist()):
                tot[b, t] += x
    assert np.allclose(got, tot, rtol=1e-12)


def test_evict_by_hand():
    nan, inf = float("nan"), float("inf")
    totals = np.array([[3, 1, 2, 1, 0, 5, 4, 9], [-0.0, 0.0, -0.0, 7, 1, 1, 1, 1],
                       [nan, inf, 2, nan, 0, 0, 0, 0], [1, 1, 1, 1, 1, 1, 1, 1]], np.float32)
    lens = [7, 4, 4, 8]
    new, keep = oracle.cache_evict(lens, 4, totals)
    assert new.tolist() == [4, 4, 4, 4]
    # 4 (0), 1 and 3 (both 1) leave; 5 and 6 move to places 1 and 3
    assert keep[0, :4].tolist() == [0, 5, 2, 6]
    assert keep[1, :4].tolist() == [0, 1, 2, 3] and keep[2, :4].tolist() == [0, 1, 2, 3]
    assert keep[3, :4].tolist() == [4, 5, 6, 7]
    new, keep = oracle.cache_evict(lens, 2, totals)
    assert keep[1, :2].tolist() == [2, 3]      # -0, +0 and -0 are equal: the lower positions leave
    assert keep[2, :2].tolist() == [0, 3]      # NaN stays longest
    pos = np.tile(np.arange(8), (4, 1))
    new, keep = oracle.cache_evict(lens, 0, totals, pos, [4, 0, 4, 8])
    assert new.tolist() == [3, 4, 0, 0]        # protected ones never leave
    assert keep[0, :3].tolist() == [4, 5, 6]


MUTANTS = {
    "norm_without_eps": ("1.0 / sqrt(sum / D + eps)", "1.0 / sqrt(sum / D)"),
    "norm_sum_not_mean": ("sqrt(sum / D + eps)", "sqrt(sum + eps)"),
    "turned_the_other_way": ("y[a] = ya * c - yb * s;", "y[a] = ya * c + yb * s;"),
    "forms_swapped": ("*a = pairs ? 2 * i : i;\n  *b = pairs ? 2 * i + 1 : i + rot_dim / 2;",
                      "*a = pairs ? i : 2 * i;\n  *b = pairs ? i + rot_dim / 2 : 2 * i + 1;"),
    "gradient_not_turned_back": ("u[a] = va * c + vb * s;", "u[a] = va * c - vb * s;"),
    "gradient_without_mean": ("mean += u[e] * xn / D;", "mean += 0.0 * xn;"),
    "weight_gradient_with_w": ("dw[e] += u[e] * xn;", "dw[e] += u[e] * xn * w[e];"),
    "place_in_page": ("t % c->page_size * c->pos_stride", "t / c->page_size * c->pos_stride"),
    "key_head": ("const int32_t hk = h / (q_heads / c->kv_heads);",
                 "const int32_t hk = h % c->kv_heads;"),
    "window_off_by_one": ("n > window ? n - window : 0", "n > window ? n - window + 1 : 0"),
    "missing_page_read": ("if (page < 0 || page >= c->n_pages) return -1;",
                          "if (page < 0 || page >= c->n_pages) return 0;"),
    "scale_dropped": ("s[t] *= scale;", "s[t] *= 1.0;"),
    "ties_by_last": ("if (best < 0 || less_total(w[t], w[best])) best = t;",
                     "if (best < 0 || !less_total(w[best], w[t])) best = t;"),
    "nan_first": ("if (x != x) return 0;", "if (x != x) return 1;"),
    "protected_leave": ("pos[b * ldt + t] >= horizon[b]", "pos[b * ldt + t] > horizon[b]"),
    "movers_from_the_end": ("keep[b * ldt + t] = from++;", "keep[b * ldt + t] = n - 1;"),
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
