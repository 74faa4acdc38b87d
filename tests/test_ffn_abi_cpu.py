"""The entry points of tpp_residual.h and tpp_q8.h on the host: struct layouts, what is refused with
which status, and the calls that have nothing to do.  No device work happens here."""
from __future__ import annotations

import ctypes

import pytest


@pytest.fixture(scope="module")
def tpp():
    import paper_2104_05755_amd as tpp
    return tpp


P, Q, R = 0x1000, 0x2000, 0x3000   # pointers that are only looked at
INV, UNS = "TPP_ERR_INVALID_ARG", "TPP_ERR_UNSUPPORTED"
NAN = float("nan")


def test_struct_layouts(tpp):
    assert ctypes.sizeof(tpp.tpp_residual_desc) == 40 and tpp.tpp_residual_desc.gate_every.offset == 32
    assert ctypes.sizeof(tpp.tpp_q8_desc) == 20
    assert ctypes.sizeof(tpp.tpp_q8_gemm_desc) == 56 and tpp.tpp_q8_gemm_desc.lda.offset == 16


def refused(tpp, status, f):
    with pytest.raises(tpp.TppError) as e:
        f()
    assert e.value.status == getattr(tpp, status), str(e.value)


def norm(tpp, dkw={}, tokens=3, desc=True, **kw):
    d = dict(features=64, dtype=1, after=1, before=2, gate=1, gate_type=0, scale=1.0, eps=1e-5, gate_every=0)
    a = dict(x=P, ldx=64, b=Q, ldb=64, gate=P, ldg=64, wa=P, ca=None, wb=P, cb=P, r=R, ldr=64, y=0x4000,
             ldy=64, q=P, ldq=64, qs=P)
    tpp.tpp_residual_norm(tpp.tpp_residual_desc(**dict(d, **dkw)) if desc else None, tokens,
                          *dict(a, **kw).values())


def norm_bwd(tpp, dkw={}, tokens=3, **kw):
    d = dict(features=64, dtype=1, after=2, before=2, gate=1, gate_type=0, scale=1.0, eps=1e-5, gate_every=0)
    a = dict(b=P, ldb=64, gate=P, ldg=64, wa=P, ca=P, wb=P, r=P, ldr=64, gr=P, ldgr=64, gy=P, ldgy=64, dx=Q,
             lddx=64, db=R, lddb=64, dgate=P, lddg=64, dwa=P, dca=P, dwb=P, dcb=P)
    tpp.tpp_residual_norm_backward(tpp.tpp_residual_desc(**dict(d, **dkw)), tokens, *dict(a, **kw).values())


BAD_DESC = [
    (INV, dict(features=0)), (INV, dict(features=-1)), (INV, dict(dtype=2)), (INV, dict(gate_type=-1)),
    (INV, dict(after=3)), (INV, dict(before=-1)), (INV, dict(gate=4)), (INV, dict(scale=NAN)),
    (INV, dict(eps=-1.0)), (INV, dict(eps=float("inf"))), (INV, dict(gate_every=-1)),
    (INV, dict(features=65))]   # the last: leading dimensions too small


@pytest.mark.parametrize("status,kw", BAD_DESC, ids=str)
def test_residual_refuses_descriptions(tpp, status, kw):
    refused(tpp, status, lambda: norm(tpp, kw))
    refused(tpp, status, lambda: norm_bwd(tpp, kw))


def test_residual_refuses_wide_rows(tpp):
    f = (1 << 20) + 1
    ld = {k: f for k in ("ldx", "ldb", "ldg", "ldr", "ldy", "ldq")}
    refused(tpp, UNS, lambda: norm(tpp, dict(features=f), **ld))


@pytest.mark.parametrize("kw", [
    dict(x=None), dict(b=None), dict(gate=None), dict(wa=None), dict(wb=None), dict(r=None), dict(ldx=63),
    dict(ldb=63), dict(ldg=63), dict(ldr=63), dict(ldy=63), dict(ldq=63), dict(q=None), dict(qs=None),
    dict(r=Q), dict(y=P), dict(y=R), dict(r=P, ldr=65), dict(y=Q, ldy=65), dict(tokens=-1),
    dict(desc=False)], ids=str)
def test_residual_refuses_arguments(tpp, kw):
    refused(tpp, INV, lambda: norm(tpp, **kw))


@pytest.mark.parametrize("kw", [
    dict(b=None), dict(gate=None), dict(wa=None), dict(wb=None), dict(r=None), dict(gr=None, gy=None),
    dict(ldb=63), dict(ldg=63), dict(ldr=63), dict(ldgr=63), dict(ldgy=63), dict(lddx=63), dict(lddb=63),
    dict(lddg=63), dict(dx=P), dict(db=P), dict(tokens=-1), dict(dkw=dict(gate=0)),
    dict(dkw=dict(after=0), dca=None), dict(dkw=dict(after=1)), dict(dkw=dict(before=0), dcb=None),
    dict(dkw=dict(before=1))], ids=str)
def test_residual_backward_refuses(tpp, kw):
    refused(tpp, INV, lambda: norm_bwd(tpp, **kw))


def test_residual_without_tokens(tpp):
    norm(tpp, tokens=0, x=None, b=None, r=None, y=None, q=None, qs=None, gate=None)
    norm_bwd(tpp, tokens=0, dwa=None, dca=None, dwb=None, dcb=None, dgate=None, b=None, r=None)


def rows(tpp, which, dkw={}, tokens=3, desc=True, **kw):
    d = tpp.tpp_q8_desc(**dict(dict(features=64, group=32, dtype=1, act=3, gated=1), **dkw)) if desc else None
    wide = dict(q=P, ldq=128, s=P, lds=4)
    if which == "quantize":
        a = dict(z=P, ldz=128, q=P, ldq=64, s=P, lds=2)
        return tpp.tpp_q8_quantize(d, tokens, *dict(a, **kw).values())
    if which == "act":
        a = dict(dict(z=P, ldz=128, h=Q, ldh=64), **wide)
        return tpp.tpp_q8_act(d, tokens, *dict(a, **kw).values())
    a = dict(wide, gh=P, ldgh=64, dz=Q, lddz=128, h2=R, ldh2=64, dbias=P)
    return tpp.tpp_q8_act_backward(d, tokens, *dict(a, **kw).values())


@pytest.mark.parametrize("which", ["quantize", "act", "backward"])
@pytest.mark.parametrize("status,dkw", [
    (INV, dict(features=0)), (INV, dict(group=-1)), (UNS, dict(group=8)), (UNS, dict(group=48)),
    (UNS, dict(group=1024)), (INV, dict(dtype=7)), (INV, dict(act=4)), (INV, dict(gated=2)),
    (UNS, dict(features=(1 << 19) + 1)), (INV, dict(features=65)), (INV, dict(group=16))], ids=str)
def test_rows_refuse_descriptions(tpp, which, status, dkw):
    refused(tpp, status, lambda: rows(tpp, which, dkw))


@pytest.mark.parametrize("which,kws", [
    ("quantize", [dict(z=None), dict(q=None), dict(s=None), dict(ldz=127), dict(ldq=63), dict(lds=1)]),
    ("act", [dict(z=None), dict(q=None), dict(s=None), dict(ldz=127), dict(ldh=63), dict(ldq=127),
             dict(lds=3), dict(h=P)]),
    ("backward", [dict(q=None), dict(s=None), dict(gh=None), dict(ldq=127), dict(lds=3), dict(ldgh=63),
                  dict(lddz=127), dict(ldh2=63), dict(dz=P), dict(h2=P, ldh2=65), dict(h2=Q)])], ids=str)
def test_rows_refuse_arguments(tpp, which, kws):
    for kw in kws + [dict(tokens=-1), dict(desc=False)]:
        refused(tpp, INV, lambda: rows(tpp, which, **kw))


def test_rows_without_tokens(tpp):
    rows(tpp, "quantize", tokens=0, z=None, q=None, s=None)
    rows(tpp, "act", tokens=0, z=None, q=None, s=None, h=None)
    rows(tpp, "backward", tokens=0, q=None, s=None, gh=None, dbias=None)


def product(tpp, which, dkw={}, desc=True, **kw):
    d = dict(m=64, n=3, k=40, lda=48, ldb=48, ldc=64, b_type=1, c_type=1, flags=tpp.TPP_EPI_BIAS)
    d = tpp.tpp_q8_gemm_desc(**dict(d, **dkw)) if desc else None
    a = dict(a=P, sa=P, b=Q, sb=P, c=R, bias=P) if which == "gemm" else dict(a=P, sa=P, x=Q, c=R, bias=P)
    f = tpp.tpp_q8_gemm if which == "gemm" else tpp.tpp_q8_linear
    f(d, *dict(a, **kw).values())


@pytest.mark.parametrize("which", ["gemm", "linear"])
def test_products_refuse(tpp, which):
    for status, dkw in ((INV, dict(m=0)), (INV, dict(n=-1)), (INV, dict(k=0)), (INV, dict(lda=39)),
                        (INV, dict(ldb=39)), (INV, dict(ldc=63)), (INV, dict(b_type=2)), (INV, dict(c_type=3)),
                        (INV, dict(flags=6)), (INV, dict(flags=8)), (INV, dict(flags=32)),
                        (UNS, dict(k=131072, lda=131072, ldb=131072)), (UNS, dict(n=2 ** 31 - 511)),
                        (UNS, dict(m=2 ** 31 - 1, ldc=2 ** 31))):
        refused(tpp, status, lambda: product(tpp, which, dkw))
    for kw in [dict(a=None), dict(sa=None), dict(c=None), dict(bias=None), dict(desc=False)] + (
            [dict(b=None), dict(sb=None)] if which == "gemm" else [dict(x=None), dict(c=Q)]):
        refused(tpp, INV, lambda: product(tpp, which, **kw))
    product(tpp, which, dict(n=0), a=None, c=None, bias=None)


OUTPUTS = ("dx", "db", "dgate", "dwa", "dca", "dwb", "dcb")


@pytest.mark.parametrize("first,second", [(a, b) for i, a in enumerate(OUTPUTS) for b in OUTPUTS[i + 1:]], ids=str)
def test_residual_backward_refuses_one_place_for_two_gradients(tpp, first, second):
    """Of two gradients stored to one place the call would lose one."""
    at = {k: 0x100000 * (i + 2) for i, k in enumerate(OUTPUTS)}
    refused(tpp, "TPP_ERR_INVALID_ARG", lambda: norm_bwd(tpp, **dict(at, **{second: at[first]})))
