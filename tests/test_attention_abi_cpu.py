"""The attention entry points on the host: struct layouts, what is refused with which status, and the
calls that have nothing to do.  No device work happens here."""
from __future__ import annotations

import ctypes

import pytest


@pytest.fixture(scope="module")
def tpp():
    import paper_2104_05755_amd as tpp
    return tpp


P = 0x1000   # a pointer that is only looked at


def test_struct_layouts(tpp):
    assert ctypes.sizeof(tpp.tpp_qk_desc) == 40 and tpp.tpp_qk_desc.n_positions.offset == 32
    assert ctypes.sizeof(tpp.tpp_kv_cache) == 64 and tpp.tpp_kv_cache.n_pages.offset == 32
    assert ctypes.sizeof(tpp.tpp_attn_desc) == 32 and tpp.tpp_attn_desc.window.offset == 16


def refused(tpp, status, f):
    with pytest.raises(tpp.TppError) as e:
        f()
    assert e.value.status == getattr(tpp, status), str(e.value)


def qk_desc(tpp, **kw):
    d = dict(head_dim=64, rot_dim=64, rot_form=0, q_heads=4, k_heads=2, dtype=1, eps=1e-6,
             n_positions=100)
    return tpp.tpp_qk_desc(**dict(d, **kw))


def cache(tpp, **kw):
    d = dict(k=P, v=P, dtype=1, head_dim=64, kv_heads=2, page_size=16, n_pages=8, page_stride=2048,
             pos_stride=128, head_stride=64)
    return tpp.tpp_kv_cache(**dict(d, **kw))


def rope(tpp, desc, tokens=3, **kw):
    a = dict(q=P, ldq=256, k=P, ldk=128, wq=P, wk=P, rot=P, pos=P, q_out=P, ldqo=256, k_out=P,
             ldko=128)
    tpp.tpp_qk_norm_rope(desc, tokens, *dict(a, **kw).values())


def append(tpp, desc, c, tokens=3, **kw):
    a = dict(q=P, ldq=256, k=P, ldk=128, v=P, ldv=128, wq=P, wk=P, rot=P, pos=P, q_out=P, ldqo=256)
    a = dict(a, **{k: v for k, v in kw.items() if k != "slot"})
    tpp.tpp_qk_norm_rope_append(desc, tokens, *a.values(), c, kw.get("slot", P))


def backward(tpp, desc, tokens=3, **kw):
    a = dict(q=P, ldq=256, k=P, ldk=128, wq=P, wk=P, rot=P, pos=P, gq=P, ldgq=256, gk=P, ldgk=128,
             dq=P, lddq=256, dk=P, lddk=128, dwq=P, dwk=P)
    tpp.tpp_qk_norm_rope_backward(desc, tokens, *dict(a, **kw).values())


def attend(tpp, c, n=2, q_heads=4, out_type=1, scale=0.1, window=0, max_len=40, **kw):
    a = dict(q=P, ldq=q_heads * 64, lens=P, pages=P, ld_pages=3, out=P, ldo=q_heads * 64, lse=P,
             totals_in=None, totals_out=None, ldt=0)
    d = tpp.tpp_attn_desc(q_heads, out_type, scale, window, max_len)
    tpp.tpp_paged_attention(d, c, n, *dict(a, **kw).values())


def evict(tpp, c, n=2, max_len=40, budget=8, **kw):
    a = dict(lens=P, pages=P, ld_pages=3, totals=P, pos=P, horizon=P, ldt=40, len_out=P,
             totals_out=P, pos_out=P)
    tpp.tpp_cache_evict(c, n, max_len, budget, *dict(a, **kw).values())


INV, UNS = "TPP_ERR_INVALID_ARG", "TPP_ERR_UNSUPPORTED"


@pytest.mark.parametrize("status,kw", [
    (INV, dict(head_dim=0)), (INV, dict(head_dim=-1)), (UNS, dict(head_dim=513)),
    (INV, dict(rot_dim=3)), (INV, dict(rot_dim=66)), (INV, dict(rot_dim=-2)),
    (INV, dict(rot_form=2)), (INV, dict(q_heads=-1)), (INV, dict(k_heads=-1)), (INV, dict(dtype=2)),
    (INV, dict(eps=-1.0)), (INV, dict(eps=float("nan"))), (INV, dict(n_positions=-1)),
    (INV, dict(q_heads=5)), (INV, dict(k_heads=3))], ids=str)   # the last two: ld too small
def test_norm_rope_refuses_descriptions(tpp, status, kw):
    big = dict(ldq=600, ldk=600, ldqo=600, ldko=600) if kw.get("head_dim") == 513 else {}
    if big:
        kw = dict(kw, q_heads=1, k_heads=1)
    refused(tpp, status, lambda: rope(tpp, qk_desc(tpp, **kw), 3, **big))


@pytest.mark.parametrize("kw", [dict(q=None), dict(k=None), dict(wq=None), dict(wk=None),
                                dict(rot=None), dict(pos=None), dict(q_out=None), dict(k_out=None),
                                dict(ldq=255), dict(ldk=127), dict(ldqo=255), dict(ldko=127)], ids=str)
def test_norm_rope_refuses_arguments(tpp, kw):
    refused(tpp, INV, lambda: rope(tpp, qk_desc(tpp), 3, **kw))


@pytest.mark.parametrize("kw", [dict(gq=None), dict(gk=None), dict(dq=None), dict(dk=None),
                                dict(dwq=None), dict(dwk=None), dict(ldgq=255), dict(ldgk=127),
                                dict(lddq=255), dict(lddk=127), dict(pos=None)], ids=str)
def test_backward_refuses(tpp, kw):
    refused(tpp, INV, lambda: backward(tpp, qk_desc(tpp), 3, **kw))


def test_append_refuses(tpp):
    d = qk_desc(tpp)
    for kw in (dict(v=None), dict(ldv=127), dict(slot=None)):
        refused(tpp, INV, lambda: append(tpp, d, cache(tpp), **kw))
    for kw in (dict(head_dim=32), dict(kv_heads=1), dict(dtype=0), dict(page_size=0), dict(k=None),
               dict(n_pages=-1), dict(pos_stride=-1)):
        refused(tpp, INV, lambda: append(tpp, d, cache(tpp, **kw)))
    refused(tpp, INV, lambda: append(tpp, d, None))
    refused(tpp, INV, lambda: rope(tpp, None))
    refused(tpp, INV, lambda: rope(tpp, d, -1))


@pytest.mark.parametrize("status,ckw,kw", [
    (INV, dict(kv_heads=0), {}), (INV, dict(kv_heads=3), {}), (UNS, dict(head_dim=257), {}),
    (UNS, dict(head_dim=7), {}), (INV, dict(dtype=5), {}), (INV, dict(page_size=0), {}),
    (INV, dict(v=None), {}), (INV, dict(page_stride=-1), {}), (INV, dict(n_pages=1 << 62), {}),
    (INV, {}, dict(n=-1)), (INV, {}, dict(q_heads=0)), (INV, {}, dict(q_heads=3, ldq=256, ldo=256)),
    (INV, {}, dict(out_type=7)), (INV, {}, dict(scale=float("inf"))), (INV, {}, dict(window=-1)),
    (INV, {}, dict(max_len=-1)), (UNS, {}, dict(max_len=(1 << 30) + 1)),
    (INV, {}, dict(ldq=255)), (INV, {}, dict(ldo=255)), (INV, {}, dict(ld_pages=2)),
    (INV, {}, dict(q=None)), (INV, {}, dict(out=None)), (INV, {}, dict(lens=None)),
    (INV, {}, dict(pages=None)), (INV, {}, dict(totals_in=P, ldt=40)),
    (INV, {}, dict(totals_out=P, ldt=39)), (UNS, {}, dict(n=1 << 40)), (UNS, {}, dict(n=1 << 30)),
    (UNS, dict(kv_heads=1), dict(q_heads=1 << 20, n=1 << 20))], ids=str)
def test_attention_refuses(tpp, status, ckw, kw):
    refused(tpp, status, lambda: attend(tpp, cache(tpp, **ckw), **kw))


@pytest.mark.parametrize("kw", [
    dict(n=-1), dict(max_len=-1), dict(budget=-1), dict(max_len=(1 << 30) + 1), dict(ldt=39),
    dict(ld_pages=2), dict(lens=None), dict(pages=None), dict(totals=None), dict(totals_out=None),
    dict(len_out=None), dict(pos=None), dict(horizon=None), dict(pos_out=None)], ids=str)
def test_evict_refuses(tpp, kw):
    refused(tpp, INV, lambda: evict(tpp, cache(tpp), **kw))


def test_evict_refuses_more_than_a_grid(tpp):
    refused(tpp, UNS, lambda: evict(tpp, cache(tpp), n=1 << 40))
    refused(tpp, UNS, lambda: evict(tpp, cache(tpp, kv_heads=64, page_size=1 << 28), max_len=1 << 30, ldt=1 << 30,
                                    ld_pages=4))


def test_nothing_to_do(tpp):
    none = dict(q=None, k=None, wq=None, wk=None, rot=None, pos=None)
    rope(tpp, qk_desc(tpp), 0, **none, q_out=None, k_out=None)
    rope(tpp, qk_desc(tpp, q_heads=0, k_heads=0), 3, **dict(none, pos=P, rot=P), q_out=None, k_out=None)
    append(tpp, qk_desc(tpp), cache(tpp), 0, **none, q_out=None, v=None, slot=None)
    attend(tpp, cache(tpp), n=0, q=None, out=None, lens=None, pages=None)
    evict(tpp, cache(tpp), n=0, lens=None, pages=None, totals=None, totals_out=None, len_out=None)


@pytest.mark.parametrize("kw,ckw", [
    (dict(n=1 << 23), {}),                                            # 2^24 workgroups of one launch
    (dict(n=1 << 18, max_len=1 << 15, ld_pages=1 << 11), {}),         # of its spans
    (dict(n=1 << 19, q_heads=64, max_len=1 << 15, ld_pages=1 << 11), dict(kv_heads=1)),   # of the join's rows
    (dict(n=1 << 19, max_len=1 << 13, ld_pages=1 << 9, totals_out=P, ldt=1 << 13), dict(kv_heads=1))],   # and positions
    ids=str)
def test_attention_refuses_a_grid_of_2_pow_32_threads(tpp, kw, ckw):
    """Before it asks for work space or launches anything."""
    refused(tpp, UNS, lambda: attend(tpp, cache(tpp, **ckw), **kw))


@pytest.mark.parametrize("kw", [dict(n=1 << 22), dict(n=1 << 22, budget=39),
                                dict(n=1 << 18, max_len=1 << 16, ldt=1 << 16, ld_pages=1 << 12)], ids=str)
def test_evict_refuses_a_grid_of_2_pow_32_threads(tpp, kw):
    a = dict(kw)
    refused(tpp, UNS, lambda: evict(tpp, cache(tpp), **dict(a, totals_out=2 * P)))
