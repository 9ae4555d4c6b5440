"""Host-side refusals of the batched serving step's operators: every check runs before any device work, so that
these calls need no GPU (none of them is one that would launch)."""
import ctypes

import pytest

E_ARG, E_SHAPE = -1, -2
P = 1 << 20   # a stand-in for a device pointer (aligned, never read on the host)


@pytest.fixture(scope="module")
def lib():
    from paper_2410_05165_gb300.build import build
    build()
    from paper_2410_05165_gb300 import load
    return load()


def _pages(**kw):
    from paper_2410_05165_gb300.binding import KvPages
    d = dict(d_k=P, d_v=P, k_type=1, v_type=1, n_pages=4, page_size=16, n_kv_heads=2, head_dim=64,
             k_stride=(16 * 128, 128, 64), v_stride=(16 * 128, 128, 64))
    d.update(kw)
    for s in ("k_stride", "v_stride"):
        d[s] = (ctypes.c_int64 * 3)(*d[s])
    return KvPages(**d)


def _plan(lib, **kw):
    d = dict(stream=None, n=3, q_len=P, kv_len=P, parent=None, page=16, table=P, width=4, free=P, n_free=P, T=8, words=0,
             cu_q=P, ctx=P, state=P, pages=P, req=P, pos=P, slot=P, mask=None)
    d.update(kw)
    return lib.atspeed_op_batch_plan(*d.values())


@pytest.mark.parametrize("kw,status", [
    (dict(q_len=None), E_ARG), (dict(kv_len=None), E_ARG), (dict(table=None), E_ARG), (dict(free=None), E_ARG),
    (dict(n_free=None), E_ARG), (dict(slot=None), E_ARG), (dict(pages=None), E_ARG), (dict(state=None), E_ARG), (dict(n=0), E_ARG), (dict(page=0), E_ARG),
    (dict(width=0), E_ARG), (dict(T=0), E_ARG), (dict(parent=P), E_ARG), (dict(mask=P, words=1), E_ARG),
    (dict(parent=P, mask=P, words=0), E_ARG), (dict(parent=P, mask=P, words=129), E_SHAPE), (dict(n=16385), E_SHAPE)])
def test_batch_plan_refuses(lib, kw, status):
    assert _plan(lib, **kw) == status


def _append(lib, cache, **kw):
    d = dict(stream=None, qkv=P, src=0, stride=512, T=3, heads=4, pages=ctypes.byref(cache), slot=P, pos=P,
             theta=10000.0, q=P, q_stride=256)
    d.update(kw)
    return lib.atspeed_op_rope_append(*d.values())


@pytest.mark.parametrize("pages,kw,status", [
    ({}, dict(qkv=None), E_ARG), ({}, dict(slot=None), E_ARG), ({}, dict(q=None), E_ARG), ({}, dict(pages=None), E_ARG),
    ({}, dict(T=0), E_ARG), ({}, dict(heads=-1), E_ARG), ({}, dict(src=2), E_ARG), ({}, dict(src=7), E_ARG),
    ({}, dict(stride=511), E_ARG), ({}, dict(stride=514), E_ARG), ({}, dict(q_stride=255), E_ARG), ({}, dict(q_stride=260), E_ARG),
    ({}, dict(qkv=P + 8), E_ARG), ({}, dict(q=P + 8), E_ARG), ({}, dict(theta=0.0), E_ARG), ({}, dict(theta=float("nan")), E_ARG),
    (dict(head_dim=24), {}, E_SHAPE), (dict(head_dim=272), {}, E_SHAPE), (dict(d_k=None), {}, E_ARG), (dict(d_v=P + 2), {}, E_ARG),
    (dict(k_type=2, v_type=1), {}, E_ARG), (dict(k_type=0, v_type=0), {}, E_ARG), (dict(k_stride=(2048, 100, 64)), {}, E_ARG),
    (dict(v_stride=(2048, 128, -64)), {}, E_ARG), (dict(n_pages=0), {}, E_ARG)])
def test_rope_append_refuses(lib, pages, kw, status):
    assert _append(lib, _pages(**pages), **kw) == status


def _attention(lib, cache, **kw):
    d = dict(stream=None, pages=ctypes.byref(cache), q=P, q_stride=256, heads=4, n=2, T=3, cu_q=P, ctx=P, table=P,
             width=4, mask=None, words=0, scale=0.125, out=P, out_stride=256, lse=None, ws=P)
    d.update(kw)
    return lib.atspeed_op_tree_attention(*d.values())


@pytest.mark.parametrize("pages,kw,status", [
    ({}, dict(q=None), E_ARG), ({}, dict(out=None), E_ARG), ({}, dict(cu_q=None), E_ARG), ({}, dict(ctx=None), E_ARG),
    ({}, dict(table=None), E_ARG), ({}, dict(ws=None), E_ARG), ({}, dict(ws=P + 16), E_ARG), ({}, dict(n=0), E_ARG),
    ({}, dict(T=0), E_ARG), ({}, dict(width=0), E_ARG), ({}, dict(mask=P, words=0), E_ARG), ({}, dict(scale=0.0), E_ARG),
    ({}, dict(scale=float("inf")), E_ARG), ({}, dict(scale=float("nan")), E_ARG), ({}, dict(q_stride=248), E_ARG),
    ({}, dict(out_stride=260), E_ARG), ({}, dict(q=P + 4), E_ARG), ({}, dict(heads=3), E_SHAPE), ({}, dict(n=16385), E_SHAPE),
    ({}, dict(heads=512, q_stride=1 << 15, out_stride=1 << 15), E_SHAPE), (dict(head_dim=96), {}, E_SHAPE),
    (dict(head_dim=256), dict(q_stride=1024, out_stride=1024), E_SHAPE), (dict(page_size=24), {}, E_SHAPE),
    (dict(page_size=512), {}, E_SHAPE), (dict(d_k=P + 8), {}, E_ARG), (dict(k_type=2, v_type=1), {}, E_ARG),
    (dict(v_stride=(2048, 128, 4)), {}, E_ARG)])
def test_tree_attention_refuses(lib, pages, kw, status):
    assert _attention(lib, _pages(**pages), **kw) == status


def _adjust(lib, fields, **kw):
    from paper_2410_05165_gb300.binding import LogitRulesDesc
    r = dict(n_req=2)
    r.update(fields)
    d = dict(stream=None, logits=P, in_type=1, ld_in=100, R=3, V=100, req=P, rules=ctypes.byref(LogitRulesDesc(**r)), mask=None,
             words=0, state=None, out=2 * P, out_type=1, ld_out=100)
    d.update(kw)
    return lib.atspeed_op_adjust_logits(*d.values())


@pytest.mark.parametrize("rules,kw,status", [
    ({}, dict(logits=None), E_ARG), ({}, dict(out=None), E_ARG), ({}, dict(req=None), E_ARG), ({}, dict(rules=None), E_ARG),
    ({}, dict(R=0), E_ARG), ({}, dict(V=0), E_ARG), ({}, dict(ld_in=99), E_ARG), ({}, dict(ld_out=99), E_ARG),
    ({}, dict(in_type=3), E_ARG), ({}, dict(in_type=0), E_ARG), ({}, dict(out_type=2), E_ARG), ({}, dict(logits=P + 1), E_ARG),
    ({}, dict(out=P, out_type=0), E_ARG), ({}, dict(out=P, ld_out=104), E_ARG), (dict(n_req=-1), {}, E_ARG),
    (dict(d_hist=P), {}, E_ARG), (dict(d_bias_off=P), {}, E_ARG), (dict(d_bias_off=P, d_bias_tok=P), {}, E_ARG),
    ({}, dict(mask=P, words=1), E_ARG), (dict(d_tree_tok=P, d_cu_q=P), dict(mask=P, words=0), E_ARG),
    ({}, dict(state=P), E_ARG), (dict(d_grammar=P, n_states=2, grammar_stride=3), dict(state=P), E_ARG),
    (dict(d_grammar=P, n_states=0, grammar_stride=4), dict(state=P), E_ARG)])
def test_adjust_logits_refuses(lib, rules, kw, status):
    assert _adjust(lib, rules, **kw) == status
