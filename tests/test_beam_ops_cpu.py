"""Host-side refusals of beam selection, page fork, page copy and token compaction: every check runs before any device work, so that these
calls need no GPU (none of them is one that would launch)."""
import ctypes

import pytest
import torch

from test_step_ops_cpu import P, _pages
from test_step_ops_devices_cpu import BF16, F32, HERE, I32, OTHER, Launched, Stand, library as stand_library  # noqa: F401

E_ARG, E_SHAPE = -1, -2


@pytest.fixture(scope="module")
def lib():
    from paper_2410_05165_gb300.build import build
    build()
    from paper_2410_05165_gb300 import load
    return load()


def _select(lib, **kw):
    from paper_2410_05165_gb300.binding import BeamsDesc
    d = dict(d_logits=P, ld=100, type=0, R=3, vocab=100, n_req=2, width=10, norm=0, d_cu_beam=P, d_score=P, d_token=P, d_parent=P, d_out_score=P)
    names = dict(logits="d_logits", V="vocab", n="n_req", cu="d_cu_beam", state="d_state", grammar="d_grammar", stride="grammar_stride",
                 token="d_token", parent="d_parent", out="d_out_score")
    ws = kw.pop("ws", P)
    d.update((names.get(k, k), v) for k, v in kw.items())
    return lib.atspeed_op_beam_select(None, bytes(BeamsDesc(**d)), ws)


@pytest.mark.parametrize("kw,status", [
    (dict(logits=None), E_ARG), (dict(cu=None), E_ARG), (dict(token=None), E_ARG), (dict(parent=None), E_ARG), (dict(out=None), E_ARG),
    (dict(ws=None), E_ARG), (dict(ws=P + 8), E_ARG), (dict(R=0), E_ARG), (dict(V=0), E_ARG), (dict(n=0), E_ARG), (dict(width=0), E_ARG),
    (dict(ld=99), E_ARG), (dict(type=3), E_ARG), (dict(type=-1), E_ARG), (dict(logits=P + 2), E_ARG), (dict(type=1, logits=P + 1), E_ARG),
    (dict(norm=2), E_ARG), (dict(state=P), E_ARG), (dict(state=P, grammar=P, stride=3, n_states=1), E_ARG),
    (dict(state=P, grammar=P, stride=4, n_states=0), E_ARG), (dict(width=257), E_SHAPE), (dict(V=(1 << 30) + 1, ld=(1 << 30) + 1), E_SHAPE)])
def test_beam_select_refuses(lib, kw, status):
    assert _select(lib, **kw) == status


def test_null_descriptions_are_refused(lib):
    assert lib.atspeed_op_beam_select(None, None, P) == E_ARG and lib.atspeed_op_fork_pages(None, None) == E_ARG


def test_beam_select_workspace(lib):
    assert lib.atspeed_op_beam_select_workspace(0, 5, 5) == 0 and lib.atspeed_op_beam_select_workspace(5, 5, -1) == 0
    small, large = lib.atspeed_op_beam_select_workspace(1, 1, 1), lib.atspeed_op_beam_select_workspace(1 << 14, 1 << 17, 256)
    assert 0 < small < 4096 and small < large < 1 << 30


def _fork(lib, **kw):
    from paper_2410_05165_gb300.binding import PageForkDesc
    d = dict(n_old=4, n_new=4, table_width=3, page_size=16, n_pages=9, d_table=P, d_kv_len=P, d_ref=P, d_free=P, d_n_free=P, d_new_table=2 * P,
             d_new_len=2 * P, d_new_state=2 * P, d_src=P, d_dst=P, d_new_ref=2 * P, d_new_free=2 * P, d_new_n_free=2 * P)
    names = dict(width="table_width", page="page_size", kv="d_kv_len")
    d.update((names.get(k, k if k.startswith("n_") and k != "n_free" else "d_" + k), v) for k, v in kw.items())
    return lib.atspeed_op_fork_pages(None, bytes(PageForkDesc(**d)))


@pytest.mark.parametrize("kw,status", [(dict([(k, None)]), E_ARG) for k in (
    "table", "kv", "ref", "free", "n_free", "new_table", "new_len", "new_state", "src", "dst", "new_ref", "new_free", "new_n_free")] + [
    (dict(n_old=0), E_ARG), (dict(n_new=0), E_ARG), (dict(width=0), E_ARG), (dict(page=0), E_ARG), (dict(n_pages=0), E_ARG),
    (dict(n_new=5), E_ARG), (dict(new_table=P), E_ARG), (dict(new_ref=P), E_ARG), (dict(new_free=P), E_ARG), (dict(new_len=P), E_ARG),
    (dict(new_n_free=P), E_ARG), (dict(old_state=2 * P), E_ARG), (dict(length=2 * P), E_ARG),
    (dict(n_old=16385, parent=P), E_SHAPE), (dict(n_new=16385, parent=P), E_SHAPE), (dict(n_pages=(1 << 26) + 1), E_SHAPE)])
def test_fork_pages_refuses(lib, kw, status):
    assert _fork(lib, **kw) == status


def _array(*pages):
    return (type(pages[0]) * len(pages))(*pages)


OTHER_LAYERS = [dict(head_dim=32), dict(n_pages=5), dict(page_size=8), dict(n_kv_heads=1), dict(k_type=2, v_type=2), dict(k_stride=(4096, 128, 64)),
                dict(v_stride=(4096, 128, 64)), dict(d_k=None), dict(d_v=P + 8)]


def _copy(lib, layers, **kw):
    d = dict(stream=None, layers=layers, n_layers=0 if layers is None else len(layers), n=3, src=P, dst=P, length=None)
    d.update(kw)
    return lib.atspeed_op_copy_pages(*d.values())


def _compact(lib, layers, **kw):
    d = dict(stream=None, layers=layers, n_layers=0 if layers is None else len(layers), n=2, T=8, slot=P, cu_q=P, kv=P, state=None,
             keep=P, width=3, n_keep=P, new_len=P)
    d.update(kw)
    return lib.atspeed_op_compact_tokens(*d.values())


@pytest.mark.parametrize("call", [_copy, _compact])
def test_layers_of_two_kinds_are_refused(lib, call):
    for other in OTHER_LAYERS:
        assert call(lib, _array(_pages(), _pages(**other))) == E_ARG
    assert call(lib, None, n_layers=1) == E_ARG
    assert call(lib, _array(_pages()), n_layers=0) == E_ARG
    assert call(lib, _array(_pages(head_dim=20))) == E_SHAPE
    assert call(lib, _array(_pages(page_size=(1 << 20) + 1))) == E_SHAPE


@pytest.mark.parametrize("kw", [dict(src=None), dict(dst=None), dict(n=0)])
def test_copy_pages_refuses(lib, kw):
    assert _copy(lib, _array(_pages()), **kw) == E_ARG


@pytest.mark.parametrize("kw,status", [(dict([(k, None)]), E_ARG) for k in ("slot", "cu_q", "kv", "keep", "n_keep", "new_len")] + [
    (dict(n=0), E_ARG), (dict(T=0), E_ARG), (dict(width=0), E_ARG), (dict(n=16385), E_SHAPE)])
def test_compact_tokens_refuses(lib, kw, status):
    assert _compact(lib, _array(_pages()), **kw) == status


# ---------------------------------------------------------------------------------------------------
# the binding's own checks, with stand-ins for tensors
# ---------------------------------------------------------------------------------------------------
@pytest.fixture
def binding(stand_library, monkeypatch):  # noqa: F811
    from paper_2410_05165_gb300 import binding as b
    entry = b.load().__class__

    class Lib(entry):
        def __getattr__(self, name):
            return (lambda *a: 64) if name == "atspeed_op_beam_select_workspace" else super().__getattr__(name)

    monkeypatch.setattr(b, "load", Lib)
    monkeypatch.setattr(b, "_raw_alloc", lambda n, stream: 1 << 20)
    monkeypatch.setattr(b, "_raw_delete", lambda p: None)
    monkeypatch.setattr(Stand, "split_with_sizes", lambda self, sizes: [Stand((n,), self.dtype, self.device) for n in sizes], raising=False)
    monkeypatch.setattr(Stand, "view", lambda self, *shape: Stand(shape, self.dtype, self.device), raising=False)
    return b


def _b_select(b, **kw):
    a = dict(logits=Stand((4, 100), F32), cu_beam=Stand((3,), I32), width=5, score=Stand((4,), F32), final=Stand((4,), I32),
             grammar=Stand((2, 4), I32), state=Stand((4,), I32))
    a.update(kw)
    return b.op_beam_select(**a)


def _b_fork(b, **kw):
    a = dict(table=Stand((4, 6), I32), kv_len=Stand((4,), I32), ref=Stand((9,), I32), free=Stand((5,), I32), n_free=Stand((1,), I32), page_size=16,
             q_len=Stand((4,), I32), state=Stand((4,), I32), used=Stand((2,), I32), parent=Stand((7,), I32), length=Stand((7,), I32))
    a.update(kw)
    return b.op_fork_pages(**a)


def _cache(device=HERE, **kw):
    return Stand(kw.get("shape", (4, 16, 2, 64)), kw.get("dtype", BF16), device)


def _b_copy(b, layers=None, **kw):
    a = dict(src=Stand((3,), I32), dst=Stand((3,), I32), length=Stand((3,), I32))
    a.update(kw)
    return b.op_copy_pages(layers or b.CacheLayers([(_cache(), _cache())]), **a)


def _b_compact(b, layers=None, **kw):
    a = dict(slot=Stand((8,), torch.int64), cu_q=Stand((3,), I32), kv_len=Stand((2,), I32), keep=Stand((2, 3), I32), n_keep=Stand((2,), I32),
             state=Stand((2,), I32))
    a.update(kw)
    return b.op_compact_tokens(layers or b.CacheLayers([(_cache(), _cache())]), **a)


CALLS = {"select": (_b_select, dict(logits=Stand((4, 100), F32, OTHER), cu_beam=Stand((3,), I32, OTHER), score=Stand((4,), F32, OTHER),
                                    final=Stand((4,), I32, OTHER), grammar=Stand((2, 4), I32, OTHER), state=Stand((4,), I32, OTHER))),
         "fork": (_b_fork, dict(table=Stand((4, 6), I32, OTHER), kv_len=Stand((4,), I32, OTHER), ref=Stand((9,), I32, OTHER),
                                free=Stand((5,), I32, OTHER), n_free=Stand((1,), I32, OTHER), q_len=Stand((4,), I32, OTHER),
                                state=Stand((4,), I32, OTHER), used=Stand((2,), I32, OTHER), parent=Stand((7,), I32, OTHER),
                                length=Stand((7,), I32, OTHER))),
         "copy": (_b_copy, dict(src=Stand((3,), I32, OTHER), dst=Stand((3,), I32, OTHER), length=Stand((3,), I32, OTHER))),
         "compact": (_b_compact, dict(slot=Stand((8,), torch.int64, OTHER), cu_q=Stand((3,), I32, OTHER), kv_len=Stand((2,), I32, OTHER),
                                      keep=Stand((2, 3), I32, OTHER), n_keep=Stand((2,), I32, OTHER), state=Stand((2,), I32, OTHER)))}


@pytest.mark.parametrize("name", list(CALLS))
def test_binding_launches_what_is_right(binding, name):
    with pytest.raises(Launched):
        CALLS[name][0](binding)


@pytest.mark.parametrize("name,key", [(n, k) for n in CALLS for k in CALLS[n][1]])
def test_binding_refuses_tensors_of_another_device(binding, name, key):
    with pytest.raises(binding.AtSpeedError):
        CALLS[name][0](binding, **{key: CALLS[name][1][key]})
    with pytest.raises(binding.AtSpeedError):
        CALLS[name][0](binding, **{key: Stand(CALLS[name][1][key].shape, torch.int16)})   # a type that nothing here has


@pytest.mark.parametrize("name", list(CALLS))
def test_binding_refuses_a_stream_of_another_device(binding, name):
    import types
    with pytest.raises(binding.AtSpeedError):
        CALLS[name][0](binding, stream=types.SimpleNamespace(device=OTHER, cuda_stream=5))


@pytest.mark.parametrize("name,kw", [
    ("select", dict(logits=Stand((400,), F32))), ("select", dict(logits=Stand((0, 100), F32))), ("select", dict(width=0)),
    ("select", dict(cu_beam=Stand((1,), I32))), ("select", dict(score=Stand((3,), F32))), ("select", dict(final=Stand((3,), I32))),
    ("select", dict(state=Stand((3,), I32))), ("select", dict(state=None)), ("select", dict(grammar=None)), ("select", dict(grammar=Stand((8,), I32))),
    ("fork", dict(table=Stand((24,), I32))), ("fork", dict(table=Stand((5, 6), I32))), ("fork", dict(q_len=Stand((3,), I32))),
    ("fork", dict(state=Stand((3,), I32))), ("fork", dict(length=Stand((6,), I32))), ("fork", dict(n_free=Stand((0,), I32))),
    ("fork", dict(parent=None)), ("fork", dict(ref=Stand((0,), I32))), ("fork", dict(kv_len=Stand((3,), I32))),
    ("copy", dict(src=Stand((0,), I32))), ("copy", dict(dst=Stand((2,), I32))), ("copy", dict(length=Stand((2,), I32))),
    ("compact", dict(keep=Stand((3, 3), I32))), ("compact", dict(keep=Stand((6,), I32))), ("compact", dict(n_keep=Stand((1,), I32))),
    ("compact", dict(cu_q=Stand((2,), I32))), ("compact", dict(state=Stand((1,), I32))), ("compact", dict(slot=Stand((0,), torch.int64)))])
def test_binding_refuses_shapes(binding, name, kw):
    with pytest.raises(binding.AtSpeedError):
        CALLS[name][0](binding, **kw)


def test_fork_refuses_outputs_of_other_sizes(binding):
    shapes = dict(table=(7, 6), kv_len=(7,), state=(7,), src=(7,), dst=(7,), ref=(9,), free=(9,), n_free=(1,))
    out = binding.PageFork(**{k: Stand(s, I32) for k, s in shapes.items()})
    with pytest.raises(Launched):
        _b_fork(binding, out=out)
    for k, s in shapes.items():
        setattr(out, k, Stand((s[0] - 1, *s[1:]), I32))
        with pytest.raises(binding.AtSpeedError):
            _b_fork(binding, out=out)
        setattr(out, k, Stand(s, I32))


def test_cache_layers_refuse(binding):
    good = (_cache(), _cache())
    for caches in ([], [good, (_cache(), _cache(device=OTHER))], [(_cache(device=torch.device("cpu")),) * 2],
                   [(_cache(), _cache(shape=(4, 16, 2, 32)))], [(_cache(shape=(4, 16, 128)),) * 2], [(_cache(dtype=I32),) * 2]):
        with pytest.raises(binding.AtSpeedError):
            binding.CacheLayers(caches)
    with pytest.raises(binding.AtSpeedError):   # not on the current device
        _b_copy(binding, binding.CacheLayers([(_cache(device=OTHER),) * 2]))
