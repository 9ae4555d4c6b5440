"""Host-side checks of beam selection, page fork and moves at the edges of what they allow: no GPU."""
import pytest
import torch

from test_beam_ops_cpu import (E_ARG, E_SHAPE, P, _array, _b_compact, _b_copy, _b_fork, _b_select, _compact, _copy, _fork, _pages, _select,  # noqa: F401
                               binding, lib, stand_library)
from test_step_ops_devices_cpu import I32, Launched, Stand


@pytest.mark.parametrize("entries,room", [(5, 5), (1, 1), (0, -1)])
def test_fork_says_how_long_its_free_list_is(binding, monkeypatch, entries, room):  # noqa: F811
    """A count of free pages on the device may be past the list: the kernel is told where it ends."""
    seen = []

    class Lib:
        def atspeed_op_fork_pages(self, stream, fork):
            seen.append(binding.PageForkDesc.from_buffer_copy(fork))
            raise Launched

    monkeypatch.setattr(binding, "load", Lib)
    with pytest.raises(Launched):
        _b_fork(binding, free=Stand((entries,), I32))
    assert seen[0].free_size == room and seen[0].n_pages == 9 and seen[0].n_new == 7 and seen[0].d_table == 1 << 20


INS = dict(table=12, kv_len=4, q_len=4, old_state=4, parent=5, length=5, ref=9, free=6, n_free=1, used=1)      # entries
OUTS = dict(new_table=15, new_len=5, new_state=5, src=5, dst=5, new_ref=9, new_free=9, new_n_free=1)


@pytest.mark.parametrize("out", list(OUTS))
def test_fork_refuses_outputs_that_overlap(lib, out):  # noqa: F811
    """The first or the last entry of an input, or of another output, is one of an output's."""
    from paper_2410_05165_gb300.binding import PageForkDesc
    at = {k: P + 4096 * i for i, k in enumerate((*INS, *OUTS))}
    for other, n in (*INS.items(), *OUTS.items()):
        for place in (at[other], at[other] + 4 * (n - 1), at[other] - 4 * (OUTS[out] - 1)):
            if other != out:
                fork = PageForkDesc(n_old=4, n_new=5, table_width=3, page_size=16, n_pages=9, free_size=6,
                                    **{"d_" + k: p for k, p in {**at, out: place}.items()})
                assert lib.atspeed_op_fork_pages(None, bytes(fork)) == E_ARG, (other, place)


def test_lists_that_end_near_2_31(lib):  # noqa: F811
    """A kernel's indices go on behind a list's end by less than a CTA's step."""
    assert _copy(lib, _array(_pages()), n=2 ** 31 - 1) == E_SHAPE and _copy(lib, _array(_pages()), n=2 ** 31 - 1024) == E_SHAPE
    assert _compact(lib, _array(_pages()), width=2 ** 31 - 256) == E_SHAPE
    assert _fork(lib, width=2 ** 31 - 512) == E_SHAPE


def test_counts_past_2_31_are_not_cut(binding, monkeypatch):  # noqa: F811
    """2^32 + 3 of anything are not 3."""
    many = 2 ** 32 + 3
    for src in (many, 2 ** 31):
        with pytest.raises(binding.AtSpeedError):
            _b_copy(binding, src=Stand((src,), I32), dst=Stand((src,), I32), length=Stand((src,), I32))
    with pytest.raises(binding.AtSpeedError):
        _b_compact(binding, keep=Stand((2, many), I32))
    with pytest.raises(binding.AtSpeedError):
        _b_compact(binding, cu_q=Stand((many + 1,), I32), kv_len=Stand((many,), I32), keep=Stand((many, 3), I32), n_keep=Stand((many,), I32), state=None)
    seen = []

    class Lib:
        def atspeed_op_compact_tokens(self, *args):
            seen.append(args)
            raise Launched

    monkeypatch.setattr(binding, "load", Lib)
    with pytest.raises(Launched):   # (offsets among them have 32 bits)
        _b_compact(binding, slot=Stand((many,), torch.int64))
    assert seen[0][4] == 2 ** 31 - 1


@pytest.mark.parametrize("missing", ["_raw_alloc", "_raw_delete"])
def test_select_without_raw_allocations(binding, monkeypatch, missing):  # noqa: F811
    """A torch that lacks them: the workspace is a tensor."""
    monkeypatch.setattr(binding, missing, None)
    with pytest.raises(Launched):
        _b_select(binding)


def test_select_refuses_outputs_that_overlap(lib):  # noqa: F811
    """Places [2][10] of a request are written while another's rows are read."""
    ins = dict(logits=1200, cu=12, d_score=12, d_final=12, state=12, grammar=32)   # bytes: 3 rows of 100, two states
    outs = dict(token=80, parent=80, out=80)
    at = {k: P + 4096 * i for i, k in enumerate((*ins, *outs))}
    for out in outs:
        for other, size in (*ins.items(), *outs.items()):
            for place in (at[other], at[other] + size - 4, at[other] - 76):
                if other != out:
                    assert _select(lib, n_states=2, stride=4, ws=2 * P, **{**at, out: place}) == E_ARG, (out, other, place)


def test_compact_refuses_a_new_length_over_an_input(lib):  # noqa: F811
    ins = dict(slot=64, cu_q=12, kv=8, state=8, keep=24, n_keep=8)   # bytes: 2 requests, 8 tokens, 3 kept at most
    at = {k: P + 4096 * i for i, k in enumerate(ins)}
    for other, size in ins.items():
        for place in (at[other], at[other] + size - 4, at[other] - 4):
            if (other, place) != ("kv", at["kv"]):   # (that one is right)
                assert _compact(lib, _array(_pages(d_k=2 * P, d_v=3 * P)), **at, new_len=place) == E_ARG, (other, place)
