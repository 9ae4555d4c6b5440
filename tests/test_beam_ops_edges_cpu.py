"""Host-side checks of beam selection, page fork and moves at the edges of what they allow: no GPU."""
import pytest
import torch

from test_beam_ops_cpu import E_ARG, P, _b_fork, binding, lib, stand_library  # noqa: F401
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
