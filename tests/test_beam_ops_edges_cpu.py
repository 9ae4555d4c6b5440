"""Host-side checks of beam selection, page fork and moves at the edges of what they allow: no GPU."""
import pytest
import torch

from test_beam_ops_cpu import (E_ARG, E_SHAPE, P, _array, _b_fork, _b_select, _cache, _copy, _fork, _pages, binding, lib,  # noqa: F401
                               stand_library)
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
