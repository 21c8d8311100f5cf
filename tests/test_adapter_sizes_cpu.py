"""Widths next to 2^31, which the adapters' kernels cannot step over, are refused on the
host before any launch; no GPU is needed."""
import pytest

from paper_2606_09508_amd import binding as eb
from test_adapter_abi_cpu import BAD, BATCH, FAKE, L, add  # noqa: F401

LAST = 2 ** 31 - 8       # the last multiple of 8


@pytest.mark.parametrize("width", [LAST, LAST - 4088])
def test_widths_next_to_the_end_of_32_bits(L, width):  # noqa: F811
    # (no workspace: the widths are looked at before it)
    assert add(L, n_in=width, ws=None, ws_nb=0) == BAD
    assert add(L, outs=(64, width), ws=None, ws_nb=0) == BAD
    assert L.ei_adapter_add_workspace_bytes(BATCH, width, 16, 2) == 0


def test_the_widest_rows(L):  # noqa: F811
    width = LAST - 4096
    assert L.ei_adapter_add_workspace_bytes(BATCH, width, 16, 2) > 0
    assert add(L, n_in=width, outs=(width,), ws=None, ws_nb=0) == -4      # the workspace
    assert eb.AdapterTarget(FAKE, FAKE, None, FAKE, width).n_out == width
