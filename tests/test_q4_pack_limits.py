"""Limits of packing that are those of a launch (CPU only): refused before any launch, not by it."""
import pytest

import paper_2606_01007_amd as tacg
from test_moe_host import L, _pack  # noqa: F401


@pytest.mark.parametrize("rows, cols, group", [(1 << 26, 2048, 32), (1 << 26, 2017, 32), (1 << 26, 65536, 256), ((1 << 32) // 2048, 65505, 128),
                                               (1 << 26, 1800, 256)])
def test_more_pieces_than_a_launch_holds(L, rows, cols, group):  # noqa: F811
    assert _pack(L, rows=rows, cols=cols, stride=0, group=group) == tacg.E_UNSUPPORTED
