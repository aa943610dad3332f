"""The tests' own statement of a map's tile lists, on the CPU: against the library's sizes and by hand."""

import ctypes

import numpy as np
import pytest

from paper_2508_02343_amd import binding as b
from tests import group_lists as G


@pytest.mark.parametrize("rows,experts", [(1, 1), (1, 8), (40, 4), (33, 1024), (4096, 7), (4097, 7), (65536, 128), (600_001, 17),
                                          (2**26, 1024)])
def test_layout_is_the_library_s(rows, experts):
    sz = b.MMGroupSizes()
    assert b.lib.mm_group_layout_sizes(rows, experts, ctypes.byref(sz)) == 0
    l = G.layout(rows, experts)
    assert (sz.capacity, sz.slots, sz.owners, sz.bytes) == (l["capacity"], l["slots"], l["owners"], 4 * l["words"])


def test_lists_by_hand():
    ids = np.array([2] * 300 + [0] * 33 + [-1] * 5 + [3] * 7, np.int32)
    small, middle, wide = G.lists(ids, 4)
    assert small[:3].tolist() == [[0, 0 | 32 << 16], [1, 0 | 1 << 16], [2, 2 | 32 << 16]] and len(small) == 2 + 10 + 1
    assert middle.tolist() == [[0, 0 | 33 << 16], [2, 2 | 128 << 16], [6, 2 | 128 << 16], [10, 2 | 44 << 16], [12, 3 | 7 << 16]]
    assert wide.tolist() == [[0, 0 | 33 << 16], [2, 2 | 256 << 16], [10, 2 | 44 << 16], [12, 3 | 7 << 16]]
