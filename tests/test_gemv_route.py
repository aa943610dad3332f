"""mm_gemv's choice of a kernel and its workspace, on the CPU (the pointers are fake: every call here is refused)."""

import ctypes

import pytest

from paper_2508_02343_amd import binding as b
from tests.gemv_routes import CASES, SPLITS, plan

FAKE = 0x10000  # 16-byte aligned, never dereferenced: validation fails first
SPLIT, K = (64, 32, 32), 128


def _size(rows, split):
    n = ctypes.c_int64(-1)
    assert b.lib.mm_gemv_workspace_size(rows, sum(split), b.MMSplit(*split), ctypes.byref(n)) == 0
    return n.value


def _gemv(rows, experts, ids, ws, nbytes, split=SPLIT):
    w = b.MMTensor()
    w.rows, w.K, w.split = 16, sum(split), b.MMSplit(*split)
    w.q4 = w.q6 = w.q8 = w.sc = FAKE
    return b.STATUS_NAMES[b.lib.mm_gemv(FAKE, sum(split), rows, 1, FAKE, 0, ctypes.byref(w), experts, ids, ws, nbytes, FAKE, 16,
                                        None)]


@pytest.mark.parametrize("rows,experts", [(16, 16), (16, 64), (7, 7), (16, 1024)])
def test_no_workspace_is_asked_for_where_none_is_used(rows, experts):
    """Rows that find their own experts go through LDS.  (A misaligned workspace is refused behind its size: the call
    got past the size, and nothing is launched.)"""
    assert _size(rows, SPLIT) > 0
    assert _gemv(rows, experts, FAKE, FAKE + 4, 0) == "MM_ERR_ALIGN"


@pytest.mark.parametrize("rows,experts", [(16, 15), (16, 1), (8, 4)])
def test_workspace_is_asked_for_where_it_is_used(rows, experts):
    need = _size(rows, SPLIT)
    assert _gemv(rows, experts, FAKE, FAKE, need - 1) == "MM_ERR_WORKSPACE"
    assert _gemv(rows, experts, FAKE, None, 0) == "MM_ERR_NULL"
    assert _gemv(rows, 1, None, FAKE, need - 1) == "MM_ERR_WORKSPACE"


@pytest.mark.parametrize("split", [(32, 0, 0), SPLIT, (2048, 1024, 1024), (20736, 5184, 1728), (24576, 6144, 2048)], ids=str)
def test_one_rule_for_launch_and_workspace(split):
    """The launch reads a workspace exactly where the call asks for one, and the size query is enough for it."""
    for rows in range(1, 17):
        for experts in (0, 1, 2, rows - 1, rows, rows + 1, 1024):
            *_, in_lds, need = plan(rows, 5000, split, max(experts, 0))
            assert (need == 0) == in_lds
            assert need in (0, _size(rows, split))
            assert in_lds or experts < rows  # (with an expert for every row never)


@pytest.mark.parametrize("form,rows,experts,N", CASES, ids=str)
def test_every_form_is_reached(form, rows, experts, N):
    for split in SPLITS:
        assert plan(rows, N, split, experts)[:3] == form
