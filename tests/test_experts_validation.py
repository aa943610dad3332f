"""CPU checks of the calls on rows grouped by expert and of mm_gemv: the map's
sizes, the plain reference itself, and every refusal, before anything reaches a
launch (the pointers are fake)."""

import ctypes

import numpy as np
import pytest
import torch

from paper_2508_02343_amd import binding as b
from tests import expert_cases as C

FAKE = 0x10000  # 16-byte aligned, never dereferenced: validation fails first
SPLIT, K = (64, 32, 32), 128


def _name(status):
    return b.STATUS_NAMES[status]


def _tensor(rows, split=SPLIT, ptr=FAKE):
    d = b.MMTensor()
    d.rows, d.K, d.split = rows, sum(split), b.MMSplit(*split)
    for name, p in zip(("q4", "q6", "q8"), split):
        setattr(d, name, ptr if p else None)
    d.sc = ptr
    return d


def _groups(rows=40, experts=4, ptr=FAKE):
    return b.MMRowGroups(rows, experts, ptr)


CAPACITY = 32 * ((40 + 31 * 4) // 32)


@pytest.mark.parametrize("rows,experts", [(1, 1), (1, 8), (40, 4), (33, 1024), (4096, 7), (4097, 7), (65536, 128), (2**26, 1024)])
def test_map_sizes(rows, experts):
    sz = b.MMGroupSizes()
    assert b.lib.mm_group_layout_sizes(rows, experts, ctypes.byref(sz)) == 0
    assert sz.capacity == 32 * ((rows + 31 * min(rows, experts)) // 32) and sz.capacity < 2**31
    assert sz.slots % 4 == 0 and sz.slots >= experts + 1
    assert sz.owners == sz.slots + sz.capacity
    assert sz.bytes >= 4 * (sz.owners + sz.capacity // 32)


@pytest.mark.parametrize("rows,experts", [(1, 1), (7, 3), (40, 4), (100, 100), (64, 2)])
def test_capacity_holds_the_worst_case(rows, experts):
    """Experts with one row more than whole row groups need the most packed rows."""
    most = 0
    for kind in ("even", "one", "holes"):
        m = C.group_map(C.make_ids(rows, experts, kind), experts)
        most = max(most, int(m["starts"][-1]))
    worst = np.concatenate([np.arange(min(rows, experts)), np.zeros(rows - min(rows, experts), int)]).astype(np.int32)
    m = C.group_map(worst, experts)
    assert max(most, int(m["starts"][-1])) <= b._group_sizes(rows, experts)[0]


@pytest.mark.parametrize("rows,experts,status", [(0, 4, "MM_ERR_SHAPE"), (-1, 4, "MM_ERR_SHAPE"), (2**26 + 1, 4, "MM_ERR_SHAPE"),
                                                 (40, 0, "MM_ERR_SHAPE"), (40, 1025, "MM_ERR_SHAPE")])
def test_group_shapes_refused(rows, experts, status):
    sz = b.MMGroupSizes()
    assert _name(b.lib.mm_group_layout_sizes(rows, experts, ctypes.byref(sz))) == status
    assert _name(b.lib.mm_group_rows(FAKE, ctypes.byref(_groups(rows, experts)), None)) == status
    assert b.lib.mm_last_error()


def test_group_rows_refused():
    f = b.lib.mm_group_rows
    assert _name(b.lib.mm_group_layout_sizes(1, 1, None)) == "MM_ERR_NULL"
    assert _name(f(None, ctypes.byref(_groups()), None)) == "MM_ERR_NULL"
    assert _name(f(FAKE, None, None)) == "MM_ERR_NULL"
    assert _name(f(FAKE, ctypes.byref(_groups(ptr=None)), None)) == "MM_ERR_NULL"
    assert _name(f(FAKE, ctypes.byref(_groups(ptr=FAKE + 4)), None)) == "MM_ERR_ALIGN"
    assert _name(f(FAKE + 2, ctypes.byref(_groups()), None)) == "MM_ERR_ALIGN"


def _quantize(x=FAKE, ldx=K, top_k=2, perm=FAKE, stride=0, groups=None, out=None):
    g = groups or _groups()
    o = out or _tensor(CAPACITY)
    return _name(b.lib.mm_quantize_act_grouped(x, ldx, top_k, perm, stride, ctypes.byref(g), ctypes.byref(o), None))


@pytest.mark.parametrize("kw,status", [
    ({"x": None}, "MM_ERR_NULL"), ({"perm": None}, "MM_ERR_NULL"), ({"groups": _groups(ptr=None)}, "MM_ERR_NULL"),
    ({"ldx": K - 8}, "MM_ERR_SHAPE"), ({"ldx": K + 4}, "MM_ERR_ALIGN"), ({"x": FAKE + 8}, "MM_ERR_ALIGN"),
    ({"perm": FAKE + 4}, "MM_ERR_ALIGN"), ({"stride": K - 4}, "MM_ERR_SHAPE"), ({"stride": -K}, "MM_ERR_SHAPE"),
    ({"stride": K + 2}, "MM_ERR_ALIGN"), ({"top_k": 0}, "MM_ERR_VALUE"), ({"top_k": -1}, "MM_ERR_VALUE"),
    ({"out": _tensor(CAPACITY + 32)}, "MM_ERR_SHAPE"), ({"out": _tensor(40)}, "MM_ERR_SHAPE"),
    ({"out": _tensor(CAPACITY, (32768, 32, 0)), "ldx": 32800}, "MM_ERR_SHAPE"),
    ({"out": _tensor(CAPACITY, (64, 16, 48))}, "MM_ERR_SPLIT"), ({"out": _tensor(CAPACITY, ptr=FAKE + 4)}, "MM_ERR_ALIGN")])
def test_quantize_grouped_refused(kw, status):
    assert _quantize(**kw) == status


def _gemm(a=None, w=None, groups=None, y=FAKE, ldy=16):
    a, w, g = a or _tensor(CAPACITY), w or _tensor(16), groups or _groups()
    return _name(b.lib.mm_gemm_grouped(ctypes.byref(a), ctypes.byref(w), ctypes.byref(g), y, ldy, None))


def _other_formats(rows):
    t = _tensor(rows)
    t.formats = b.MMFormats(1, 0)
    return t


@pytest.mark.parametrize("kw,status", [
    ({"a": _tensor(40)}, "MM_ERR_SHAPE"), ({"w": _tensor(16, (64, 64, 32))}, "MM_ERR_SHAPE"),
    ({"w": _tensor(16, (32, 64, 32))}, "MM_ERR_SHAPE"), ({"w": _other_formats(16)}, "MM_ERR_FORMAT"),
    ({"y": None}, "MM_ERR_NULL"), ({"y": FAKE + 8}, "MM_ERR_ALIGN"), ({"ldy": 8}, "MM_ERR_SHAPE"),
    ({"ldy": 20}, "MM_ERR_ALIGN"), ({"groups": _groups(ptr=None)}, "MM_ERR_NULL"),
    ({"groups": _groups(experts=2000)}, "MM_ERR_SHAPE"), ({"w": _tensor(16, ptr=FAKE + 8)}, "MM_ERR_ALIGN")])
def test_gemm_grouped_refused(kw, status):
    assert _gemm(**kw) == status


def _gemv(x=FAKE, ldx=K, rows=4, top_k=2, perm=FAKE, stride=0, w=None, experts=4, ids=FAKE, ws=FAKE, nbytes=1 << 20, y=FAKE,
          ldy=16):
    w = w or _tensor(16)
    return _name(b.lib.mm_gemv(x, ldx, rows, top_k, perm, stride, ctypes.byref(w), experts, ids, ws, nbytes, y, ldy, None))


@pytest.mark.parametrize("kw,status", [
    ({"x": None}, "MM_ERR_NULL"), ({"perm": None}, "MM_ERR_NULL"), ({"y": None}, "MM_ERR_NULL"),
    ({"rows": 0}, "MM_ERR_SHAPE"), ({"rows": 17}, "MM_ERR_SHAPE"), ({"experts": 0}, "MM_ERR_SHAPE"),
    ({"experts": 1025}, "MM_ERR_SHAPE"), ({"top_k": 0}, "MM_ERR_VALUE"), ({"top_k": 17}, "MM_ERR_VALUE"),
    ({"ldx": K - 1}, "MM_ERR_SHAPE"), ({"x": FAKE + 1}, "MM_ERR_ALIGN"), ({"ids": FAKE + 2}, "MM_ERR_ALIGN"),
    ({"stride": K - 4}, "MM_ERR_SHAPE"), ({"stride": K + 1}, "MM_ERR_ALIGN"), ({"perm": FAKE + 8}, "MM_ERR_ALIGN"),
    ({"ldy": 15}, "MM_ERR_SHAPE"), ({"ldy": 17}, "MM_ERR_ALIGN"), ({"y": FAKE + 2}, "MM_ERR_ALIGN"),
    ({"w": _tensor(16, (64, 32, 16))}, "MM_ERR_SHAPE"), ({"w": _tensor(16, (64, 48, 16))}, "MM_ERR_SPLIT"),
    ({"ws": FAKE + 4}, "MM_ERR_ALIGN"), ({"w": _tensor(16, (32768, 32, 0)), "ldx": 32800}, "MM_ERR_SHAPE"),
    ({"w": _tensor(2**28 + 1), "ldy": 2**28 + 8}, "MM_ERR_SHAPE")])
def test_gemv_refused(kw, status):
    assert _gemv(**kw) == status


def test_gemv_workspace():
    n = ctypes.c_int64()
    f = b.lib.mm_gemv_workspace_size
    assert _name(f(4, K, b.MMSplit(*SPLIT), None)) == "MM_ERR_NULL"
    assert _name(f(17, K, b.MMSplit(*SPLIT), ctypes.byref(n))) == "MM_ERR_SHAPE"
    assert _name(f(4, K, b.MMSplit(64, 32, 64), ctypes.byref(n))) == "MM_ERR_SPLIT"
    assert f(16, 14336, b.MMSplit(14336, 0, 0), ctypes.byref(n)) == 0
    need = n.value
    if need:
        big = _tensor(16, (14336, 0, 0))
        assert _gemv(rows=16, ldx=14336, w=big, nbytes=need - 1) == "MM_ERR_WORKSPACE"
        assert _gemv(rows=16, ldx=14336, w=big, ws=None) == "MM_ERR_NULL"


# ---- the binding ----


def test_stack_views():
    w = b.MXStack.empty(3, 70, 256, (128, 64, 64), device="cpu")
    sizes = b.layout_sizes(70, 256, (128, 64, 64))
    assert len(w) == 3
    for name in ("q4", "q6", "q8", "sc"):
        assert getattr(w, name).numel() == 3 * sizes[name]
        for e in (0, 1, 2, -1):
            t = getattr(w[e], name)
            assert t.numel() == sizes[name]
            assert t.data_ptr() == getattr(w, name).data_ptr() + (e % 3) * sizes[name]
    b._check_mx(w[1], 70, 256, (128, 64, 64), torch.device("cpu"), "w[1]")
    with pytest.raises(IndexError):
        w[3]
    with pytest.raises(ValueError):
        b.MXStack.empty(0, 70, 256, (128, 64, 64), device="cpu")
    assert b.MXStack.empty(2, 5, 64, (64, 0, 0), device="cpu")[1].q6 is None


def test_groups_views_and_refusals():
    g = b.RowGroups.empty(40, 4, device="cpu")
    assert g.capacity == CAPACITY and g.starts.numel() == 5 and g.slots.numel() == CAPACITY
    assert g.owners.numel() == CAPACITY // 32
    with pytest.raises(ValueError):
        b.RowGroups(40, 4, g.map[:-1])
    with pytest.raises(ValueError):
        b.RowGroups(40, 4, g.map.float())
    with pytest.raises(b.MMError, match="MM_ERR_SHAPE"):
        b.RowGroups.empty(0, 4, device="cpu")
    with pytest.raises(AttributeError):  # the views go with the map
        g.map = g.map.clone()


def test_host_tensors_refused():
    ids = torch.zeros(40, dtype=torch.int32)
    g = b.RowGroups.empty(40, 4, device="cpu")
    x = torch.zeros(20, K, dtype=torch.bfloat16)
    perm = torch.arange(K, dtype=torch.int32)
    a = b.MXTensor.empty(CAPACITY, K, SPLIT, device="cpu")
    w = b.MXStack.empty(4, 16, K, SPLIT, device="cpu")
    for call in (lambda: b.group_rows(ids, 4), lambda: b.group_rows(ids.long(), 4), lambda: b.group_rows(ids[::2], 4),
                 lambda: b.quantize_act_grouped(x, g, perm, SPLIT, top_k=2),
                 lambda: b.gemm_grouped(a, w, g), lambda: b.gemv(x[:2], w, perm, ids=ids[:4], top_k=2)):
        with pytest.raises(ValueError):
            call()


def test_sigma_and_result_checks():
    """What the calls check of sigma, the weights and the result, on host tensors."""
    perm = torch.arange(4 * K, dtype=torch.int32)
    assert b._check_perms(perm[:K], 4, K, -1) == 0 and b._check_perms(perm.view(4, K), 4, K, -1) == K
    for bad in (perm[:K - 1], perm.view(2, 2 * K), perm.view(4, K)[:3], perm.view(K, 4).T, perm[:K].long()):
        with pytest.raises(ValueError):
            b._check_perms(bad, 4, K, -1)
    w = b.MXStack.empty(4, 16, K, SPLIT, device="cpu")
    for t, count in ((w, 4), (w[0], 1)):
        assert b._packed_checked(t, -1, "w", count) == t._packed()
    for name in ("q4", "q6", "q8", "sc"):
        full = getattr(w, name)
        for bad in (full[:-1], torch.cat([full, full])[::2], None):
            setattr(w, name, bad)
            with pytest.raises(ValueError, match=rf"w\.{name}"):
                b._packed_checked(w, -1, "w", 4)
        setattr(w, name, full)
    with pytest.raises(ValueError, match=r"w\.q4 must be contiguous and on cuda:3"):
        b._packed_checked(w, 3, "w", 4)
    y = torch.zeros(40, 16, dtype=torch.bfloat16)
    assert b._result(y, 40, 16, -1, y.device) is y
    for bad in (y[:39], y.float(), y.T, y[:, :15]):
        with pytest.raises(ValueError):
            b._result(bad, 40, 16, -1, y.device)
    made = b._result(None, 3, 13, -1, torch.device("cpu"))
    assert made.shape == (3, 13) and made.stride(0) % 8 == 0 and not made.any()
