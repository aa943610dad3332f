"""GPU checks of what the grouped calls take from a row-group map: its tile lists, and maps whose
single parts were changed behind mm_group_rows (results are unspecified then, but everything stays in
bounds: no row outside the result, no row of a slot that no longer has a place is written)."""

import functools

import numpy as np
import pytest
import torch

from tests import expert_cases as C
from tests import group_lists as G
from tests import grouped_routes as R
from tests.gpu_helpers import note, to_dev_bf16, to_dev_perm

pytestmark = pytest.mark.gpu

INT_MIN, INT_MAX = -2**31, 2**31 - 1


@functools.lru_cache(maxsize=None)
def _b():
    from paper_2508_02343_amd import binding

    return binding


@pytest.mark.parametrize("kind", ("even", "one", "none", "skewed", "holes"))
@pytest.mark.parametrize("slots,experts", [(1, 1), (16, 8), (300, 1024), (1000, 1), (1025, 33), (4096, 8), (4097, 64), (9999, 1024),
                                           (65536, 128), (200_001, 700)])
def test_tile_lists(slots, experts, kind):
    note(f"tile lists {slots} slots, {experts} experts, {kind}")
    ids = C.make_ids(slots, experts, kind, seed=2)
    b = _b()
    out = b.RowGroups.empty(slots, experts)
    out.map.fill_(0x7A7A7A7A)
    b.group_rows(torch.from_numpy(ids).cuda(), experts, out=out)
    torch.cuda.synchronize()
    words, l = out.map.cpu().numpy(), G.layout(slots, experts)
    want = G.lists(ids, experts)
    assert words[l["tile_counts"]:l["tile_counts"] + 3].tolist() == [len(t) for t in want]
    for k, tiles in enumerate(want):
        got = words[l["tiles"][k]:l["tiles"][k] + 2 * l["ntiles"][k]].reshape(-1, 2)
        assert np.array_equal(got[:len(tiles)], tiles), (k, np.argwhere(got[:len(tiles)] != tiles)[:3])
        assert (got[len(tiles):] == (-1, 0)).all(), k


class _Product:
    """One product with guard rows and columns around its result."""

    def __init__(self, kernel, slots, experts, N, split):
        cus = torch.cuda.get_device_properties(0).multi_processor_count
        assert R.route(slots, experts, N, split, cus)[0] == kernel
        b, K = _b(), sum(split)
        self.slots, self.experts, self.N, self.split = slots, experts, N, split
        self.ids = C.make_ids(slots, experts, "skewed", seed=8)
        xb, perms = C.activations(slots, K, experts, seed=3)
        wb = C.weights(experts, N, K, seed=4)
        self.w = b.MXStack.empty(experts, N, K, split)
        for e in range(experts):
            b.quantize_weight(to_dev_bf16(wb[e]), to_dev_perm(perms[e]), split, out=self.w[e])
        self.perm, self.x = to_dev_perm(perms), to_dev_bf16(xb)
        self.groups = b.group_rows(torch.from_numpy(self.ids).cuda(), experts)
        self.at = G.layout(slots, experts)

    def run(self, change):
        """The result after change(words of the map, on the host), the guards checked."""
        b = _b()
        words = self.groups.map.cpu().numpy().copy()
        change(words)
        groups = b.RowGroups(self.slots, self.experts, torch.from_numpy(words).cuda())
        a = b.MXTensor.empty(groups.capacity, sum(self.split), self.split)
        for n in ("q4", "q6", "q8", "sc"):
            if getattr(a, n) is not None:
                getattr(a, n).zero_()
        b.quantize_act_grouped(self.x, groups, self.perm, self.split, out=a)
        columns = (self.N + 7) // 8 * 8
        wide = torch.full((self.slots + 2, columns + 16), 7.0, dtype=torch.bfloat16, device="cuda")
        y = wide[1:-1, 8:8 + self.N]
        b.gemm_grouped(a, self.w, groups, y=y)
        torch.cuda.synchronize()
        assert bool((wide[0] == 7).all() and (wide[-1] == 7).all() and (wide[:, :8] == 7).all()
                    and (wide[:, 8 + self.N:] == 7).all()), "outside of the result"
        assert np.array_equal(groups.map.cpu().numpy(), words), "the map"
        return y.float().cpu().numpy()


CASES = pytest.mark.parametrize("kernel,slots,experts,N,split", R.CASES, ids=str)


@CASES
def test_any_tile_count(kernel, slots, experts, N, split):
    """Counts below the number of tiles leave rows out, larger ones change nothing."""
    note(f"tile counts {kernel}")
    p = _Product(kernel, slots, experts, N, split)
    want = p.run(lambda words: None)
    live = (p.ids >= 0) & (p.ids < experts)
    assert (want[~live] == 7).all() and not (want[live] == 7).all(1).any()
    for count in (0, -1, -257, -(1 << 30), INT_MIN, -0x5A5A5A5B, 0x7A7A7A7A, INT_MAX):
        def change(words):
            words[p.at["tile_counts"]:p.at["tile_counts"] + 3] = count

        note(f"tile counts {kernel} {count}")
        got = p.run(change)
        if count <= 0 and not kernel.startswith("split"):  # (the K-splitting kernel takes the whole list)
            assert (got == 7).all(), count
        else:
            assert np.array_equal(got, want), count


@CASES
def test_slots_outside_the_result(kernel, slots, experts, N, split):
    """Rows whose slot is no row of the result go nowhere, the others where they belong."""
    note(f"slots {kernel}")
    p = _Product(kernel, slots, experts, N, split)
    want = p.run(lambda words: None)
    gone = np.zeros(slots, bool)

    def change(words):
        rows = words[p.at["slots"]:p.at["slots"] + p.at["capacity"]]
        filled = np.flatnonzero(rows >= 0)
        for k, other in enumerate((slots, slots + 1, INT_MAX, INT_MIN, -7)):
            take = filled[k::11]
            gone[rows[take]] = True
            rows[take] = other

    got = p.run(change)
    assert gone.any() and (got[gone] == 7).all() and np.array_equal(got[~gone], want[~gone])


@CASES
def test_tiles_that_are_none(kernel, slots, experts, N, split):
    """Listed tiles with an expert, a row group or a number of rows that cannot be are passed over; one with
    another expert is that expert's (any result, in bounds)."""
    p = _Product(kernel, slots, experts, N, split)
    live = (p.ids >= 0) & (p.ids < experts)
    groups = p.at["capacity"] // 32
    for what, first, owner_rows in (("expert", None, lambda e, n: experts | n << 16), ("expert", None, lambda e, n: 0xFFFF | n << 16),
                                    ("rows", None, lambda e, n: e | 257 << 16), ("rows", None, lambda e, n: e | 0xFFFF << 16),
                                    ("rows", None, lambda e, n: e), ("group", groups, None), ("group", INT_MAX, None),
                                    ("group", -2, None), ("group", INT_MIN, None), ("other", None, lambda e, n: (e + 1) % experts | n << 16)):
        def change(words):
            for at, n in zip(p.at["tiles"], p.at["ntiles"]):
                for t in range(n):
                    if words[at + 2 * t] < 0:
                        break
                    if first is not None:
                        words[at + 2 * t] = first
                    else:
                        v = int(words.view(np.uint32)[at + 2 * t + 1])
                        words.view(np.uint32)[at + 2 * t + 1] = owner_rows(v & 0xFFFF, v >> 16)

        note(f"tiles {kernel} {what}")
        got = p.run(change)
        assert (got[~live] == 7).all(), what
        if what != "other":
            assert (got == 7).all(), what
