"""GPU checks of mm_gemv by the form that a call takes (tests/gemv_routes.py), against the plain 64-bit
product and the bound counted from the kernel's roundings (expert_cases.gemv_product)."""

import ctypes
import functools

import numpy as np
import pytest
import torch

from tests import expert_cases as C
from tests import gemv_routes as R
from tests.gpu_helpers import note, to_dev_bf16, to_dev_perm, y_to_f64

pytestmark = pytest.mark.gpu

DEFAULT = ("E3M2", "E4M3")


@functools.lru_cache(maxsize=None)
def _b():
    from paper_2508_02343_amd import binding

    return binding


def _cus():
    return torch.cuda.get_device_properties(0).multi_processor_count


def _stack(wb, perms, split, formats=DEFAULT):
    b = _b()
    w = b.MXStack.empty(*wb.shape, split, formats=formats)
    for e in range(len(wb)):
        b.quantize_weight(to_dev_bf16(wb[e]), to_dev_perm(perms[e if len(perms) > 1 else 0]), split, out=w[e])
    return w


def _check(y, ref, tol, before, ctx):
    got = y_to_f64(y)
    live = ~np.isnan(ref).any(axis=1)
    err = np.abs(got[live] - ref[live])
    assert np.all(err <= tol[live]), (ctx, float((err - tol[live]).max()), np.argwhere(err > tol[live])[:3])
    assert np.all(got[~live] == before), (ctx, "rows without an expert")


@pytest.mark.parametrize("rows,top_k,experts", [(16, 8, 64), (12, 2, 12), (7, 1, 9)])
def test_rows_with_experts_of_their_own_take_no_workspace(rows, top_k, experts):
    """At least as many experts as rows: the C call goes without a workspace, and the binding's allocates nothing."""
    b, split, N = _b(), (1024, 256, 128), 72
    K = sum(split)
    assert b.gemv_workspace_size(rows, K, split) > 0
    assert R.plan(rows, N, split, experts, _cus())[2:] == (True, 0)
    note(f"gemv without a workspace, {rows} rows of {experts} experts")
    ids = C.make_ids(rows, experts, "holes", seed=3)
    xb, perms = C.activations(rows // top_k, K, 1, seed=rows)
    wb = C.weights(experts, N, K, seed=rows)
    w, x, p = _stack(wb, perms, split), to_dev_bf16(xb), to_dev_perm(perms[0])
    d = torch.from_numpy(ids).cuda()
    ref, tol = C.gemv_product(xb, ids, top_k, perms, wb, split, DEFAULT)
    y = torch.full((rows, N), 7.0, dtype=torch.bfloat16, device="cuda")
    desc = w[0].descriptor()
    status = b.lib.mm_gemv(x.data_ptr(), x.stride(0), rows, top_k, p.data_ptr(), 0, ctypes.byref(desc), experts, d.data_ptr(),
                           None, 0, y.data_ptr(), y.stride(0), torch.cuda.current_stream().cuda_stream)
    assert status == 0, b.lib.mm_last_error()
    torch.cuda.synchronize()
    _check(y, ref, tol, 7.0, "C call")
    y.fill_(7.0)
    before = torch.cuda.memory_stats()["allocation.all.allocated"]
    b.gemv(x, w, p, ids=d, top_k=top_k, y=y)
    assert torch.cuda.memory_stats()["allocation.all.allocated"] == before
    torch.cuda.synchronize()
    _check(y, ref, tol, 7.0, "binding")
