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


@pytest.mark.parametrize("formats", [("E3M2", "E4M3"), ("E2M3", "E5M2"), ("E3M2", "E5M2"), ("E2M3", "E4M3")], ids="-".join)
@pytest.mark.parametrize("split", R.SPLITS, ids=str)
@pytest.mark.parametrize("form,rows,experts,N", R.CASES, ids=str)
def test_every_form(form, rows, experts, N, split, formats):
    """Every compiled kernel with every format set, three groups and each alone, widths that are no multiple of a strip;
    x with a stride, guard columns beside y."""
    assert R.plan(rows, N, split, experts, _cus())[:3] == form
    note(f"gemv {form} rows={rows} E={experts} N={N} {split} {formats}")
    b, K, E = _b(), sum(split), max(experts, 1)
    xb, perms = C.activations(rows, K, E, seed=rows + N)
    # columns of the result to compare: some of every strip's 16-row halves, and the last ones
    cols = np.unique(np.concatenate([np.arange(0, N, max(1, N // 60)), np.arange(N - min(N, 40), N)]))
    at = torch.from_numpy(cols).cuda()
    w = b.MXStack.empty(E, N, K, split, formats=formats)
    wb = np.zeros((E, len(cols), K), np.uint16)
    for e in range(E):
        g = torch.Generator("cuda").manual_seed(1000 * N + e)
        we = (torch.randn(N, K, generator=g, device="cuda") * 0.02).bfloat16()
        b.quantize_weight(we, to_dev_perm(perms[e]), split, out=w[e])
        wb[e] = we[at].cpu().view(torch.int16).numpy().view(np.uint16)
    ids = C.make_ids(rows, experts, "even", seed=N) if experts else None
    if experts:
        ids[1] = -1
    wide_x = torch.full((rows, K + 8), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide_x[:, :K] = to_dev_bf16(xb)
    wide = torch.full((rows, (N + 7) // 8 * 8 + 8), 7.0, dtype=torch.bfloat16, device="cuda")
    b.gemv(wide_x[:, :K], w if experts else w[0], to_dev_perm(perms if experts else perms[0]),
           ids=None if ids is None else torch.from_numpy(ids).cuda(), y=wide[:, :N])
    torch.cuda.synchronize()
    ref, tol = C.gemv_product(xb, ids, 1, perms, wb, split, formats)
    _check(wide[:, at], ref, tol, 7.0, (form, split, formats))
    assert bool((wide[:, N:] == 7.0).all()), "columns behind the result"


@pytest.mark.parametrize("experts", [257, 1024])
def test_many_experts(experts):
    """Rows of the first and the last of many experts, and of those around 256."""
    note(f"gemv {experts} experts")
    b, N, split = _b(), 40, (96, 64, 64)
    K = sum(split)
    ids = np.array([0, experts - 1, 255, 256, 1, experts, -1, experts - 1, experts - 2, 128], np.int32)
    xb, perms = C.activations(len(ids), K, experts, seed=experts)
    wb = C.weights(experts, N, K, seed=experts)
    w = _stack(wb, perms, split)
    y = torch.full((len(ids), N), 7.0, dtype=torch.bfloat16, device="cuda")
    b.gemv(to_dev_bf16(xb), w, to_dev_perm(perms), ids=torch.from_numpy(ids).cuda(), y=y)
    torch.cuda.synchronize()
    ref, tol = C.gemv_product(xb, ids, 1, perms, wb, split, DEFAULT)
    _check(y, ref, tol, 7.0, experts)


@pytest.mark.parametrize("experts", [0, 8])
def test_no_rows_are_refused_as_a_shape(experts):
    b, split = _b(), (64, 32, 32)
    w = b.MXStack.empty(max(experts, 1), 40, 128, split)
    x = torch.zeros(4, 128, dtype=torch.bfloat16, device="cuda")
    p = torch.arange(128, dtype=torch.int32, device="cuda")
    ids = torch.zeros(0, dtype=torch.int32, device="cuda") if experts else None
    with pytest.raises(b.MMError, match="MM_ERR_SHAPE"):
        b.gemv(x[:0], w if experts else w[0], p, ids=ids)
    assert b.gemv(x[:1], w[0], p).shape == (1, 40)
