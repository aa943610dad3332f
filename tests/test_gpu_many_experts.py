"""GPU parity of the grouped quantiser and product with hundreds of experts (1024 are the most), against the plain
64-bit references."""

import numpy as np
import pytest
import torch

from oracle import mx_oracle as O
from tests import expert_cases as C
from tests import grouped_routes as R
from tests import packed_layout as L
from tests.gpu_helpers import assert_gemm_close, note, to_dev_bf16, to_dev_perm, y_to_f64

pytestmark = pytest.mark.gpu

DEFAULT = ("E3M2", "E4M3")


@pytest.mark.parametrize("kernel,slots,experts,N,split", [
    ("split32x32", 700, 300, 96, (96, 64, 64)), ("split32x32", 2100, 1024, 70, (96, 64, 64)),
    ("tiled128x128", 9000, 300, 150, (224, 64, 96)), ("tiled128x128", 20000, 1024, 264, (96, 64, 64))], ids=str)
def test_many_experts(kernel, slots, experts, N, split):
    from paper_2508_02343_amd import binding as b

    assert R.route(slots, experts, N, split, torch.cuda.get_device_properties(0).multi_processor_count)[0] == kernel
    note(f"{kernel} {slots} slots, {experts} experts")
    K = sum(split)
    ids = C.make_ids(slots, experts, "even", seed=experts)
    ids[::7] = experts - 1  # a long run for the last one
    ids[1:40:3], ids[2:40:3], ids[5] = 255, 256, -1
    xb, perms = C.activations(slots, K, experts, seed=1)
    wb = C.weights(experts, N, K, seed=2)
    w = b.MXStack.empty(experts, N, K, split)
    p = to_dev_perm(perms)
    for e in range(experts):
        b.quantize_weight(to_dev_bf16(wb[e]), p[e], split, out=w[e])
    g = b.group_rows(torch.from_numpy(ids).cuda(), experts)
    a = b.quantize_act_grouped(to_dev_bf16(xb), g, p, split)
    y = torch.full((slots, N + (-N) % 8), 7.0, dtype=torch.bfloat16, device="cuda")[:, :N]
    b.gemm_grouped(a, w, g, y=y)
    torch.cuda.synchronize()
    want = C.group_map(ids, experts)
    codes = L.untile(a.raw_host(), a.rows, split)
    for e in (0, 1, 255, 256, experts - 2, experts - 1):
        rows = np.flatnonzero((np.repeat(want["owners"], 32) == e) & (want["slots"] >= 0))
        ref = O.quantize_mixed(xb[want["slots"][rows]], perms[e], split, C.formats_of(DEFAULT))
        for n in ("q4", "q6", "q8", "sc"):
            assert np.array_equal(codes[n][rows], getattr(ref, n)), (e, n)
    ref = C.grouped_product(xb, ids, 1, perms, wb, split, DEFAULT)
    live = ~np.isnan(ref).any(axis=1)
    assert not live[5]
    got = y_to_f64(y)
    assert_gemm_close(got[live], ref[live], ctx=f"{kernel} {experts}")
    assert (got[~live] == 7).all()
