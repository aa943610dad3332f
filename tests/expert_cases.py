"""Inputs and plain references (numpy, 64 bits) for the calls on rows grouped by
expert and for mm_gemv."""

from __future__ import annotations

import numpy as np

from oracle import mx_oracle as O
from paper_2508_02343_amd import workloads as W

INT_MIN, INT_MAX = -2**31, 2**31 - 1


def make_ids(slots: int, experts: int, kind: str, seed: int = 0) -> np.ndarray:
    """int32 [slots]: experts of the slots, distributed as `kind` says."""
    rng = np.random.default_rng([seed, slots, experts])
    if kind == "even":
        ids = rng.integers(0, experts, slots)
    elif kind == "one":  # a single expert has every row
        ids = np.full(slots, experts - 1 - seed % experts)
    elif kind == "none":
        ids = np.full(slots, -1)
    elif kind == "skewed":  # expert e with weight 1 / (1 + e)^2, and some slots padded at the end
        p = 1.0 / (1.0 + np.arange(experts)) ** 2
        ids = rng.choice(experts, slots, p=p / p.sum())
        ids[slots - slots // 5:] = -1
    elif kind == "holes":  # every other expert without rows, some ids far outside
        ids = rng.integers(0, (experts + 1) // 2, slots) * 2
        out = rng.random(slots) < 0.2
        ids = np.where(out, rng.choice([INT_MIN, -1, experts, experts + 7, INT_MAX], slots), ids)
    else:
        raise ValueError(kind)
    return ids.astype(np.int32)


def group_map(ids: np.ndarray, experts: int) -> dict:
    """The row-group map by its definition, one slot at a time."""
    rows = len(ids)
    capacity = 32 * ((rows + 31 * min(experts, rows)) // 32)
    of = [[] for _ in range(experts)]
    for s, e in enumerate(ids.tolist()):
        if 0 <= e < experts:
            of[e].append(s)
    starts = np.zeros(experts + 1, np.int32)
    slots = np.full(capacity, -1, np.int32)
    owners = np.full(capacity // 32, -1, np.int32)
    for e in range(experts):
        n = len(of[e])
        groups = -(-n // 32)
        slots[starts[e]:starts[e] + n] = of[e]
        owners[starts[e] // 32:starts[e] // 32 + groups] = e
        starts[e + 1] = starts[e] + 32 * groups
    return {"capacity": capacity, "starts": starts, "slots": slots, "owners": owners}


def activations(rows: int, K: int, experts: int, seed: int):
    """bf16 bits [rows, K] with outlier channels, and a sigma per expert int32 [experts, K]."""
    rng = np.random.default_rng([seed, rows, K])
    x = rng.standard_normal((rows, K)).astype(np.float32)
    x[:, rng.choice(K, max(1, K // 64), replace=False)] *= 25
    return W.f32_to_bf16_bits(x), np.stack([rng.permutation(K) for _ in range(experts)]).astype(np.int32)


def weights(experts: int, N: int, K: int, seed: int) -> np.ndarray:
    rng = np.random.default_rng([seed, N, K, 5])
    return W.f32_to_bf16_bits((rng.standard_normal((experts, N, K)) * 0.02).astype(np.float32))


def formats_of(formats) -> tuple:
    return O.E2M1, O.FORMATS[formats[0]], O.FORMATS[formats[1]]


def grouped_product(xb, ids, top_k, perms, wb, split, formats) -> np.ndarray:
    """float64 [slots, N]: each slot's quantised row times its expert's quantised weight; NaN where the id names none."""
    fm = formats_of(formats)
    experts, N, _ = wb.shape
    y = np.full((len(ids), N), np.nan)
    for e in range(experts):
        rows = np.flatnonzero(ids == e)
        if rows.size:
            perm = perms[e if len(perms) > 1 else 0]
            y[rows] = O.gemm_mixed(O.quantize_mixed(xb[rows // top_k], perm, split, fm),
                                   O.quantize_mixed(wb[e], perm, split, fm))
    return y


def gemv_product(xb, ids, top_k, perms, wb, split, formats):
    """float64 [rows, N] of bf16 rows times quantised weights, and how far a bf16 result may be from it: half a bf16
    step (2^-8 of the value), and 2^-23 (a truncating 2^-24 rounding counted twice) of the sum of |terms| for each of the
    at most K / 32 + 40 additions that a term goes through (32 to a matrix instruction, at most 32 inside one, 8
    partial sums); the products of two bf16 values are exact in 32 bits."""
    fm = formats_of(formats)
    experts, N, K = wb.shape
    rows = len(xb) * top_k
    ids = np.zeros(rows, np.int32) if ids is None else ids
    y, tol = np.full((rows, N), np.nan), np.zeros((rows, N))
    for e in range(experts):
        r = np.flatnonzero(ids == e)
        if r.size:
            perm = perms[e if len(perms) > 1 else 0]
            x = O.bf16_bits_to_f64(xb[r // top_k])[:, perm]
            w = O.dequantize_mixed(O.quantize_mixed(wb[e], perm, split, fm))
            y[r] = x @ w.T
            # the sum's error moves the value that is rounded as well (1 + 2^-8)
            tol[r] = np.abs(y[r]) * 2.0**-8 + (1 + 2.0**-8) * (K / 32 + 40) * 2.0**-23 * (np.abs(x) @ np.abs(w).T)
    return y, tol
