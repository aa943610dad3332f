"""GPU parity of the calls on rows grouped by expert (mm_group_rows,
mm_quantize_act_grouped, mm_gemm_grouped) and of mm_gemv against plain 64-bit
references: the map and the codes exactly, products within the GEMM's tolerance
(|gpu - ref| <= 2^-8 |ref| + 1e-3 rms(ref)) or, for mm_gemv, within a bound counted
from its roundings."""

import functools

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
KINDS = ("even", "one", "none", "skewed", "holes")


@functools.lru_cache(maxsize=None)
def _b():
    from paper_2508_02343_amd import binding

    return binding


def _dev_ids(ids):
    return torch.from_numpy(ids).cuda()


def _stack(wb, perms, split, formats=DEFAULT):
    b = _b()
    E, N, K = wb.shape
    w = b.MXStack.empty(E, N, K, split, formats=formats)
    for e in range(E):
        b.quantize_weight(to_dev_bf16(wb[e]), to_dev_perm(perms[e if len(perms) > 1 else 0]), split, out=w[e])
    return w


def _perm_arg(perms):
    return to_dev_perm(perms if len(perms) > 1 else perms[0])


def _garbage(t):
    """Fill an MXTensor's buffers with 0xFF: NaN codes and NaN scales."""
    for n in ("q4", "q6", "q8", "sc"):
        if getattr(t, n) is not None:
            getattr(t, n).fill_(255)
    return t


# ---- the map ----


def _check_map(g, ids, experts, ctx):
    want = C.group_map(ids, experts)
    assert g.capacity == want["capacity"], ctx
    for name in ("starts", "slots", "owners"):
        got = getattr(g, name).cpu().numpy()
        assert np.array_equal(got, want[name]), (ctx, name, np.flatnonzero(got != want[name])[:5])


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("slots,experts", [(1, 1), (1, 8), (16, 8), (37, 5), (64, 64), (300, 1024), (1000, 1), (1025, 33),
                                           (4096, 8), (4097, 64), (9999, 1024), (65536, 128)])
def test_group_rows(slots, experts, kind):
    note(f"group {slots} slots, {experts} experts, {kind}")
    ids = C.make_ids(slots, experts, kind)
    b = _b()
    out = b.RowGroups.empty(slots, experts)
    out.map.fill_(0x7A7A7A7A)  # whatever was there before does not matter
    b.group_rows(_dev_ids(ids), experts, out=out)
    torch.cuda.synchronize()
    _check_map(out, ids, experts, (slots, experts, kind))


def test_group_rows_many_slots():
    """More slots than the workgroups' single turns take (128 workgroups of 4096)."""
    slots, experts = 600_001, 17
    note(f"group {slots} slots, {experts} experts")
    ids = C.make_ids(slots, experts, "skewed")
    g = _b().group_rows(_dev_ids(ids), experts)
    torch.cuda.synchronize()
    _check_map(g, ids, experts, "many")


def test_group_rows_2d_ids_and_unaligned():
    """ids in the router's [tokens, top_k] shape, at an address that is no multiple of 16."""
    note("group 2-D ids at an odd address")
    ids = C.make_ids(42, 6, "even")
    buf = torch.zeros(43, dtype=torch.int32, device="cuda")
    buf[1:] = _dev_ids(ids)
    g = _b().group_rows(buf[1:].view(21, 2), 6)
    torch.cuda.synchronize()
    _check_map(g, ids, 6, "2-D")


# ---- the quantiser ----


def _check_quantised(a, xb, ids, top_k, experts, perms, split, formats, before, ctx):
    """Rows with a slot hold the oracle's codes; the others' bytes are what they were."""
    want_map = C.group_map(ids, experts)
    got = L.untile(a.raw_host(), a.rows, split)
    fm = C.formats_of(formats)
    for e in range(experts):
        p = np.flatnonzero((np.repeat(want_map["owners"], 32) == e) & (want_map["slots"] >= 0))
        if p.size == 0:
            continue
        ref = O.quantize_mixed(xb[want_map["slots"][p] // top_k], perms[e if len(perms) > 1 else 0], split, fm)
        for n in ("q4", "q6", "q8", "sc"):
            assert np.array_equal(got[n][p], getattr(ref, n)), (ctx, e, n)
    empty = np.flatnonzero(want_map["slots"] < 0)
    for n in ("q4", "q6", "q8", "sc"):
        assert np.all(got[n][empty] == before), (ctx, n, "rows without a slot")


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("tokens,top_k,experts,split,own_sigma", [
    (1, 1, 1, (32, 0, 0), False), (1, 2, 8, (96, 160, 96), False), (5, 3, 4, (0, 352, 0), True),
    (40, 2, 8, (0, 0, 352), True), (77, 4, 6, (2048, 1024, 1024), False), (300, 2, 5, (128, 0, 224), True)])
def test_quantize_grouped(tokens, top_k, experts, split, own_sigma, kind):
    note(f"quantise grouped T={tokens} k={top_k} E={experts} {split} {kind}")
    K, b = sum(split), _b()
    ids = C.make_ids(tokens * top_k, experts, kind, seed=3)
    xb, perms = C.activations(tokens, K, experts if own_sigma else 1, seed=tokens)
    g = b.group_rows(_dev_ids(ids), experts)
    out = b.MXTensor.empty(g.capacity, K, split)
    for n in ("q4", "q6", "q8", "sc"):
        if getattr(out, n) is not None:
            getattr(out, n).fill_(0xA5)
    b.quantize_act_grouped(to_dev_bf16(xb), g, _perm_arg(perms), split, top_k=top_k, out=out)
    torch.cuda.synchronize()
    _check_quantised(out, xb, ids, top_k, experts, perms, split, DEFAULT, 0xA5, (tokens, top_k, experts, split, kind))


@pytest.mark.parametrize("formats", [("E2M3", "E5M2"), ("E2M3", "E4M3")], ids="-".join)
@pytest.mark.parametrize("split", [(10752, 2688, 896), (24576, 6144, 2048), (4096, 1536, 1024)], ids=str)
def test_quantize_grouped_widths(split, formats):
    """Every number of rows per pass, the widest K, a row stride beyond K, many rows."""
    K, b = sum(split), _b()
    tokens, top_k, experts = (200, 3, 4) if K < 8192 else (30, 2, 3)
    note(f"quantise grouped K={K} {formats}")
    ids = C.make_ids(tokens * top_k, experts, "skewed", seed=1)
    xb, perms = C.activations(tokens, K, experts, seed=9)
    wide = torch.full((tokens, K + 64), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[:, :K] = to_dev_bf16(xb)
    g = b.group_rows(_dev_ids(ids), experts)
    out = _garbage(b.MXTensor.empty(g.capacity, K, split, formats=formats))
    b.quantize_act_grouped(wide[:, :K], g, _perm_arg(perms), split, top_k=top_k, out=out)
    torch.cuda.synchronize()
    _check_quantised(out, xb, ids, top_k, experts, perms, split, formats, 0xFF, (K, formats))


# ---- the grouped product ----


def _grouped(tokens, top_k, experts, N, split, kind, formats=DEFAULT, own_sigma=False, seed=0, cols=None):
    """The product's inputs on the GPU, and its reference (of the columns `cols` alone where given).  kind: make_ids'
    or the ids themselves."""
    b, K = _b(), sum(split)
    ids = C.make_ids(tokens * top_k, experts, kind, seed) if isinstance(kind, str) else kind
    xb, perms = C.activations(tokens, K, experts if own_sigma else 1, seed)
    wb = C.weights(experts, N, K, seed)
    w = _stack(wb, perms, split, formats)
    g = b.group_rows(_dev_ids(ids), experts)
    a = _garbage(b.MXTensor.empty(g.capacity, K, split, formats=formats))
    b.quantize_act_grouped(to_dev_bf16(xb), g, _perm_arg(perms), split, top_k=top_k, out=a)
    return ids, g, a, w, C.grouped_product(xb, ids, top_k, perms, wb if cols is None else wb[:, cols], split, formats)


def _check_rows(y, ref, before, ctx):
    """Rows with an expert within tolerance, the others as they were."""
    got = y_to_f64(y)
    live = ~np.isnan(ref).any(axis=1)
    if live.any():
        assert_gemm_close(got[live], ref[live], ctx=str(ctx))
    assert np.all(got[~live] == before), (ctx, "rows in no group")


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("tokens,top_k,experts,N,split", [
    (1, 1, 1, 1, (32, 0, 0)), (1, 2, 8, 33, (96, 160, 96)), (7, 2, 3, 70, (0, 352, 0)), (33, 1, 2, 130, (0, 0, 352)),
    (100, 3, 5, 264, (128, 0, 224)), (500, 2, 4, 300, (320, 96, 64)), (1500, 2, 3, 520, (160, 32, 64))])
def test_gemm_grouped(tokens, top_k, experts, N, split, kind):
    """From one row to more than the widest tile's, odd widths; packed rows without a slot hold NaN codes and scales."""
    note(f"gemm grouped T={tokens} k={top_k} E={experts} N={N} {split} {kind}")
    ids, g, a, w, ref = _grouped(tokens, top_k, experts, N, split, kind, own_sigma=tokens % 2 == 1)
    wide = torch.full((tokens * top_k, (N + 7) // 8 * 8 + 8), 7.0, dtype=torch.bfloat16, device="cuda")
    y = _b().gemm_grouped(a, w, g, y=wide[:, :N])
    torch.cuda.synchronize()
    _check_rows(y, ref, 7.0, (tokens, top_k, experts, N, split, kind))
    assert bool((wide[:, N:] == 7.0).all()), "columns behind the result"


@pytest.mark.parametrize("formats", [("E2M3", "E5M2"), ("E3M2", "E5M2"), ("E2M3", "E4M3")], ids="-".join)
@pytest.mark.parametrize("tokens,N", [(3, 96), (90, 515), (1200, 600)])
def test_gemm_grouped_formats(tokens, N, formats):
    note(f"gemm grouped formats {formats} T={tokens}")
    ids, g, a, w, ref = _grouped(tokens, 2, 4, N, (128, 96, 96), "skewed", formats, own_sigma=True, seed=2)
    y = _b().gemm_grouped(a, w, g)  # (without y its rows in no group are zero)
    torch.cuda.synchronize()
    _check_rows(y, ref, 0.0, (formats, tokens))


@pytest.mark.parametrize("tokens,top_k,experts,N,split", [(4, 2, 8, 4100, (2048, 512, 512)), (64, 2, 3, 1000, (10752, 2688, 896)),
                                                          (3000, 1, 2, 1030, (640, 96, 160))])
def test_gemm_grouped_long(tokens, top_k, experts, N, split):
    """Several batches of steps per wavefront, many tiles."""
    note(f"gemm grouped long T={tokens} N={N} {split}")
    ids, g, a, w, ref = _grouped(tokens, top_k, experts, N, split, "even", seed=4)
    y = _b().gemm_grouped(a, w, g)
    torch.cuda.synchronize()
    _check_rows(y, ref, 0.0, (tokens, N, split))


@pytest.mark.parametrize("formats", [("E3M2", "E4M3"), ("E2M3", "E5M2"), ("E3M2", "E5M2"), ("E2M3", "E4M3")], ids="-".join)
@pytest.mark.parametrize("kernel,slots,experts,N,split", R.CASES, ids=str)
def test_gemm_grouped_kernels(kernel, slots, experts, N, split, formats):
    """Every compiled kernel with every format set, at sizes that are no multiple of its tile."""
    assert R.route(slots, experts, N, split, torch.cuda.get_device_properties(0).multi_processor_count)[0] == kernel
    note(f"gemm grouped {kernel} {formats}")
    cols = np.unique(np.concatenate([np.arange(0, N, max(1, N // 200)), np.arange(max(0, N - 40), N)]))
    ids, g, a, w, ref = _grouped(slots, 1, experts, N, split, "skewed", formats, own_sigma=True, seed=8, cols=cols)
    y = _b().gemm_grouped(a, w, g)
    torch.cuda.synchronize()
    _check_rows(y[:, torch.from_numpy(cols).cuda()], ref, 0.0, (kernel, formats))


@pytest.mark.parametrize("formats", [("E3M2", "E4M3"), ("E2M3", "E5M2"), ("E3M2", "E5M2"), ("E2M3", "E4M3")], ids="-".join)
@pytest.mark.parametrize("first,second", [(1501, 1499), (0, 2999), (1000, 0), (1500, 0), (0, 0), (1, 129)])
def test_gemm_grouped_last_round(first, second, formats):
    """256 x 256 tiles with the last round's in quarters: whole rounds with few tiles behind them, tiles for quarters
    alone or for whole tiles alone, none.  Rows of the two experts; the others of the 3000 are in no group."""
    slots, N, split, cus = 3000, 5400, (1024, 160, 832), torch.cuda.get_device_properties(0).multi_processor_count
    if cus == 256:
        assert R.route(slots, 2, N, split, cus)[0] == "tiled256x256+rest"
    note(f"gemm grouped last round {first} {second} {formats}")
    ids = np.full(slots, -1, np.int32)
    at = np.random.default_rng(first).permutation(slots)
    ids[at[:first]], ids[at[first:first + second]] = 0, 1
    cols = np.unique(np.concatenate([np.arange(0, N, 27), np.arange(N - 40, N)]))
    ids, g, a, w, ref = _grouped(slots, 1, 2, N, split, ids, formats, seed=10, cols=cols)
    y = _b().gemm_grouped(a, w, g)
    torch.cuda.synchronize()
    _check_rows(y[:, torch.from_numpy(cols).cuda()], ref, 0.0, (first, second, formats))


def test_last_round_captured_and_replayed():
    """One captured graph, ids that leave the quarters some, all or none of the tiles in turn."""
    note("last round captured")
    b, slots, N, split = _b(), 3000, 5400, (1024, 160, 832)
    K = sum(split)
    xb, perms = C.activations(slots, K, 1, seed=12)
    w, x, p = _stack(C.weights(2, N, K, seed=12), perms, split), to_dev_bf16(xb), to_dev_perm(perms[0])
    ids = torch.zeros(slots, dtype=torch.int32, device="cuda")
    g, a = b.RowGroups.empty(slots, 2), b.MXTensor.empty(b.RowGroups.empty(slots, 2).capacity, K, split)
    y = torch.zeros(slots, N, dtype=torch.bfloat16, device="cuda")

    def chain(y):
        b.group_rows(ids, 2, out=g)
        b.quantize_act_grouped(x, g, p, split, out=a)
        b.gemm_grouped(a, w, g, y=y)

    chain(y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        chain(y)
    for live in (3000, 1000, 1500, 0, 2990, 130):
        ids.fill_(-1)
        ids[:live] = torch.arange(live, device="cuda", dtype=torch.int32) % 2
        for t in (y, eager := torch.empty_like(y)):
            t.fill_(7.0)
        graph.replay()
        chain(eager)
        torch.cuda.synchronize()
        assert torch.equal(y, eager), live
        assert bool((y[live:] == 7.0).all()) and (live == 0 or not bool((y[:live] == 7.0).all(1).any())), live


def test_gemm_grouped_matches_gemm_alone():
    """One expert with every row is mm_gemm, up to the order of the fp32 sums."""
    note("gemm grouped against gemm")
    b, split, N, T = _b(), (320, 96, 64), 200, 70
    K = sum(split)
    xb, perms = C.activations(T, K, 1, seed=6)
    wb = C.weights(1, N, K, seed=6)
    w = _stack(wb, perms, split)
    p, x = to_dev_perm(perms[0]), to_dev_bf16(xb)
    g = b.group_rows(torch.zeros(T, dtype=torch.int32, device="cuda"), 1)
    y = b.gemm_grouped(b.quantize_act_grouped(x, g, p, split), w, g)
    alone = b.gemm(b.quantize_act(x, p, split), w[0])
    torch.cuda.synchronize()
    ref = O.gemm_mixed(O.quantize_mixed(xb, perms[0], split), O.quantize_mixed(wb[0], perms[0], split))
    assert_gemm_close(y_to_f64(y), ref, "grouped")
    assert_gemm_close(y_to_f64(alone), ref, "alone")


@pytest.mark.parametrize("word", [0, -1, 7, 0x00200005], ids=hex)
@pytest.mark.parametrize("tokens", [3, 900])
def test_map_that_was_not_filled(tokens, word):
    """A map that holds something else: nothing outside the buffers is touched (the rows between the results' columns,
    and the other operands, stay as they are)."""
    note(f"map of {word:#x}, {tokens} tokens")
    b, split, N, E = _b(), (96, 64, 64), 70, 3
    K = sum(split)
    xb, perms = C.activations(tokens, K, E, seed=61)
    w = _stack(C.weights(E, N, K, seed=62), perms, split)
    before = w.q4.clone()
    g = b.RowGroups.empty(tokens, E)
    g.map.fill_(word)
    a = _garbage(b.MXTensor.empty(g.capacity, K, split))
    b.quantize_act_grouped(to_dev_bf16(xb), g, _perm_arg(perms), split, out=a)
    wide = torch.full((tokens + 2, 88), 7.0, dtype=torch.bfloat16, device="cuda")
    b.gemm_grouped(a, w, g, y=wide[1:-1, 8:78])
    torch.cuda.synchronize()
    assert bool((wide[0] == 7).all() and (wide[-1] == 7).all() and (wide[:, :8] == 7).all() and (wide[:, 78:] == 7).all())
    assert torch.equal(w.q4, before) and bool((g.map == word).all())


# ---- matrix-vector products ----


def _check_gemv(y, ref, tol, before, ctx):
    got = y_to_f64(y)
    live = ~np.isnan(ref).any(axis=1)
    err = np.abs(got[live] - ref[live])
    assert np.all(err <= tol[live]), (ctx, float((err - tol[live]).max()), np.argwhere(err > tol[live])[:3])
    assert np.all(got[~live] == before), (ctx, "rows without an expert")


GEMV_FORMATS = [("E3M2", "E4M3"), ("E2M3", "E5M2"), ("E3M2", "E5M2"), ("E2M3", "E4M3")]


@pytest.mark.parametrize("formats", GEMV_FORMATS, ids="-".join)
@pytest.mark.parametrize("split", [(32, 0, 0), (352, 0, 0), (0, 352, 0), (0, 0, 352), (96, 160, 96), (2048, 1024, 1024),
                                   (128, 0, 224)], ids=str)
@pytest.mark.parametrize("rows,N", [(1, 1), (1, 70), (2, 32), (5, 129), (15, 40), (16, 264)])
def test_gemv_one_weight(rows, N, split, formats):
    note(f"gemv rows={rows} N={N} {split} {formats}")
    b, K = _b(), sum(split)
    xb, perms = C.activations(rows, K, 1, seed=rows)
    wb = C.weights(1, N, K, seed=rows + N)
    p = to_dev_perm(perms[0])
    w = b.quantize_weight(to_dev_bf16(wb[0]), p, split, formats=formats)
    wide = torch.full((rows, (N + 7) // 8 * 8 + 8), 7.0, dtype=torch.bfloat16, device="cuda")
    y = b.gemv(to_dev_bf16(xb), w, p, y=wide[:, :N])
    torch.cuda.synchronize()
    ref, tol = C.gemv_product(xb, None, 1, perms, wb, split, formats)
    _check_gemv(y, ref, tol, 7.0, (rows, N, split, formats))
    assert bool((wide[:, N:] == 7.0).all()), "columns behind the result"


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("tokens,top_k,experts,N,split,own_sigma", [
    (1, 1, 1, 33, (32, 0, 0), False), (1, 2, 8, 130, (96, 160, 96), False), (2, 8, 64, 72, (256, 0, 96), True),
    (16, 1, 3, 264, (512, 128, 128), True), (5, 3, 4, 40, (0, 224, 0), False)])
def test_gemv_experts(tokens, top_k, experts, N, split, own_sigma, kind):
    note(f"gemv T={tokens} k={top_k} E={experts} N={N} {split} {kind}")
    b, K = _b(), sum(split)
    ids = C.make_ids(tokens * top_k, experts, kind, seed=5)
    xb, perms = C.activations(tokens, K, experts if own_sigma else 1, seed=11)
    wb = C.weights(experts, N, K, seed=12)
    w = _stack(wb, perms, split)
    y = torch.full((tokens * top_k, (N + 7) // 8 * 8), -3.0, dtype=torch.bfloat16, device="cuda")[:, :N]
    b.gemv(to_dev_bf16(xb), w, _perm_arg(perms), ids=_dev_ids(ids), top_k=top_k, y=y)
    torch.cuda.synchronize()
    ref, tol = C.gemv_product(xb, ids, top_k, perms, wb, split, DEFAULT)
    _check_gemv(y, ref, tol, -3.0, (tokens, top_k, experts, N, split, kind))


@pytest.mark.parametrize("rows,split", [(1, (20736, 5184, 1728)), (8, (10752, 2688, 896)), (2, (0, 0, 8192))], ids=str)
def test_gemv_long(rows, split):
    """The widest down projections; x with a stride and at an address that is a multiple of 2 bytes only."""
    note(f"gemv long rows={rows} {split}")
    b, K, N = _b(), sum(split), 100
    xb, perms = C.activations(rows, K, 1, seed=21)
    wb = C.weights(1, N, K, seed=22)
    p = to_dev_perm(perms[0])
    w = b.quantize_weight(to_dev_bf16(wb[0]), p, split)
    wide = torch.full((rows, K + 3), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[:, 1:K + 1] = to_dev_bf16(xb)
    y = b.gemv(wide[:, 1:K + 1], w, p)
    torch.cuda.synchronize()
    ref, tol = C.gemv_product(xb, None, 1, perms, wb, split, DEFAULT)
    _check_gemv(y, ref, tol, 0.0, (rows, split))


# ---- offsets beyond 32 bits ----


def test_offsets_beyond_32_bits():
    """Weights behind 4 GiB of other experts', rows of x and of the results further apart than 4 GiB in all."""
    note("offsets beyond 32 bits")
    b, E, N, split = _b(), 5, 33000, (0, 0, 32768)
    K, last = sum(split), E - 1
    cols = np.unique(np.concatenate([np.arange(0, N, 2111), np.arange(N - 3, N)]))
    perm = np.random.default_rng(71).permutation(K).astype(np.int32)
    p = to_dev_perm(perm)
    w = b.MXStack.empty(E, N, K, split)
    assert last * (w.q8.nbytes // E) > 1 << 32
    wb = np.zeros((E, len(cols), K), np.uint16)
    for e in (0, last):
        torch.manual_seed(e)
        we = (torch.randn(N, K, device="cuda") * 0.02).bfloat16()
        b.quantize_weight(we, p, split, out=w[e])
        wb[e] = we[torch.from_numpy(cols).cuda()].cpu().view(torch.int16).numpy().view(np.uint16)
        del we
    at = torch.from_numpy(cols).cuda()
    for tokens in (3, 5, 700):  # the K-splitting kernel, 256 x 128 and 256 x 256 tiles
        ids = np.random.default_rng(tokens).choice(np.array([0, last, -1], np.int32), tokens)
        ids[-1] = last
        xb, _ = C.activations(tokens, K, 1, seed=tokens)
        apart = -(-(1 << 32) // (2 * (tokens - 1))) // 64 * 64 + 64  # elements from row to row
        apart = max(apart, K + 64)
        x = torch.empty(tokens * apart, dtype=torch.bfloat16, device="cuda").view(tokens, apart)[:, :K]
        x.copy_(to_dev_bf16(xb))
        yb = torch.empty(tokens * max(apart, N + 64), dtype=torch.bfloat16, device="cuda").view(tokens, -1)[:, :N]
        assert (tokens - 1) * x.stride(0) * 2 > 1 << 32 and (tokens - 1) * yb.stride(0) * 2 > 1 << 32
        yb.fill_(7.0)
        d = _dev_ids(ids)
        g = b.group_rows(d, E)
        b.gemm_grouped(b.quantize_act_grouped(x, g, p, split), w, g, y=yb)
        torch.cuda.synchronize()
        _check_rows(yb[:, at], C.grouped_product(xb, ids, 1, [perm], wb, split, DEFAULT), 7.0, (tokens, "gemm"))
        if tokens <= 16:
            yb.fill_(7.0)
            b.gemv(x, w, p, ids=d, y=yb)
            torch.cuda.synchronize()
            ref, tol = C.gemv_product(xb, ids, 1, [perm], wb, split, DEFAULT)
            _check_gemv(yb[:, at], ref, tol, 7.0, (tokens, "gemv"))
        del x, yb
    del w
    torch.cuda.empty_cache()


# ---- used together ----


def test_sparse_mlp():
    """A sparse MLP as it is served: router, up projections, gate, down projections with each expert's own sigma, the
    weighted sum; each product against its reference on the inputs that it had, and the single-token form against the
    same references."""
    note("sparse MLP")
    b = _b()
    T, k, E, H, F = 37, 2, 6, 352, 416
    up_split, down_split = (192, 96, 64), (224, 96, 96)
    xb, up_perm = C.activations(T, H, 1, seed=31)
    _, down_perms = C.activations(1, F, E, seed=32)
    wu, wd = C.weights(E, 2 * F, H, seed=33), C.weights(E, H, F, seed=34)
    up, down = _stack(wu, up_perm, up_split), _stack(wd, down_perms, down_split)
    x = to_dev_bf16(xb)
    logits = torch.randn((T, E), generator=torch.Generator("cuda").manual_seed(1), device="cuda")
    top = torch.topk(logits, k, dim=1)
    share, ids = torch.softmax(top.values, dim=1), top.indices.to(torch.int32)
    g = b.group_rows(ids, E)
    h = b.gemm_grouped(b.quantize_act_grouped(x, g, _perm_arg(up_perm), up_split, top_k=k), up, g)
    act = (torch.nn.functional.silu(h[:, :F].float()) * h[:, F:].float()).to(torch.bfloat16)
    y = b.gemm_grouped(b.quantize_act_grouped(act, g, _perm_arg(down_perms), down_split), down, g)
    out = (y.float().view(T, k, H) * share[:, :, None]).sum(1)
    torch.cuda.synchronize()
    n = ids.cpu().numpy().reshape(-1)
    assert_gemm_close(y_to_f64(h), C.grouped_product(xb, n, k, up_perm, wu, up_split, DEFAULT), "up")
    ab = act.view(torch.int16).cpu().numpy().view(np.uint16)
    ref = C.grouped_product(ab, n, 1, down_perms, wd, down_split, DEFAULT)
    assert_gemm_close(y_to_f64(y), ref, "down")
    assert bool(torch.isfinite(out).all())
    # one token alone, its experts' rows not quantised
    h1 = b.gemv(x[:1], up, _perm_arg(up_perm), ids=ids[0].contiguous(), top_k=k)
    act1 = (torch.nn.functional.silu(h1[:, :F].float()) * h1[:, F:].float()).to(torch.bfloat16)
    y1 = b.gemv(act1, down, _perm_arg(down_perms), ids=ids[0].contiguous())
    torch.cuda.synchronize()
    r, tol = C.gemv_product(xb[:1], n[:k], k, up_perm, wu, up_split, DEFAULT)
    _check_gemv(h1, r, tol, 0.0, "up, one token")
    a1 = act1.view(torch.int16).cpu().numpy().view(np.uint16)
    r, tol = C.gemv_product(a1, n[:k], 1, down_perms, wd, down_split, DEFAULT)
    _check_gemv(y1, r, tol, 0.0, "down, one token")


def _layer(x, ids, E, w, perm, split, k, keep):
    b = _b()
    g = b.group_rows(ids, E, out=keep["g"])
    a = b.quantize_act_grouped(x, g, perm, split, top_k=k, out=keep["a"])
    keep["y"].zero_()
    b.gemm_grouped(a, w, g, y=keep["y"])
    keep["v"].zero_()
    b.gemv(x[:2], w, perm, ids=ids[:2 * k], top_k=k, y=keep["v"], workspace=keep["ws"])
    return keep["y"], keep["v"]


def _keep(T, k, E, K, N, split):
    b = _b()
    g = b.RowGroups.empty(T * k, E)
    return {"g": g, "a": _garbage(b.MXTensor.empty(g.capacity, K, split)),
            "y": torch.zeros(T * k, N, dtype=torch.bfloat16, device="cuda"),
            "v": torch.zeros(2 * k, N, dtype=torch.bfloat16, device="cuda"),
            "ws": torch.empty(max(16, b.gemv_workspace_size(2 * k, K, split)), dtype=torch.uint8, device="cuda")}


@pytest.mark.parametrize("T", [9, 700])
def test_captured_and_replayed(T):
    """The whole chain captured once and replayed with other ids and rows, eager calls of the same on other buffers
    between the replays: bit for bit the eager results."""
    note(f"capture and replay T={T}")
    b, k, E, N, split = _b(), 2, 5, 264, (96, 64, 96)
    K = sum(split)
    xb, perms = C.activations(4 * T, K, E, seed=41)
    w = _stack(C.weights(E, N, K, seed=42), perms, split)
    perm, xs = _perm_arg(perms), to_dev_bf16(xb)
    all_ids = [_dev_ids(C.make_ids(T * k, E, kind, seed=7)) for kind in ("even", "holes", "none", "one")]
    x, ids = xs[:T].clone(), all_ids[0].clone()
    kept, eager = _keep(T, k, E, K, N, split), _keep(T, k, E, K, N, split)
    _layer(x, ids, E, w, perm, split, k, kept)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, v = _layer(x, ids, E, w, perm, split, k, kept)
    for turn in range(6):
        j = turn % 4
        x.copy_(xs[j * T:(j + 1) * T])
        ids.copy_(all_ids[j])
        graph.replay()
        ye, ve = _layer(x.clone(), ids.clone(), E, w, perm, split, k, eager)
        torch.cuda.synchronize()
        assert torch.equal(y, ye) and torch.equal(v, ve), (T, turn)


def test_two_streams():
    """Two chains at once on two streams, each with its own buffers."""
    note("two streams")
    T, k, E, N, split = 300, 2, 4, 520, (256, 128, 128)
    K = sum(split)
    xb, perms = C.activations(2 * T, K, 1, seed=51)
    w = _stack(C.weights(E, N, K, seed=52), perms, split)
    perm, xs = _perm_arg(perms), to_dev_bf16(xb)
    ids = [_dev_ids(C.make_ids(T * k, E, kind, seed=8)) for kind in ("even", "skewed")]
    x = [xs[:T], xs[T:]]
    want = [[t.clone() for t in _layer(x[i], ids[i], E, w, perm, split, k, _keep(T, k, E, K, N, split))] for i in (0, 1)]
    keeps = [_keep(T, k, E, K, N, split) for _ in (0, 1)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = [None, None]
    for _ in range(3):
        for i in (0, 1):
            with torch.cuda.stream(streams[i]):
                got[i] = _layer(x[i], ids[i], E, w, perm, split, k, keeps[i])
    torch.cuda.synchronize()
    for i in (0, 1):
        assert torch.equal(got[i][0], want[i][0]) and torch.equal(got[i][1], want[i][1]), i


def test_new_tensors_belong_to_the_call_stream():
    """stream=: what a call allocates is ordered with its kernels, not with the current stream, which is busy here."""
    note("stream= and new tensors")
    b = _b()
    T, k, E, N, split = 5, 2, 4, 520, (12288, 3584, 512)  # (gemv of ten rows: with a workspace)
    K = sum(split)
    xb, perms = C.activations(T, K, 1, seed=61)
    w = _stack(C.weights(E, N, K, seed=62), perms, split)
    perm, x = _perm_arg(perms), to_dev_bf16(xb)
    ids = _dev_ids(C.make_ids(T * k, E, "even", seed=9))
    assert b.gemv_workspace_size(T * k, K, split) > 0

    def layer(stream):
        g = b.group_rows(ids, E, stream=stream)
        q = b.quantize_act_grouped(x, g, perm, split, top_k=k, stream=stream)
        return b.gemm_grouped(q, w, g, stream=stream), b.gemv(x, w, perm, ids=ids, top_k=k, stream=stream)

    want = [t.clone() for t in layer(None)]
    other, busy = torch.cuda.Stream(), torch.zeros(1 << 28, device="cuda")
    torch.cuda.synchronize()
    for turn in range(3):
        for _ in range(100):
            busy.add_(1.0)
        got = layer(other)
        scratch = [torch.full((1 << 20,), 7, dtype=torch.uint8, device="cuda") for _ in range(8)]  # (behind the freed workspace)
        torch.cuda.synchronize()
        for a, e in zip(got, want):
            assert torch.equal(a, e), turn
        del scratch
