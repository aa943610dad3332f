"""The operators of sparse (mixture-of-experts) layers as cases that can be timed
and checked: each in a plain form of elementary torch operations, and as the
calls of `paper_2508_02343_amd.binding` (where `own` is true).

  group   group_rows: the rows (slots) of a batch ordered by the expert that
          each is routed to
  linear  quantize_act_grouped -> gemm_grouped: a linear layer whose rows are
          multiplied by their expert's weight, both operands in mixed MX formats
  gemv    gemv: a few bf16 rows (a single token's experts, or one dense weight)
          against weights in mixed MX formats

A slot is one (token, choice) pair: with top_k choices per token, slot s
belongs to token s // top_k.  Slots at the end of a padded batch have the
id -1 and take part in nothing.
"""

import math

import numpy as np
import torch

own = False

OUTLIERS, OUTLIER_SCALE, W_STD = 0.01, 30.0, 0.02
MAX_WEIGHT = 8 * 14336 * 4096  # elements of all experts' weights
MAX_PRODUCT = 8192 * 14336 * 4096  # rows x N x K of a linear case
MAX_GEMV = 8 * 14336 * 4096  # rows x N x K of a gemv case


def _split(K, f4=0.75, f6=0.1875):
    p4 = round(K * f4 / 32) * 32
    p6 = min(round(K * f6 / 32) * 32, K - p4)
    return p4, p6, K - p4 - p6


def _group(tokens, top_k, experts, skew=0.0, pad=0.0):
    return {"op": "group", "tokens": tokens, "top_k": top_k, "experts": experts, "skew": skew, "pad": pad}


def _linear(tokens, top_k, experts, K, N, up=True, split=None, skew=0.5, pad=0.0, fp6="E3M2", fp8="E4M3"):
    """up: the rows are the tokens' (each read top_k times) and the experts share sigma; else one row per slot and a
    sigma per expert (a down projection)."""
    p4, p6, p8 = split or _split(K)
    return {"op": "linear", "tokens": tokens, "top_k": top_k, "experts": experts, "K": K, "N": N, "up": up, "p4": p4,
            "p6": p6, "p8": p8, "skew": skew, "pad": pad, "fp6": fp6, "fp8": fp8}


def _gemv(tokens, top_k, experts, K, N, split=None, fp6="E3M2", fp8="E4M3"):
    """experts 0: one weight for every row (top_k 1)."""
    p4, p6, p8 = split or _split(K)
    return {"op": "gemv", "tokens": tokens, "top_k": top_k, "experts": experts, "K": K, "N": N, "p4": p4, "p6": p6,
            "p8": p8, "fp6": fp6, "fp8": fp8}


def listed():
    return [
        # eight sequences' tokens, two of eight experts each: a decode step's routing, the smallest call
        {"name": "group_decode_16", **_group(8, 2, 8)},
        # a prefill of 8192 tokens over many small experts, a sixteenth of the batch padding
        {"name": "group_prefill_65536", **_group(8192, 8, 128, skew=1.0, pad=1 / 16)},
        # a decode step of four sequences through the up projections of eight large experts
        {"name": "linear_decode_4_up", **_linear(4, 2, 8, 4096, 14336)},
        # a serving batch of 64 sequences through the down projections, each expert's own channel order
        {"name": "linear_batch_64_down", **_linear(64, 2, 8, 14336, 4096, up=False)},
        # a serving batch of 256 sequences through many small experts, eight of them per token
        {"name": "linear_batch_256_fine", **_linear(256, 8, 64, 2048, 1024, skew=0.25)},
        # a ragged prompt chunk, a padded batch, the other element formats, uneven experts, an odd width
        {"name": "linear_chunk_777_ragged", **_linear(777, 4, 16, 2080, 5400, split=(1024, 544, 512), skew=1.0,
                                                      pad=0.1, fp6="E2M3", fp8="E5M2")},
        # prefill of 2048 tokens through the up projections of eight large experts
        {"name": "linear_prefill_2048_up", **_linear(2048, 2, 8, 4096, 14336)},
        # prefill of 4096 tokens through their down projections: the largest call
        {"name": "linear_prefill_4096_down", **_linear(4096, 2, 8, 14336, 4096, up=False)},
        # one token through an attention projection in about 5.5 bits per weight
        {"name": "gemv_1_attn", **_gemv(1, 1, 0, 4096, 4096, (2048, 1024, 1024))},
        # one token's two experts, weights in four bits alone
        {"name": "gemv_1_top2_4bit", **_gemv(1, 2, 8, 4096, 14336, (4096, 0, 0))},
        # two tokens' eight small experts each
        {"name": "gemv_2_top8_fine", **_gemv(2, 8, 64, 2048, 1024)},
        # eight sequences through the widest dense down projection
        {"name": "gemv_8_wide_down", **_gemv(8, 1, 0, 27648, 5120)},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    op = rng.choice(["group"] + ["linear"] * 5 + ["gemv"] * 2)
    if op == "group":
        E = _log(rng, 2, 256)
        k = rng.randint(1, min(8, E))
        return _group(_log(rng, 1, 65536 // k), k, E, skew=rng.choice([0.0, 0.5, 1.0, 2.0]),
                      pad=rng.choice([0.0, 0.0, rng.uniform(0, 0.5)]))
    K = 32 * _log(rng, 512 // 32, 14336 // 32)
    fp6, fp8 = rng.choice([("E3M2", "E4M3")] * 4 + [("E2M3", "E5M2"), ("E2M3", "E4M3")])
    # mostly the split of about 5 bits per element, now and then one format alone or nearly even groups
    f4, f6 = rng.choice([(0.75, 0.1875)] * 2 + [(rng.uniform(0.5, 0.9), 0.1), (0.5, 0.25), (1.0, 0.0), (0.0, 0.0)])
    split = _split(K, f4, f6)
    if op == "gemv":
        E = rng.choice([0, 0, _log(rng, 2, 64)])
        k = rng.randint(1, min(8, E)) if E else 1
        tokens = _log(rng, 1, 16 // k)
        N = _log(rng, 256, min(28672, MAX_WEIGHT // (max(E, 1) * K), MAX_GEMV // (tokens * k * K)))
        return _gemv(tokens, k, E, K, N, split, fp6, fp8)
    E = _log(rng, 2, 64)
    k = rng.randint(1, min(8, E))
    N = _log(rng, 256, min(14336, MAX_WEIGHT // (E * K)))
    tokens = _log(rng, 1, max(1, min(8192, MAX_PRODUCT // (N * K)) // k))
    return _linear(tokens, k, E, K, N, up=rng.random() < 0.5, split=split, skew=rng.choice([0.0, 0.25, 0.5, 1.0, 2.0]),
                   pad=rng.choice([0.0, 0.0, rng.uniform(0, 0.5)]), fp6=fp6, fp8=fp8)


# ---- inputs ----


def _generator(seed, k):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 1000003 + k)
    return g


def _ids(case, seed):
    """int32 [tokens * top_k]: each token's top_k different experts, the later experts rarer with skew, the last tokens'
    ids -1."""
    T, k, E = case["tokens"], case["top_k"], case["experts"]
    score = -torch.log(-torch.log(torch.rand((T, E), generator=_generator(seed, 1), device="cuda").clamp(1e-20, 1 - 1e-7)))
    score -= case.get("skew", 0.0) * torch.log(1.0 + torch.arange(E, device="cuda"))
    ids = torch.topk(score, k, dim=1).indices.to(torch.int32)
    pad = int(T * case.get("pad", 0.0))
    if pad:
        ids[T - pad:] = -1
    return ids.reshape(-1)


def _activations(seed, rows, K, sigmas):
    """bf16 [rows, K] with a few large channels, and int32 [sigmas, K]: the regular channels in a random order, then the
    large ones."""
    g = _generator(seed, 2)
    order = torch.randperm(K, generator=g, device="cuda")
    n = max(1, round(OUTLIERS * K))
    x = torch.randn((rows, K), generator=g, device="cuda")
    x[:, order[K - n:]] *= OUTLIER_SCALE
    perms = [torch.cat([order[:K - n][torch.randperm(K - n, generator=g, device="cuda")], order[K - n:]])
             for _ in range(sigmas)]
    return x.to(torch.bfloat16), torch.stack(perms).to(torch.int32)


def _weight(seed, e, N, K):
    """Expert e's weight in the channels' own order, before it is quantised."""
    return torch.randn((N, K), generator=_generator(seed, 10 + e), device="cuda").mul_(W_STD).to(torch.bfloat16)


def _layer(case, seed):
    """(x, sigma of each expert or one of all, the experts' number) of a linear or gemv case."""
    E = max(case["experts"], 1)
    slots = case["tokens"] * case["top_k"]
    up = case.get("up", True)
    x, perms = _activations(seed, case["tokens"] if up else slots, case["K"], 1 if up else E)
    return x, perms, E


def _of(case):
    return (case["p4"], case["p6"], case["p8"]), (case["fp6"], case["fp8"])


def prepare(case, seed):
    if case["op"] == "group":
        s = {"op": "group", "experts": case["experts"], "ids": _ids(case, seed)}
        if own:
            from paper_2508_02343_amd import binding as B

            s["out"] = B.RowGroups.empty(s["ids"].numel(), case["experts"])
        return s
    split, formats = _of(case)
    x, perms, E = _layer(case, seed)
    N, K, slots = case["N"], case["K"], case["tokens"] * case["top_k"]
    sigma = lambda e: perms[e if perms.shape[0] > 1 else 0]
    s = {"op": case["op"], "x": x, "split": split, "formats": formats, "perm": perms if perms.shape[0] > 1 else perms[0],
         "each": case["top_k"] if case.get("up", True) else 1, "ids": _ids(case, seed) if case["experts"] else None}
    # the result's buffer, kept from call to call; its rows of slots without an expert stay zero
    s["y"] = torch.zeros((slots, (N + 7) // 8 * 8), dtype=torch.bfloat16, device="cuda")[:, :N]
    if own:
        from paper_2508_02343_amd import binding as B

        w = B.MXStack.empty(E, N, K, split, formats=formats)
        for e in range(E):
            B.quantize_weight(_weight(seed, e, N, K), sigma(e), split, out=w[e])
        s["w"] = w if case["experts"] else w[0]
        if case["op"] == "linear":
            s["groups"] = B.group_rows(s["ids"], E)
            s["a"] = B.MXTensor.empty(s["groups"].capacity, K, split, formats=formats)
        return s
    # the experts' weights as the values that the codes stand for, channels in sigma's order
    s["w"] = torch.empty((E, N, K), dtype=torch.bfloat16, device="cuda")
    for e in range(E):
        s["w"][e] = _mixed(_weight(seed, e, N, K).float()[:, sigma(e).long()], split, formats)
    if case["op"] == "linear":  # the routing in hand: slots by expert, and where each expert's end
        counts = torch.bincount(s["ids"].clamp(min=-1).long() + 1, minlength=E + 1)
        s["order"] = torch.argsort(s["ids"], stable=True)
        s["ends"] = torch.cumsum(counts, 0).tolist()
    return s


# ---- the plain forms ----

FORMATS = {  # mantissa bits, smallest normal exponent, largest value's exponent, largest value
    "E2M1": (1, 0, 2, 6.0), "E3M2": (2, -2, 4, 28.0), "E2M3": (3, 0, 2, 7.5), "E4M3": (3, -6, 8, 448.0),
    "E5M2": (2, -14, 15, 57344.0)}


def _scaled(x, e):
    """x 2^e (32 bits), e whole, -126 to 127: the power made from its bits, as a power function may be a step off."""
    return x * ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _mx(x, fmt):
    """x (32 bits, [rows, 32 n]) rounded to MX blocks of 32 elements of format fmt, as values: every scaling is by a power
    of two, so each step but the rounding to the element format is exact."""
    m, emin, emax, top = FORMATS[fmt]
    b = x.reshape(x.shape[0], -1, 32)
    amax = b.abs().amax(dim=2, keepdim=True)
    e = (torch.frexp(amax).exponent - 1 - emax).clamp(min=-126)  # (these inputs' blocks lie far above that)
    v = _scaled(b, -e)
    step = (torch.frexp(v).exponent - 1).clamp(min=emin) - m
    q = _scaled(torch.round(_scaled(v, -step)), step).clamp(-top, top)
    return _scaled(q, e).reshape(x.shape)


def _mixed(x, split, formats):
    """x (32 bits, channels in sigma's order) rounded to the three groups' formats."""
    p4, p6, _ = split
    parts = [(x[:, :p4], "E2M1"), (x[:, p4:p4 + p6], formats[0]), (x[:, p4 + p6:], formats[1])]
    return torch.cat([_mx(p, f) for p, f in parts if p.shape[1]], dim=1)


def _plain_group(ids, experts):
    slots = ids.numel()
    capacity = (slots + 31 * min(experts, slots)) // 32 * 32
    valid = (ids >= 0) & (ids < experts)
    key = torch.where(valid, ids, experts).long()
    counts = torch.zeros(experts + 1, dtype=torch.int64, device=ids.device).scatter_add_(0, key, torch.ones_like(key))
    starts = torch.cumsum((counts + 31) // 32 * 32, 0) - (counts + 31) // 32 * 32  # (the last: behind every expert's rows)
    first = torch.cumsum(counts, 0) - counts
    order = torch.argsort(key, stable=True)
    of = key[order]
    at = torch.where(of < experts, starts[of] + torch.arange(slots, device=ids.device) - first[of], capacity)
    rows = torch.full((capacity + 1,), -1, dtype=torch.int32, device=ids.device)
    rows[at] = order.to(torch.int32)
    group = 32 * torch.arange(capacity // 32, device=ids.device)
    owners = torch.searchsorted(starts[1:], group, right=True)
    owners = torch.where(group < starts[experts], owners, -1)
    return {"starts": starts.to(torch.int32), "slots": rows[:capacity], "owners": owners.to(torch.int32)}


def _plain_linear(s):
    x, order = s["x"].float(), s["order"][s["ends"][0]:]  # (ends[0]: the slots without an expert come first)
    if s["perm"].dim() == 2:  # a row's channels in its own expert's order, else one order for all
        a = _mixed(torch.gather(x[order], 1, s["perm"].long()[s["ids"][order].long()]), s["split"], s["formats"])
    else:
        a = _mixed(x[:, s["perm"].long()], s["split"], s["formats"])[order // s["each"]]
    products = [a[lo - s["ends"][0]:hi - s["ends"][0]] @ w.float().T  # one per expert: ragged sizes have no single one
                for w, lo, hi in zip(s["w"], s["ends"], s["ends"][1:]) if hi > lo]
    y = torch.zeros_like(s["y"])
    if products:
        y[order] = torch.cat(products).to(torch.bfloat16)
    return y


def _plain_gemv(s):
    x = s["x"].float()[:, s["perm"].long()]
    if s["ids"] is None:
        return (x @ s["w"][0].float().T).to(torch.bfloat16)
    w = s["w"][s["ids"].long()].float()
    x = x.repeat_interleave(s["each"], dim=0)
    return torch.bmm(w, x.unsqueeze(2)).squeeze(2).to(torch.bfloat16)


def run(state):
    s = state
    if own:
        from paper_2508_02343_amd import binding as B

        if s["op"] == "group":
            g = B.group_rows(s["ids"], s["experts"], out=s["out"])
            return {"starts": g.starts, "slots": g.slots, "owners": g.owners}
        if s["op"] == "linear":
            a = B.quantize_act_grouped(s["x"], s["groups"], s["perm"], s["split"], top_k=s["each"], out=s["a"])
            return {"y": B.gemm_grouped(a, s["w"], s["groups"], y=s["y"])}
        return {"y": B.gemv(s["x"], s["w"], s["perm"], ids=s["ids"], top_k=s["each"], y=s["y"])}
    if s["op"] == "group":
        return _plain_group(s["ids"], s["experts"])
    return {"y": _plain_linear(s) if s["op"] == "linear" else _plain_gemv(s)}


# ---- what a case cannot do without, and how exact it is ----


def _active(case):
    """Experts that have rows, as many as expected."""
    E, k = case["experts"], case["top_k"]
    if not E:
        return 1
    tokens = case["tokens"] - int(case["tokens"] * case.get("pad", 0.0))
    share = [(1.0 + e) ** -case.get("skew", 0.0) for e in range(E)]
    return sum(1 - (1 - min(1.0, k * v / sum(share))) ** tokens for v in share)


def work(case):
    slots = case["tokens"] * case["top_k"]
    if case["op"] == "group":
        E = case["experts"]
        capacity = (slots + 31 * min(E, slots)) // 32 * 32
        return {"bytes": 4 * (slots + E + 1 + capacity + capacity // 32), "flops": slots}
    K, N = case["K"], case["N"]
    row = case["p4"] // 2 + case["p6"] * 3 // 4 + case["p8"] + K // 32
    up = case.get("up", True)
    live = (case["tokens"] - int(case["tokens"] * case.get("pad", 0.0))) * case["top_k"]
    active = _active(case)
    x = 2 * K * (live // case["top_k"] if up else live)
    sigma = 4 * K * (1 if up else active)
    return {"bytes": int(active * N * row + x + sigma + 2 * live * N + 4 * slots), "flops": 2 * live * N * K}


def _exact_mx(x, fmt):
    """x (64 bits) rounded to fmt by its table of values: the nearest, ties to the even code."""
    m, emin, emax, top = FORMATS[fmt]
    codes = np.arange(1 << 8)
    exponent, mantissa = codes >> m, codes & ((1 << m) - 1)
    value = np.where(exponent == 0, mantissa * 2.0 ** (emin - m), (2 ** m + mantissa) * 2.0 ** (exponent - 1 + emin - m))
    value = torch.from_numpy(value[value <= top]).to(x.device)
    middle = (value[1:] + value[:-1]) / 2
    b = x.reshape(x.shape[0], -1, 32)
    amax = b.abs().amax(dim=2, keepdim=True)
    e = ((amax.view(torch.int64) >> 52) - 1023 - emax).clamp(min=-127)  # floor(log2 amax) - emax
    power, inverse = ((1023 + e) << 52).view(torch.float64), ((1023 - e) << 52).view(torch.float64)
    v = (b * inverse).abs()
    low, high = torch.bucketize(v, middle), torch.bucketize(v, middle, right=True)
    code = torch.where(low % 2 == 0, low, high)
    return (torch.copysign(value[code], b) * power).reshape(x.shape)


def _exact_operand(x, split, formats):
    out, at = [], 0
    for p, f in zip(split, ("E2M1", *formats)):
        if p:
            out.append(_exact_mx(x[:, at:at + p], f))
        at += p
    return torch.cat(out, dim=1)


def exact(case, seed):
    if case["op"] == "group":
        return None
    split, formats = _of(case)
    x, perms, E = _layer(case, seed)
    slots, N, K = case["tokens"] * case["top_k"], case["N"], case["K"]
    ids = _ids(case, seed) if case["experts"] else torch.zeros(slots, dtype=torch.int32, device="cuda")
    each = case["top_k"] if case.get("up", True) else 1
    y = torch.zeros((slots, N), dtype=torch.float64, device="cuda")
    for e in range(E):
        rows = torch.nonzero(ids == e).flatten()
        if not rows.numel():
            continue
        perm = perms[e if perms.shape[0] > 1 else 0].long()
        a = x[torch.div(rows, each, rounding_mode="floor")].double()[:, perm]
        if case["op"] == "linear":
            a = _exact_operand(a, split, formats)
        y[rows] = a @ _exact_operand(_weight(seed, e, N, K).double()[:, perm], split, formats).T
    return {"y": y}
