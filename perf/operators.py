"""The operators around routed experts and 8-bit products, as measurable passes: in their plain form (elementary torch
operations) or, with ``own`` set, through the library's public entry points.

A case is a dict of plain values; ``op`` names the operator:

  route     scores of a router's logits, optional bias and groups, top-k, weights         (bitcos_route_experts)
  group     routed pairs sorted by expert, with every pair's place                        (bitcos_group_pairs_slots)
  quantize  activations to e4m3 with one scale per row and group of 128                   (bitcos_fp8_quantize)
  matmul    e4m3 product, one weight scale per 128 x 128 block                            (bitcos_fp8_matmul)
  grouped   the same over the routed pairs' experts                                       (bitcos_fp8_matmul_grouped)
  combine   the experts' outputs weighted and added, token by token                       (bitcos_combine_pairs)

Shapes are those of the library's own configurations (a 2B and a 32B dense layer, 128 experts of 768 x 2048 with eight
per token) or lie in the ranges around them.  Everything is made from the seed with torch generators on the GPU.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

GROUP = 128
E4M3_MAX = 448.0
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
SIZES = {"fp32": 4, "bf16": 2, "fp16": 2}


def listed():
    return [
        # one decode token through the router of 128 experts: latency only
        {"name": "route_1x128_top8", "op": "route", "tokens": 1, "experts": 128, "top_k": 8, "score": "softmax", "bias": False,
         "groups": 1, "top_groups": 1, "group_best": 1, "renormalise": True, "scale": 1.0, "dtype": "fp32"},
        # a long prompt, 256 experts in 8 groups of which 4 are kept by their two best, balance bias
        {"name": "route_16384x256_groups", "op": "route", "tokens": 16384, "experts": 256, "top_k": 8, "score": "sigmoid",
         "bias": True, "groups": 8, "top_groups": 4, "group_best": 2, "renormalise": True, "scale": 2.5, "dtype": "bf16"},
        # the pairs of one decode step of 16 sequences
        {"name": "group_16x8_of_128", "op": "group", "tokens": 16, "top_k": 8, "experts": 128, "dropped": 0.0},
        # the pairs of a long prompt; some places stay empty where a mask left too few experts
        {"name": "group_32768x8_of_128", "op": "group", "tokens": 32768, "top_k": 8, "experts": 128, "dropped": 0.01},
        # a decode step's activations in front of the 2B model's projections
        {"name": "quantize_16x2560", "op": "quantize", "rows": 16, "K": 2560, "dtype": "fp32"},
        # a long prompt in front of the 32B model's projections
        {"name": "quantize_8191x5120", "op": "quantize", "rows": 8191, "K": 5120, "dtype": "bf16"},
        # one decode token through the 2B model's gate projection
        {"name": "matmul_1x6912x2560", "op": "matmul", "rows": 1, "M": 6912, "K": 2560, "out": "fp32"},
        # a prompt of odd length through the 32B model's q projection
        {"name": "matmul_4095x8192x5120", "op": "matmul", "rows": 4095, "M": 8192, "K": 5120, "out": "bf16"},
        # eight decode tokens, eight experts each
        {"name": "grouped_8x8_768x2048", "op": "grouped", "tokens": 8, "top_k": 8, "experts": 128, "M": 768, "K": 2048, "out": "fp32"},
        # a prompt through the experts' gate and up projections, stacked
        {"name": "grouped_4096x8_1536x2048", "op": "grouped", "tokens": 4096, "top_k": 8, "experts": 128, "M": 1536, "K": 2048,
         "out": "bf16"},
        # one decode step's sums over the experts, on top of a residual
        {"name": "combine_5x8_2048", "op": "combine", "tokens": 5, "top_k": 8, "M": 2048, "y": "fp32", "out": "fp32", "base": True,
         "dropped": 0.0},
        # the sums of a long prompt
        {"name": "combine_8192x8_2048", "op": "combine", "tokens": 8192, "top_k": 8, "M": 2048, "y": "bf16", "out": "bf16", "base": False,
         "dropped": 0.01},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _log_groups(rng, lo, hi):
    return GROUP * _log_int(rng, lo // GROUP, hi // GROUP)


def draw(rng):
    op = rng.choice(["route", "group", "quantize", "matmul", "matmul", "grouped", "grouped", "combine"])
    if op == "route":
        groups = rng.choice([1, 1, 2, 4, 8])
        experts = groups * _log_int(rng, 8, 256 // groups) if groups > 1 else _log_int(rng, 8, 256)
        top_groups = rng.randint(1, groups)
        return {"op": op, "tokens": _log_int(rng, 1, 16384), "experts": experts, "top_k": rng.randint(1, 8),
                "score": rng.choice(["softmax", "sigmoid"]), "bias": rng.random() < 0.5, "groups": groups, "top_groups": top_groups,
                "group_best": rng.choice([1, 2]), "renormalise": rng.random() < 0.7, "scale": rng.choice([1.0, 2.5]),
                "dtype": rng.choice(["fp32", "bf16", "fp16"])}
    if op == "group":
        return {"op": op, "tokens": _log_int(rng, 1, 32768), "top_k": rng.randint(1, 8), "experts": _log_int(rng, 8, 256),
                "dropped": rng.choice([0.0, 0.01, 0.3])}
    if op == "quantize":
        return {"op": op, "rows": _log_int(rng, 1, 8191), "K": _log_groups(rng, 128, 5120), "dtype": rng.choice(["fp32", "bf16"])}
    if op == "matmul":
        while True:
            rows, M, K = _log_int(rng, 1, 4095), _log_int(rng, 64, 25600), _log_groups(rng, 128, 25600)
            if M * K <= 25600 * 5120 and rows * M * K <= 4095 * 8192 * 5120 and rows * M <= 4095 * 8192:
                return {"op": op, "rows": rows, "M": M, "K": K, "out": rng.choice(["fp32", "bf16"])}
    if op == "grouped":
        return {"op": op, "tokens": _log_int(rng, 1, 4096), "top_k": rng.randint(1, 8), "experts": _log_int(rng, 8, 128),
                "M": _log_int(rng, 64, 1536), "K": _log_groups(rng, 128, 2048), "out": rng.choice(["fp32", "bf16"])}
    y = rng.choice(["fp32", "bf16"])
    return {"op": op, "tokens": _log_int(rng, 1, 4096 if y == "fp32" else 8192), "top_k": rng.randint(1, 8), "M": _log_int(rng, 64, 2048),
            "y": y, "out": rng.choice(["fp32", "bf16"]), "base": rng.random() < 0.5, "dropped": rng.choice([0.0, 0.01, 0.3])}


# ---------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------
def _activations(rows, K, gen):
    """Variance one, every 97th channel 24 times as large (a few outlier channels carry the range)."""
    x = torch.randn(rows, K, generator=gen, device="cuda")
    x[:, ::97] *= 24.0
    return x


def _codes_by_row(x):
    """e4m3 codes and scales per row and group of 128."""
    rows, K = x.shape
    g = x.view(rows, K // GROUP, GROUP)
    scale = g.abs().amax(2).clamp_min(2.0 ** -100) / E4M3_MAX
    return (g / scale[..., None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn).view(rows, K), scale


def _weights(count, M, K, gen):
    """e4m3 codes [count, M, K] and one scale per 128 x 128 block [count, ceil(M / 128), K / 128]."""
    blocks = (M + GROUP - 1) // GROUP
    codes = torch.empty(count, M, K, dtype=torch.float8_e4m3fn, device="cuda")
    scales = torch.empty(count, blocks, K // GROUP, device="cuda")
    for e in range(count):
        w = torch.zeros(blocks * GROUP, K, device="cuda")
        w[:M] = torch.randn(M, K, generator=gen, device="cuda") * 0.02
        b = w.view(blocks, GROUP, K // GROUP, GROUP)
        s = b.abs().amax((1, 3)) / E4M3_MAX
        scales[e] = s
        codes[e] = (b / s[:, None, :, None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn).view(blocks * GROUP, K)[:M]
    return codes, scales


def _choices(tokens, top_k, experts, dropped, gen):
    """top_k distinct experts per token (fewer experts than places: -1), a share of the places dropped (-1)."""
    picks = min(top_k, experts)
    order = torch.rand(tokens, experts, generator=gen, device="cuda").argsort(1)[:, :picks]
    chosen = torch.full((tokens, top_k), -1, dtype=torch.int32, device="cuda")
    chosen[:, :picks] = order.to(torch.int32)
    if dropped > 0:
        chosen[torch.rand(tokens, top_k, generator=gen, device="cuda") < dropped] = -1
    return chosen


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    st = {"case": case}
    op = case["op"]
    if op == "route":
        st["logits"] = (torch.randn(case["tokens"], case["experts"], generator=gen, device="cuda") * 1.5).to(TYPES[case["dtype"]])
        st["bias"] = torch.rand(case["experts"], generator=gen, device="cuda") * 0.2 - 0.1 if case["bias"] else None
    elif op == "group":
        st["chosen"] = _choices(case["tokens"], case["top_k"], case["experts"], case["dropped"], gen)
    elif op == "quantize":
        st["x"] = _activations(case["rows"], case["K"], gen).to(TYPES[case["dtype"]])
    elif op == "matmul":
        codes, scales = _weights(1, case["M"], case["K"], gen)
        st["w"], st["w_scale"] = codes[0], scales[0]
        st["x"], st["x_scale"] = _codes_by_row(_activations(case["rows"], case["K"], gen))
    elif op == "grouped":
        st["w"], st["w_scale"] = _weights(case["experts"], case["M"], case["K"], gen)
        st["x"], st["x_scale"] = _codes_by_row(_activations(case["tokens"], case["K"], gen))
        pair = _choices(case["tokens"], case["top_k"], case["experts"], 0.0, gen).flatten()
        kept = (pair >= 0).nonzero().flatten()
        order = kept[pair[kept].argsort(stable=True)]
        ids, counts = pair[order].unique_consecutive(return_counts=True)
        most = min(pair.numel(), case["experts"])
        st["group_expert"] = torch.zeros(most, dtype=torch.int32, device="cuda")
        st["group_expert"][:ids.numel()] = ids
        st["group_begin"] = torch.zeros(most + 1, dtype=torch.int32, device="cuda")
        st["group_begin"][1:ids.numel() + 1] = counts.cumsum(0)
        st["n_groups"] = torch.tensor([ids.numel()], dtype=torch.int32, device="cuda")
        st["pair_xrow"] = torch.zeros(pair.numel(), dtype=torch.int32, device="cuda")
        st["pair_xrow"][:order.numel()] = (order // case["top_k"]).to(torch.int32)
        # (a program that multiplies with library calls holds the groups on the host)
        st["groups"] = list(zip(ids.tolist(), counts.tolist()))
    else:
        P = case["tokens"] * case["top_k"]
        st["y"] = torch.randn(P, case["M"], generator=gen, device="cuda").to(TYPES[case["y"]])
        slot = torch.randperm(P, generator=gen, device="cuda").to(torch.int32).view(case["tokens"], case["top_k"])
        if case["dropped"] > 0:
            slot[torch.rand(slot.shape, generator=gen, device="cuda") < case["dropped"]] = -1
        st["slot"] = slot
        weight = torch.rand(case["tokens"], case["top_k"], generator=gen, device="cuda") + 0.05
        st["weight"] = weight / weight.sum(1, keepdim=True)
        st["base"] = torch.randn(case["tokens"], case["M"], generator=gen, device="cuda").to(TYPES[case["out"]]) if case["base"] else None
    if own:
        import paper_2609_16338_b200 as bc
        bc.load_library()
        st["bc"] = bc
        if op in ("matmul", "grouped"):
            st["W"] = bc.Fp8Weights(st["w"], st["w_scale"])
            rows = case["rows"] if op == "matmul" else case["tokens"] * case["top_k"]
            st["out"] = torch.zeros(rows, case["M"], dtype=TYPES[case["out"]], device="cuda")
            st["workspace"] = bc.make_fp8_workspace()
        if op == "group":
            st["workspace"] = bc.make_group_workspace(case["tokens"] * case["top_k"], case["experts"])
    return st


# ---------------------------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------------------------
def _first_best(values, count):
    """Indices of the `count` largest of every row, largest first, equal ones by index."""
    return values.sort(dim=1, descending=True, stable=True).indices[:, :count]


def _plain_route(st, c):
    # in 64 bits: which expert is taken hangs on differences of scores
    logits = st["logits"].double()
    tokens, experts = logits.shape
    if c["score"] == "softmax":
        scores = (logits - logits.amax(1, keepdim=True)).exp()
        scores = scores / scores.sum(1, keepdim=True)
    else:
        scores = 1.0 / (1.0 + (-logits).exp())
    choice = scores + st["bias"].double() if st["bias"] is not None else scores
    if c["groups"] > 1:
        by_group = choice.view(tokens, c["groups"], experts // c["groups"])
        best = by_group.sort(dim=2, descending=True).values[:, :, :c["group_best"]].sum(2)
        kept = torch.zeros(tokens, c["groups"], dtype=torch.bool, device="cuda")
        kept.scatter_(1, _first_best(best, c["top_groups"]), True)
        choice = by_group.masked_fill(~kept[..., None], -math.inf).view(tokens, experts)
    picks = min(c["top_k"], experts)
    taken = _first_best(choice, picks)
    there = choice.gather(1, taken) > -math.inf
    weight = scores.gather(1, taken) * there
    if c["renormalise"]:
        weight = weight / (weight.sum(1, keepdim=True) + 1e-20)
    expert = torch.full((tokens, c["top_k"]), -1, dtype=torch.int32, device="cuda")
    expert[:, :picks] = torch.where(there, taken, -1).to(torch.int32)
    weights = torch.zeros(tokens, c["top_k"], device="cuda")
    weights[:, :picks] = (weight * c["scale"]).float()
    xrow = torch.arange(tokens, dtype=torch.int32, device="cuda").repeat_interleave(c["top_k"])
    return expert, weights, xrow


def _plain_group(st, c):
    pair = st["chosen"].flatten()
    P, cap = pair.numel(), min(pair.numel(), c["experts"])
    inside = (pair >= 0) & (pair < c["experts"])
    key = torch.where(inside, pair, c["experts"])
    order = key.sort(stable=True).indices
    kept = inside.sum()
    place = torch.arange(P, device="cuda")
    slot = torch.empty_like(pair)
    slot[order] = torch.where(place < kept, place, -1).to(torch.int32)
    xrow = torch.where(place < kept, order // c["top_k"], 0).to(torch.int32)
    order = torch.where(place < kept, order, -1).to(torch.int32)
    counts = torch.zeros(c["experts"] + 1, dtype=torch.int64, device="cuda").scatter_add_(0, key.long(), torch.ones_like(key, dtype=torch.int64))[:-1]
    some = counts > 0
    n_groups = some.sum()
    at = torch.where(some, some.cumsum(0) - 1, cap + 1)
    group_expert = torch.zeros(cap + 2, dtype=torch.int32, device="cuda")
    group_expert[at] = torch.arange(c["experts"], dtype=torch.int32, device="cuda")
    group_begin = torch.zeros(cap + 2, dtype=torch.int32, device="cuda")
    group_begin[at] = (counts.cumsum(0) - counts).to(torch.int32)
    group_begin[n_groups] = kept.to(torch.int32)
    return group_expert[:cap], group_begin[:cap + 1], xrow, order, slot.view_as(st["chosen"]), n_groups.to(torch.int32).view(1)


def _plain_quantize(st, c):
    # (the codes hang on these very operations: maximum, quotient and product in 32 bits, one rounding to e4m3; a number
    # divided by or into a tensor is a product with a reciprocal on the GPU, so both sides are tensors)
    x = st["x"].float().view(c["rows"], c["K"] // GROUP, GROUP)
    a = x.abs().amax(2).clamp_min(2.0 ** -100)
    most = torch.full_like(a, E4M3_MAX)
    codes = (x * (most / a)[..., None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
    return codes.view(c["rows"], c["K"]), a / most


def _plain_product(w, w_scale, x, x_scale):
    M, K = w.shape
    wide = w.float().view(M, K // GROUP, GROUP) * w_scale.repeat_interleave(GROUP, 0)[:M, :, None]
    xs = x.float().view(-1, K // GROUP, GROUP) * x_scale[..., None]
    return xs.view(-1, K) @ wide.view(M, K).T


def _plain_grouped(st, c):
    """One batched product: every group's rows padded to the longest group's."""
    groups, K = len(st["groups"]), c["K"]
    longest = max(count for _, count in st["groups"])
    expert, begin = st["group_expert"][:groups].long(), st["group_begin"][:groups + 1].long()
    at = begin[:-1, None] + torch.arange(longest, device="cuda")[None, :]
    there = at < begin[1:, None]
    rows = st["pair_xrow"][torch.where(there, at, 0)].long()
    wide = st["w"].view(torch.uint8)[expert].view(torch.float8_e4m3fn).float().view(groups, c["M"], K // GROUP, GROUP)
    wide *= st["w_scale"][expert].repeat_interleave(GROUP, 1)[:, :c["M"], :, None]
    xs = st["x"].float().view(-1, K // GROUP, GROUP) * st["x_scale"][..., None]
    y = torch.bmm(xs.view(-1, K)[rows], wide.view(groups, c["M"], K).transpose(1, 2))
    out = torch.zeros(c["tokens"] * c["top_k"], c["M"], device="cuda")
    out[at[there]] = y[there]
    return out.to(TYPES[c["out"]])


def _plain_combine(st, c):
    there = st["slot"] >= 0
    rows = st["y"][st["slot"].clamp_min(0).long()].float() * torch.where(there, st["weight"], 0.0)[..., None]
    total = rows.sum(1)
    if st["base"] is not None:
        total = total + st["base"].float()
    return total.to(TYPES[c["out"]])


def run(st):
    c = st["case"]
    op = c["op"]
    if own:
        bc = st["bc"]
        if op == "route":
            return bc.bitcos_route_experts(st["logits"], c["top_k"], bias=st["bias"], score=c["score"], n_groups=c["groups"],
                                           top_groups=c["top_groups"], group_best=c["group_best"], renormalise=c["renormalise"],
                                           scale=c["scale"])
        if op == "group":
            return bc.bitcos_group_pairs_slots(st["chosen"], c["experts"], workspace=st["workspace"])
        if op == "quantize":
            return bc.bitcos_fp8_quantize(st["x"])
        if op == "matmul":
            return bc.bitcos_fp8_matmul(st["W"], st["x"], st["x_scale"], y=st["out"], workspace=st["workspace"])
        if op == "grouped":
            return bc.bitcos_fp8_matmul_grouped(st["W"], st["group_expert"], st["group_begin"], st["n_groups"], st["pair_xrow"], st["x"],
                                                st["x_scale"], y=st["out"], workspace=st["workspace"])
        return bc.bitcos_combine_pairs(st["y"], st["slot"], st["weight"], base=st["base"], out_dtype=TYPES[c["out"]])
    if op == "route":
        return _plain_route(st, c)
    if op == "group":
        return _plain_group(st, c)
    if op == "quantize":
        return _plain_quantize(st, c)
    if op == "matmul":
        return _plain_product(st["w"], st["w_scale"], st["x"], st["x_scale"]).to(TYPES[c["out"]])
    if op == "grouped":
        return _plain_grouped(st, c)
    return _plain_combine(st, c)


# ---------------------------------------------------------------------------------------------
# what a pass cannot do without, and its results in 64 bits
# ---------------------------------------------------------------------------------------------
def work(case):
    op = case["op"]
    if op == "route":
        T, E, k = case["tokens"], case["experts"], case["top_k"]
        return {"bytes": T * E * SIZES[case["dtype"]] + (4 * E if case["bias"] else 0) + 12 * T * k, "flops": 4 * T * E}
    if op == "group":
        P, cap = case["tokens"] * case["top_k"], min(case["tokens"] * case["top_k"], case["experts"])
        return {"bytes": 16 * P + 8 * cap + 8, "flops": P}
    if op == "quantize":
        n = case["rows"] * case["K"]
        return {"bytes": n * (SIZES[case["dtype"]] + 1) + n // GROUP * 4, "flops": 3 * n}
    if op == "matmul":
        T, M, K = case["rows"], case["M"], case["K"]
        return {"bytes": M * K + T * K + 4 * (K // GROUP) * (T + (M + GROUP - 1) // GROUP) + T * M * SIZES[case["out"]], "flops": 2 * T * M * K}
    if op == "grouped":
        T, M, K = case["tokens"], case["M"], case["K"]
        P = T * min(case["top_k"], case["experts"])
        # (experts that T tokens with distinct picks reach on average)
        reached = case["experts"] * (1.0 - (1.0 - min(case["top_k"], case["experts"]) / case["experts"]) ** T)
        blocks = (M + GROUP - 1) // GROUP
        return {"bytes": int(reached * (M * K + 4 * blocks * (K // GROUP))) + T * (K + 4 * (K // GROUP)) + P * M * SIZES[case["out"]],
                "flops": 2 * P * M * K}
    T, k, M = case["tokens"], case["top_k"], case["M"]
    rows = int(T * k * (1.0 - case["dropped"]))
    return {"bytes": rows * M * SIZES[case["y"]] + T * M * SIZES[case["out"]] * (2 if case["base"] else 1) + 8 * T * k,
            "flops": 2 * rows * M}


def _exact_route(st, c):
    """Token by token in effect: numpy, 64 bits, the order of the experts from a lexicographic sort."""
    z = st["logits"].cpu().to(torch.float64).numpy()
    T, E = z.shape
    k = c["top_k"]
    if c["score"] == "softmax":
        top = z.max(axis=1)[:, None]
        s = np.exp(z - top - np.log(np.exp(z - top).sum(axis=1))[:, None])
    else:
        s = np.where(z >= 0, 1.0 / (1.0 + np.exp(-np.abs(z))), np.exp(-np.abs(z)) / (1.0 + np.exp(-np.abs(z))))
    pick = s + (st["bias"].cpu().to(torch.float64).numpy()[None, :] if st["bias"] is not None else 0.0)
    n = E // c["groups"]
    group_of = np.arange(E) // n
    allowed = np.ones((T, E), bool)
    if c["groups"] > 1:
        value = np.empty((T, c["groups"]))
        for g in range(c["groups"]):
            part = np.sort(pick[:, group_of == g], axis=1)
            value[:, g] = part[:, n - c["group_best"]:].sum(axis=1)
        # the rank of a group: how many are larger, or equal and in front of it
        for g in range(c["groups"]):
            ahead = (value > value[:, g:g + 1]).sum(axis=1) + (value[:, :g] == value[:, g:g + 1]).sum(axis=1)
            allowed[:, group_of == g] = (ahead < c["top_groups"])[:, None]
    expert, weight = np.full((T, k), -1, np.int32), np.zeros((T, k))
    left = np.where(allowed, pick, -np.inf)
    rows = np.arange(T)
    for j in range(min(k, E)):
        e = left.argmax(axis=1)                      # (the first of equal ones)
        ok = left[rows, e] > -np.inf
        expert[ok, j] = e[ok]
        weight[ok, j] = s[rows, e][ok]
        left[rows, e] = -np.inf
    if c["renormalise"]:
        weight /= weight.sum(axis=1, keepdims=True) + 1e-20
    return (torch.from_numpy(expert), torch.from_numpy(weight * c["scale"]),
            torch.from_numpy(np.repeat(np.arange(T, dtype=np.int32), k)))


def _exact_group(st, c):
    pair = st["chosen"].cpu().numpy().ravel()
    P, E = pair.size, c["experts"]
    cap = min(P, E)
    good = np.flatnonzero((pair >= 0) & (pair < E))
    want = good[np.lexsort((good, pair[good]))]
    ids, first = np.unique(pair[want], return_index=True)
    ge, gb = np.zeros(cap, np.int32), np.zeros(cap + 1, np.int32)
    ge[:ids.size], gb[:ids.size] = ids, first
    gb[ids.size] = want.size
    xrow, order, slot = np.zeros(P, np.int32), np.full(P, -1, np.int32), np.full(P, -1, np.int32)
    xrow[:want.size], order[:want.size] = want // c["top_k"], want
    slot[want] = np.arange(want.size)
    return tuple(torch.from_numpy(a) for a in (ge, gb, xrow, order, slot.reshape(c["tokens"], c["top_k"]), np.array([ids.size], np.int32)))


def _exact_quantize(st, c):
    """The rule is stated in 32-bit operations; here each is carried out in 64 bits and rounded once.  The code is the
    multiple of the step of its power of two (2^-9 below 2^-6) that lies nearest, ties to the even one."""
    x = st["x"].to(torch.float64).view(c["rows"], c["K"] // GROUP, GROUP)
    a = x.abs().max(dim=2, keepdim=True).values.clamp(min=2.0 ** -100)
    factor = (E4M3_MAX / a).float().double()
    v = (x * factor).float().double()
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3.0)
    code = (torch.round(v / step) * step).clamp(-E4M3_MAX, E4M3_MAX)
    return code.view(c["rows"], c["K"]), a.squeeze(2) / E4M3_MAX


def _exact_product(w, w_scale, x, x_scale):
    """Group of 128 by group of 128: exact integer-like sums first, then the two scales."""
    M, K = w.shape
    row_block = torch.arange(M, device=w.device) // GROUP
    total = torch.zeros(x.shape[0], M, dtype=torch.float64, device=w.device)
    for g in range(K // GROUP):
        part = slice(g * GROUP, (g + 1) * GROUP)
        total += (x[:, part].double() @ w[:, part].double().T) * x_scale[:, g].double()[:, None] * w_scale[row_block, g].double()[None, :]
    return total


def exact(case, seed):
    st = prepare(case, seed)
    op = case["op"]
    if op == "route":
        return _exact_route(st, case)
    if op == "group":
        return _exact_group(st, case)
    if op == "quantize":
        return _exact_quantize(st, case)
    if op == "matmul":
        return _exact_product(st["w"], st["w_scale"], st["x"], st["x_scale"])
    if op == "grouped":
        out = torch.zeros(case["tokens"] * case["top_k"], case["M"], dtype=torch.float64, device="cuda")
        begin = st["group_begin"].tolist()
        for g, (expert, _) in enumerate(st["groups"]):
            rows = st["pair_xrow"][begin[g]:begin[g + 1]].long()
            x = st["x"].view(torch.uint8)[rows].view(torch.float8_e4m3fn)
            out[begin[g]:begin[g + 1]] = _exact_product(st["w"][expert], st["w_scale"][expert], x, st["x_scale"][rows])
        return out
    out = torch.zeros(case["tokens"], case["M"], dtype=torch.float64, device="cuda")
    if st["base"] is not None:
        out += st["base"].double()
    for j in range(case["top_k"]):
        slot = st["slot"][:, j].long()
        mine = slot >= 0
        out[mine] += st["y"][slot[mine]].double() * st["weight"][mine, j].double()[:, None]
    return out
