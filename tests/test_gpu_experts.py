"""Around the experts' products: bitcos_route_experts, bitcos_group_pairs_slots, bitcos_combine_pairs against plain
definitions in 64 bits, and a whole routed layer of ternary experts put together from them."""
import numpy as np
import pytest

import datagen
import oracle

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

FLT_MAX = float(np.finfo(np.float32).max)


@pytest.fixture(scope="module")
def bc():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2609_16338_b200 as m
    from paper_2609_16338_b200 import build
    build.build()
    m.load_library()
    return m


def clean(a):
    a = np.asarray(a, np.float64)
    return np.where(np.isnan(a), -np.inf, np.minimum(a, FLT_MAX))


def route_reference(z, bias, score, n_groups, top_groups, group_best, top_k, renormalise, scale):
    """Token by token; returns expert, weight and the largest distance top - z among the taken logits (softmax)."""
    z = clean(z)
    T, E = z.shape
    expert, weight, far = np.full((T, top_k), -1, np.int32), np.zeros((T, top_k)), np.zeros(T)
    b = clean(bias) if bias is not None else np.zeros(E)
    for t in range(T):
        there = np.isfinite(z[t])
        if not there.any():
            continue
        s = np.zeros(E)
        if score == "softmax":
            s[there] = np.exp(z[t, there] - z[t, there].max())
            s /= s.sum()
        else:
            with np.errstate(over="ignore"):
                s[there] = 1.0 / (1.0 + np.exp(-z[t, there]))
        c = np.where(there & np.isfinite(b), s + b, -np.inf)
        n = E // n_groups
        if n_groups > 1:
            value = [np.sort(c[g * n:(g + 1) * n])[::-1][:group_best].sum() for g in range(n_groups)]
            kept = sorted(range(n_groups), key=lambda g: (-value[g], g))[:top_groups]
            c = np.where(np.isin(np.arange(E) // n, kept), c, -np.inf)
        # without sums of two the order is that of the logits (scores of distinct logits are distinct)
        rank = z[t] if bias is None and (n_groups == 1 or group_best == 1) else c
        taken = [e for e in sorted(range(E), key=lambda e: (-rank[e], e)) if np.isfinite(c[e])][:top_k]
        expert[t, :len(taken)] = taken
        w = s[taken]
        if renormalise:
            w = w / (w.sum() + 1e-20)
        weight[t, :len(taken)] = w * scale
        if taken and score == "softmax":
            far[t] = min(z[t, there].max() - z[t, taken].min(), 104.0)
    return expert, weight, far


def check_route(bc, logits, bias=None, **kw):
    kw = {**dict(score="softmax", n_groups=1, top_groups=1, group_best=1, renormalise=True, scale=1.0), **kw}
    top_k = kw.pop("top_k")
    expert, weight, xrow = bc.bitcos_route_experts(logits, top_k, bias=None if bias is None else torch.from_numpy(bias).cuda(), **kw)
    want, w_ref, far = route_reference(logits.float().cpu().numpy(), bias, top_k=top_k, **kw)
    T = logits.shape[0]
    assert np.array_equal(expert.cpu().numpy(), want)
    assert np.array_equal(xrow.cpu().numpy(), np.repeat(np.arange(T, dtype=np.int32), top_k))
    # score: exp, sum and quotient within 2^-20, the exponent's rounding far * 2^-24 (bound doubled); once more in the sum that
    # divides, whose up to 32 additions, quotient and scale round by 2^-24 each; scores under the normal range count as nothing
    rel = 2 * (2.0 ** -20 + far * 2.0 ** -23) + 36 * 2.0 ** -24
    got = weight.cpu().numpy().astype(np.float64)
    assert (np.abs(got - w_ref) <= rel[:, None] * np.abs(w_ref) + 1e-17 * kw["scale"]).all()
    return expert, weight


@pytest.mark.parametrize("tokens,experts,top_k,dtype", [(1, 1, 1, "float32"), (1, 128, 8, "float32"), (5, 31, 4, "bfloat16"), (33, 33, 8, "float16"),
                                                        (7, 64, 32, "bfloat16"), (3, 3, 8, "float32"), (1000, 256, 8, "bfloat16"),
                                                        (17, 500, 5, "float16"), (9, 1024, 8, "float32"), (6, 1000, 31, "bfloat16")])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("with_bias", [False, True])
def test_route(bc, tokens, experts, top_k, dtype, score, with_bias):
    """Sizes around the lanes' runs of experts; 16-bit logits tie often, and ties go to the lower index."""
    rng = np.random.default_rng(tokens * 7 + experts)
    z = torch.from_numpy(rng.normal(0, 2, (tokens, experts)).astype(np.float32)).cuda().to(getattr(torch, dtype))
    bias = (rng.random(experts).astype(np.float32) - 0.5) * 0.2 if with_bias else None
    check_route(bc, z, bias, top_k=top_k, score=score)
    check_route(bc, z, bias, top_k=top_k, score=score, renormalise=False, scale=2.5)


@pytest.mark.parametrize("experts,n_groups,top_groups", [(256, 8, 4), (256, 8, 1), (64, 4, 4), (60, 4, 2), (96, 32, 5), (160, 5, 3), (1024, 32, 7),
                                                         (512, 2, 1)])
@pytest.mark.parametrize("group_best", [1, 2])
@pytest.mark.parametrize("with_bias", [False, True])
def test_route_by_groups(bc, experts, n_groups, top_groups, group_best, with_bias):
    rng = np.random.default_rng(experts + n_groups)
    z = torch.from_numpy(rng.normal(0, 1.5, (50, experts)).astype(np.float32)).cuda().to(torch.bfloat16)
    bias = (rng.random(experts).astype(np.float32) - 0.5) * 0.3 if with_bias else None
    for score in ("softmax", "sigmoid"):
        check_route(bc, z, bias, top_k=8, score=score, n_groups=n_groups, top_groups=top_groups, group_best=group_best)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("with_bias", [False, True])
def test_route_masks_and_infinities(bc, score, with_bias):
    """Rows whose mask leaves nothing, one, fewer than top_k; NaN; +inf; the type's lowest value; -0 beside 0; a masked bias."""
    E, lowest = 40, float(np.finfo(np.float32).min)
    rng = np.random.default_rng(3)
    z = rng.normal(0, 1, (12, E)).astype(np.float32)
    z[0] = -np.inf
    z[1] = np.nan
    z[2] = -np.inf
    z[2, 17] = 0.5
    z[3, 5:] = -np.inf
    z[4, ::3] = np.nan
    z[5, 7] = z[5, 30] = np.inf
    z[6] = lowest
    z[7, 10:] = lowest
    z[8] = 0.0
    z[8, ::2] = -0.0
    z[9] = -300.0
    z[10, 4:] = -200.0
    z[11] = 90.0
    bias = None
    if with_bias:
        bias = (rng.random(E).astype(np.float32) - 0.5) * 0.1
        bias[3], bias[9], bias[20] = -np.inf, np.nan, np.inf
    for dtype in (torch.float32, torch.bfloat16):
        check_route(bc, torch.from_numpy(z).cuda().to(dtype), bias, top_k=8, score=score)
        check_route(bc, torch.from_numpy(z).cuda().to(dtype), bias, top_k=8, score=score, n_groups=4, top_groups=2, group_best=2)


def test_route_orders_that_32_bits_cannot_tell(bc):
    """Choices that differ by less than a rounding of 32 bits, at the border of the taken ones, inside their order, and
    between groups: 64 bits decide.  Biases step by one unit in the last place at 1, the scores move against them."""
    E = 64
    rng = np.random.default_rng(11)
    bias = (1.0 + rng.integers(-3, 4, E) * 2.0 ** -23).astype(np.float32)
    z = (rng.normal(0, 1e-6, (200, E)) - 3.0).astype(np.float32)
    check_route(bc, torch.from_numpy(z).cuda(), bias, top_k=8, score="sigmoid")
    check_route(bc, torch.from_numpy(z).cuda(), bias, top_k=8, score="softmax")
    check_route(bc, torch.from_numpy(z).cuda(), bias, top_k=8, score="sigmoid", n_groups=8, top_groups=3, group_best=2)
    check_route(bc, torch.from_numpy(z).cuda(), None, top_k=8, score="sigmoid", n_groups=8, top_groups=3, group_best=2)
    # more candidates at the border than a warp has lanes, and as many places as lanes
    check_route(bc, torch.from_numpy(z).cuda(), bias, top_k=32, score="sigmoid")
    wide = (rng.normal(0, 1e-6, (50, 300)) - 3.0).astype(np.float32)
    level = np.ones(300, np.float32)
    for top_k in (1, 8, 32):
        check_route(bc, torch.from_numpy(wide).cuda(), level, top_k=top_k, score="sigmoid")
        check_route(bc, torch.from_numpy(wide).cuda(), level, top_k=top_k, score="softmax")
    # 32-bit logits without a bias, one unit in the last place apart
    step = np.float32(1.0) + rng.permuted(np.tile(np.arange(500, dtype=np.float32), (40, 1)), axis=1) * np.float32(2.0 ** -23)
    check_route(bc, torch.from_numpy(step).cuda(), None, top_k=8)
    check_route(bc, torch.from_numpy(-step).cuda(), None, top_k=32, n_groups=4, top_groups=2)
    # equal logits and equal biases: the lower index
    check_route(bc, torch.zeros(3, E, device="cuda"), np.zeros(E, np.float32), top_k=8, score="sigmoid")


def test_route_strided_rows_and_nothing(bc):
    z = torch.randn(20, 300, device="cuda")
    check_route(bc, z[:, 3:131], top_k=8)
    check_route(bc, z[::2, :128], top_k=8)
    check_route(bc, z[4:5, 7:135], top_k=8)
    expert, weight, xrow = bc.bitcos_route_experts(torch.empty(0, 128, device="cuda"), 8)
    assert expert.shape == (0, 8) and weight.shape == (0, 8) and xrow.shape == (0,)


def test_route_the_largest_grid(bc):
    """More tokens than a grid of 65535 blocks of four; every token checked by its own properties."""
    T, E = 300_001, 16
    z = torch.randn(T, E, device="cuda")
    expert, weight, xrow = bc.bitcos_route_experts(z, 2, renormalise=False)
    order = z.sort(dim=1, descending=True, stable=True)
    assert torch.equal(expert, order.indices[:, :2].to(torch.int32))
    p = torch.softmax(z.double(), 1).gather(1, expert.long())
    assert ((weight.double() - p).abs() <= p * 2.0 ** -18).all()
    assert torch.equal(xrow, torch.arange(T, dtype=torch.int32, device="cuda").repeat_interleave(2))


def group_reference(pe, top_k, experts):
    P = pe.size
    kept = np.flatnonzero((pe >= 0) & (pe < experts))
    want = kept[np.argsort(pe[kept], kind="stable")]
    ids, first = np.unique(pe[want], return_index=True)
    cap = min(P, experts)
    ge, gb = np.zeros(cap, np.int32), np.zeros(cap + 1, np.int32)
    ge[:ids.size], gb[:ids.size], gb[ids.size] = ids, first, want.size
    xr, order, slot = np.zeros(P, np.int32), np.full(P, -1, np.int32), np.full(P, -1, np.int32)
    xr[:want.size], order[:want.size], slot[want] = want // top_k, want, np.arange(want.size)
    return ge, gb, xr, order, slot, ids.size


@pytest.mark.parametrize("tokens,top_k,experts,bad", [(1, 1, 1, 0), (1, 8, 1024, 0), (31, 1, 3, 0), (11, 3, 128, 5), (16, 8, 128, 0), (257, 1, 5, 40),
                                                      (512, 8, 1024, 100), (4096, 1, 7, 4096), (4097, 1, 33, 1), (1000, 7, 1024, 70),
                                                      (20000, 8, 128, 1000), (150000, 2, 1, 3), (33333, 3, 256, 99999), (40000, 8, 1000, 0)])
def test_pairs_of_any_number_grouped(bc, tokens, top_k, experts, bad):
    """One block and many; one expert; all pairs left out; remainders of warps, runs and blocks."""
    rng = np.random.default_rng(tokens + experts)
    P = tokens * top_k
    pe = rng.integers(0, experts, P).astype(np.int32)
    pe[rng.permutation(P)[:bad]] = rng.choice(np.array([-1, experts, 1 << 20, -(1 << 31)], np.int64), bad).astype(np.int32)
    ws = bc.make_group_workspace(P, experts)
    ws.random_(0, 255)
    out = bc.bitcos_group_pairs_slots(torch.from_numpy(pe).cuda().view(tokens, top_k), experts, workspace=ws)
    ge, gb, xr, order, slot, ng = (t.cpu().numpy() for t in out)
    ref = group_reference(pe, top_k, experts)
    assert int(ng[0]) == ref[5]
    for got, want in zip((ge, gb, xr, order, slot.ravel()), ref):
        assert np.array_equal(got, want)


@pytest.mark.parametrize("tokens,top_k,M,y_type,out_type,base", [(1, 1, 1, "float32", "float32", False), (5, 8, 2048, "float32", "float32", True),
                                                                 (7, 3, 2047, "bfloat16", "float32", True), (3, 8, 1026, "bfloat16", "bfloat16", False),
                                                                 (300, 9, 72, "bfloat16", "bfloat16", True), (64, 17, 68, "float32", "bfloat16", True),
                                                                 (2, 40, 4095, "float32", "bfloat16", False)])
def test_combine(bc, tokens, top_k, M, y_type, out_type, base):
    """Whole and odd columns, more places than a batch of loads, places without a row (also out of range ones), NaN in rows that
    nobody asks for and in rows of weight-bearing places that are left out."""
    gen = torch.Generator(device="cuda").manual_seed(tokens + M)
    rows = tokens * top_k + 3
    y = torch.randn(rows, M, generator=gen, device="cuda").to(getattr(torch, y_type))
    slot = torch.randperm(rows, generator=gen, device="cuda")[:tokens * top_k].to(torch.int32).view(tokens, top_k)
    drop = torch.rand(tokens, top_k, generator=gen, device="cuda") < 0.2
    y[slot[drop].long()] = float("nan")
    slot[drop] = torch.tensor([-1, rows, 1 << 30, -(1 << 31)], device="cuda")[torch.arange(int(drop.sum()), device="cuda") % 4].to(torch.int32)
    weight = torch.randn(tokens, top_k, generator=gen, device="cuda")
    b = torch.randn(tokens, M, generator=gen, device="cuda").to(getattr(torch, out_type)) if base else None
    out = bc.bitcos_combine_pairs(y, slot, weight, base=b, out_dtype=getattr(torch, out_type))
    use = torch.where(drop, 0, slot).long()
    terms = torch.where(drop[..., None], 0.0, y[use].double() * weight[..., None].double())
    want, mag = terms.sum(1), terms.abs().sum(1)
    if base:
        want, mag = want + b.double(), mag + b.double().abs()
    # top_k + 1 multiply-adds of half a unit each, relative to the sum of magnitudes; then the output's rounding
    bound = mag * (top_k + 1) * 2.0 ** -24 + (want.abs() * (1 + 2.0 ** -20) * 2.0 ** -8 if out_type == "bfloat16" else 0.0) + 1e-40
    assert out.dtype == getattr(torch, out_type) and ((out.double() - want).abs() <= bound).all()
    if base:      # in place
        again = b.clone()
        assert bc.bitcos_combine_pairs(y, slot, weight, base=again, out=again) is again and torch.equal(again, out)


def test_combine_rows_behind_32_bits(bc):
    """A y of more than 2^31 elements: the last rows are found."""
    M, rows = 65536, 33000
    y = torch.zeros(rows, M, dtype=torch.bfloat16, device="cuda")
    y[-1], y[-2], y[17] = 1.0, 2.0, 4.0
    slot = torch.tensor([[rows - 1, rows - 2, 17]], dtype=torch.int32, device="cuda")
    weight = torch.tensor([[1.0, 10.0, 100.0]], device="cuda")
    assert (bc.bitcos_combine_pairs(y, slot, weight, out_dtype=torch.float32) == 421.0).all()


def test_a_routed_layer_of_ternary_experts_captured(bc):
    """Logits -> experts -> groups -> the grouped ternary product -> the weighted sum, recorded once and replayed with other
    logits and activations: the pairs never leave the device."""
    M, K, E, T, k = 256, 512, 12, 16, 4
    Ws, Ss = [datagen.trits(80 + e, M, K, 0.33) for e in range(E)], [datagen.scales(80 + e, M, K) for e in range(E)]
    X = bc.DeviceExperts([bc.bitcos_pack(Ws[e], Ss[e]).to_device() for e in range(E)])
    logits = torch.empty(T, E, device="cuda")
    x, xs = torch.empty(T, K, dtype=torch.int8, device="cuda"), torch.empty(T, device="cuda")
    residual = torch.empty(T, M, device="cuda")
    ws, gws = bc.make_workspace(M, K, copies=E), bc.make_group_workspace(T * k, E)

    def layer():
        expert, weight, _ = bc.bitcos_route_experts(logits, k)
        ge, gb, xr, order, slot, ng = bc.bitcos_group_pairs_slots(expert, E, workspace=gws)
        y, _ = bc.bitcos_gemv_grouped_lists(X, ge, gb, ng, xr, T, x, xs, workspace=ws)
        return bc.bitcos_combine_pairs(y, slot, weight, base=residual), expert, weight

    def fill(seed):
        rng = np.random.default_rng(seed)
        a, s = datagen.activations(seed, T, K)
        z = rng.normal(0, 1, (T, E)).astype(np.float32)
        z[3, 2:] = -np.inf                       # two experts left for four places
        z[7] = -np.inf                           # none
        for dst, src in ((logits, z), (x, a), (xs, s), (residual, rng.normal(0, 1, (T, M)).astype(np.float32))):
            dst.copy_(torch.from_numpy(src))
        return a, s

    fill(1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            out, expert, weight = layer()
    torch.cuda.synchronize()
    for seed in (2, 3):
        a, s = fill(seed)
        graph.replay()
        torch.cuda.synchronize()
        pe, w = expert.cpu().numpy(), weight.cpu().numpy().astype(np.float64)
        assert (pe[3] >= 0).sum() == 2 and (pe[7] == -1).all() and (w[7] == 0).all()
        t, j = np.nonzero(pe >= 0)
        _, y_ref, mag = oracle.grouped_dense(Ws, Ss, pe[t, j], t.astype(np.int32), a, s)
        want, size = residual.cpu().numpy().astype(np.float64), np.abs(residual.cpu().numpy()).astype(np.float64)
        np.add.at(want, t, y_ref * w[t, j][:, None])
        np.add.at(size, t, mag * w[t, j][:, None])
        # the product's 1e-5 of its magnitudes, then five multiply-adds
        assert (np.abs(out.cpu().numpy() - want) <= size * (1e-5 + 6 * 2.0 ** -24)).all()
        assert bc.workspace_status(ws) == 0


def test_calls_on_another_stream_and_refusals(bc):
    z = torch.randn(64, 128, device="cuda")
    want = bc.bitcos_route_experts(z, 8)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = bc.bitcos_route_experts(z, 8)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    with pytest.raises(ValueError):
        bc.bitcos_route_experts(z.cpu(), 8)
    with pytest.raises(ValueError):
        bc.bitcos_route_experts(z.double(), 8)
    with pytest.raises(ValueError):
        bc.bitcos_route_experts(z.t(), 8)
    with pytest.raises(bc.BitcosError):
        bc.bitcos_route_experts(z, 8, n_groups=3)
    with pytest.raises(bc.BitcosError):
        bc.bitcos_route_experts(z[:1].expand(4, 128), 8)
    y = torch.randn(6, 16, device="cuda")
    slot, w = torch.zeros(2, 3, dtype=torch.int32, device="cuda"), torch.ones(2, 3, device="cuda")
    with pytest.raises(ValueError):
        bc.bitcos_combine_pairs(y, slot, w.double())
    with pytest.raises(ValueError):
        bc.bitcos_combine_pairs(y.t(), slot, w)
    with pytest.raises(ValueError):
        bc.bitcos_combine_pairs(y, slot, w, base=torch.zeros(2, 15, device="cuda"))
    with pytest.raises(bc.BitcosError):
        bc.bitcos_group_pairs_slots(slot, 8, workspace=torch.empty(0, dtype=torch.uint8, device="cuda"))
