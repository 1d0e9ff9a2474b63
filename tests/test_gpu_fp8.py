"""e4m3: the quantiser against its rule carried out in 64 bits, the products against their definition in 64 bits.

Bound on a product's fp32 output, relative to the sum of |terms|: products of two e4m3 codes are exact; a step of the tensor
core adds 32 of them to the accumulator, and if each of the 33 addends loses less than a unit of 2^-24 of the largest, the four steps of a
group lose 132 * 2^-24; then two products with scales, and one addition per group, round by 2^-24 each."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

GROUP = 128


@pytest.fixture(scope="module")
def bc():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2609_16338_b200 as m
    from paper_2609_16338_b200 import build
    build.build()
    m.load_library()
    return m


# ------------------------------------------------------------------ quantiser
def quantize_reference(x):
    """Every operation of the rule in 64 bits, rounded to 32 (a quotient or product of two 32-bit numbers rounds there
    as the 32-bit operation does); the code is the nearest multiple of its step, ties to even."""
    rows, K = x.shape
    g = x.astype(np.float64).reshape(rows, K // GROUP, GROUP)
    a = np.maximum(np.abs(g).max(2, keepdims=True), 2.0 ** -100)
    factor = (448.0 / a).astype(np.float32).astype(np.float64)
    v = (g * factor).astype(np.float32).astype(np.float64)
    step = 2.0 ** (np.floor(np.log2(np.maximum(np.abs(v), 2.0 ** -6))) - 3)
    code = np.clip(np.rint(v / step) * step, -448, 448)
    return code.reshape(rows, K), (a[..., 0] / 448.0).astype(np.float32)


@pytest.mark.parametrize("rows,K", [(1, 128), (3, 384), (7, 2560), (65, 640), (1000, 256)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_quantize(bc, rows, K, dtype):
    rng = np.random.default_rng(rows + K)
    x = rng.normal(0, 1, (rows, K)).astype(np.float32) * np.exp(rng.normal(0, 3, (rows, 1))).astype(np.float32)
    x[0, :128] = 0.0
    x[-1, ::3] *= 1e-3
    x[0, -5:] = [448.0, 2.0 ** -9, 2.0 ** -10, 3 * 2.0 ** -10, -17.0]        # (the last group's factor is 1: ties and the subnormal range)
    x[0, -128:-5] = np.clip(x[0, -128:-5], -400, 400)
    if K > 128:
        x[-1, :128] = 1e-36 * rng.normal(0, 1, 128)                           # under the floor
    xd = torch.from_numpy(x).cuda().to(getattr(torch, dtype))
    q, s = bc.bitcos_fp8_quantize(xd)
    code, scale = quantize_reference(xd.float().cpu().numpy())
    assert np.array_equal(q.float().cpu().numpy(), code.astype(np.float32))
    assert np.array_equal(s.cpu().numpy(), scale)


def test_quantize_nothing_and_more_groups_than_one_grid_row(bc):
    q, s = bc.bitcos_fp8_quantize(torch.empty(0, 256, device="cuda"))
    assert q.shape == (0, 256) and s.shape == (0, 2)
    x = torch.randn(70000, 8192, device="cuda").to(torch.bfloat16)            # 4.48 million groups, 70000 blocks; bytes 0 .. 2^29
    q, s = bc.bitcos_fp8_quantize(x)
    assert torch.equal(s, x.float().abs().view(70000, 64, 128).amax(2) / torch.full((1,), 448.0, device="cuda"))
    last = x[-1:].contiguous()
    q1, s1 = bc.bitcos_fp8_quantize(last)
    assert torch.equal(q1.view(torch.uint8), q[-1:].view(torch.uint8)) and torch.equal(s1, s[-1:])


# ------------------------------------------------------------------ products
def weights(count, M, K, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    w = torch.randn(count, M, K, generator=gen, device="cuda") * 60.0
    codes = w.clamp(-448, 448).to(torch.float8_e4m3fn)
    scales = torch.exp(torch.randn(count, (M + GROUP - 1) // GROUP, K // GROUP, generator=gen, device="cuda"))
    return codes, scales


def activations(rows, K, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed + 1)
    x = (torch.randn(rows, K, generator=gen, device="cuda") * 60.0).clamp(-448, 448).to(torch.float8_e4m3fn)
    return x, torch.exp(torch.randn(rows, K // GROUP, generator=gen, device="cuda"))


def product_reference(w, ws, x, xs):
    M, K = w.shape
    block = torch.arange(M, device="cuda") // GROUP
    total, mag = (torch.zeros(x.shape[0], M, dtype=torch.float64, device="cuda") for _ in range(2))
    for g in range(K // GROUP):
        part = slice(g * GROUP, (g + 1) * GROUP)
        f = xs[:, g].double()[:, None] * ws[block, g].double()[None, :]
        total += (x[:, part].double() @ w[:, part].double().T) * f
        mag += (x[:, part].double().abs() @ w[:, part].double().abs().T) * f
    return total, mag


def check(y, total, mag, G):
    bound = mag * ((132 + G + 4) * 2.0 ** -24)
    if y.dtype == torch.bfloat16:
        bound = bound * (1 + 2.0 ** -8) + total.abs() * 2.0 ** -8
    assert ((y.double() - total).abs() <= bound).all(), float(((y.double() - total).abs() / bound.clamp_min(1e-300)).max())


# one row to long prompts; odd rows and odd M; K of one group; every operand order and width; K cut over a cluster and not
SHAPES = [(1, 128, 128), (1, 1, 128), (1, 2560, 2560), (2, 33, 384), (5, 640, 2560), (16, 6912, 2560), (15, 1000, 25600), (17, 300, 1024),
          (31, 2049, 640), (32, 25600, 256), (33, 129, 5120), (64, 2560, 6912), (63, 640, 128), (65, 641, 640), (127, 257, 2560), (128, 5120, 512),
          (129, 200, 256), (300, 2560, 2560), (1000, 2561, 640), (2000, 2304, 768), (4097, 1153, 128), (511, 8200, 384), (9000, 10, 256)]


@pytest.mark.parametrize("rows,M,K", SHAPES)
@pytest.mark.parametrize("out", ["float32", "bfloat16"])
def test_matmul(bc, rows, M, K, out):
    w, ws = weights(1, M, K, rows + M)
    x, xs = activations(rows, K, rows + K)
    W, space = bc.Fp8Weights(w[0], ws[0]), bc.make_fp8_workspace()
    room = torch.full((rows + 3, M), 7.0, dtype=getattr(torch, out), device="cuda")      # rows behind the last: left as they were
    y = bc.bitcos_fp8_matmul(W, x, xs, y=room[:rows], workspace=space)
    total, mag = product_reference(w[0], ws[0], x, xs)
    check(y, total, mag, K // GROUP)
    assert (room[rows:] == 7.0).all()
    assert bc.workspace_status(space) == 0
    assert torch.equal(y, bc.bitcos_fp8_matmul(W, x, xs, out_dtype=getattr(torch, out)))      # the same bits, without a workspace


def test_matmul_extremes(bc):
    """Codes of the whole range beside one another (the smallest under the largest), NaN codes, infinite and zero scales: what
    the formula gives, confined to the rows and columns they belong to."""
    rows, M, K = 20, 384, 512
    gen = torch.Generator(device="cuda").manual_seed(5)
    bits = torch.randint(0, 256, (M + rows, K), generator=gen, device="cuda", dtype=torch.uint8)
    bits[(bits & 0x7F) == 0x7F] = 0x01
    w, x = bits[:M].view(torch.float8_e4m3fn).contiguous(), bits[M:].view(torch.float8_e4m3fn).contiguous()
    ws, xs = torch.rand(3, 4, generator=gen, device="cuda") + 0.5, torch.rand(rows, 4, generator=gen, device="cuda") + 0.5
    ws[1, 2] = 0.0
    total, mag = product_reference(w, ws, x, xs)
    for n in (rows, 1):
        check(bc.bitcos_fp8_matmul(bc.Fp8Weights(w, ws), x[:n], xs[:n]), total[:n], mag[:n], 4)
    xb, xsb = x.clone(), xs.clone()
    xb.view(torch.uint8)[3, 100] = 0x7F           # NaN
    xsb[7, 1] = float("inf")
    wb = w.clone()
    wb.view(torch.uint8)[200, 300] = 0xFF
    y = bc.bitcos_fp8_matmul(bc.Fp8Weights(wb, ws), xb, xsb)
    good = torch.ones(rows, M, dtype=torch.bool, device="cuda")
    good[3], good[7], good[:, 200] = False, False, False
    assert torch.isnan(y[3]).all() and torch.isnan(y[:, 200]).all()
    assert (~torch.isfinite(y[7])).all()
    assert torch.equal(y[good], bc.bitcos_fp8_matmul(bc.Fp8Weights(w, ws), x, xs)[good])


def test_matmul_outputs_behind_32_bits(bc):
    """rows * M over 2^31 elements: the last rows and columns against the same product of these rows alone."""
    rows, M, K = 16400, 131072 + 8, 128
    w, ws = weights(1, M, K, 1)
    x, xs = activations(rows, K, 2)
    y = bc.bitcos_fp8_matmul(bc.Fp8Weights(w[0], ws[0]), x, xs, out_dtype=torch.bfloat16)
    for r in (0, 9001, 16383, 16399):
        total, mag = product_reference(w[0], ws[0], x[r:r + 1], xs[r:r + 1])
        check(y[r:r + 1], total, mag, 1)


def routed(tokens, top_k, experts, seed, dead=()):
    """Pairs grouped by expert on the host: group_expert, group_begin, n_groups, pair_xrow and the groups' lengths."""
    rng = np.random.default_rng(seed)
    pe = np.concatenate([rng.permutation(experts)[:top_k] for _ in range(tokens)]).astype(np.int32)
    pe[np.isin(pe, dead)] = -1
    kept = np.flatnonzero(pe >= 0)
    order = kept[np.argsort(pe[kept], kind="stable")]
    ids, first, count = np.unique(pe[order], return_index=True, return_counts=True)
    cap = min(tokens * top_k, experts)
    ge, gb, xr = np.zeros(cap, np.int32), np.zeros(cap + 1, np.int32), np.zeros(tokens * top_k, np.int32)
    ge[:ids.size], gb[:ids.size], gb[ids.size], xr[:order.size] = ids, first, order.size, order // top_k
    dev = [torch.from_numpy(a).cuda() for a in (ge, gb, np.array([ids.size], np.int32), xr)]
    return dev, list(zip(ids.tolist(), first.tolist(), count.tolist()))


GROUPED = [(1, 1, 1, 128, 128), (1, 8, 128, 768, 2048), (8, 8, 128, 768, 2048), (16, 8, 32, 2048, 768), (5, 3, 7, 100, 384), (100, 4, 12, 257, 640),
           (60, 8, 16, 384, 256), (200, 8, 32, 1000, 128), (700, 2, 16, 512, 256), (513, 3, 5, 1153, 384), (2048, 8, 64, 256, 256),
           (33, 1, 1, 640, 2560), (300, 1, 1, 640, 640)]


@pytest.mark.parametrize("tokens,top_k,experts,M,K", GROUPED)
@pytest.mark.parametrize("out", ["float32", "bfloat16"])
def test_grouped(bc, tokens, top_k, experts, M, K, out):
    """Groups from one pair to more than a tile; rows gathered; rows of y behind the last group left as they were."""
    w, ws = weights(experts, M, K, tokens + M)
    x, xs = activations(tokens, K, tokens + K)
    (ge, gb, ng, xr), groups = routed(tokens, top_k, experts, tokens + experts, dead=(3, 4) if experts > 8 else ())
    W, space = bc.Fp8Weights(w, ws), bc.make_fp8_workspace()
    y = torch.full((tokens * top_k, M), 7.0, dtype=getattr(torch, out), device="cuda")
    bc.bitcos_fp8_matmul_grouped(W, ge, gb, ng, xr, x, xs, y=y, workspace=space)
    for e, begin, count in groups:
        rows = xr[begin:begin + count].long()
        total, mag = product_reference(w[e], ws[e], x.view(torch.uint8)[rows].view(torch.float8_e4m3fn), xs[rows])
        check(y[begin:begin + count], total, mag, K // GROUP)
    last = groups[-1][1] + groups[-1][2] if groups else 0
    assert (y[last:] == 7.0).all()
    assert bc.workspace_status(space) == 0
    # without a row list: pair p reads row p, the same rows written out
    flat = x.view(torch.uint8)[xr.long()].view(torch.float8_e4m3fn).contiguous()
    z = torch.full_like(y, 7.0)
    bc.bitcos_fp8_matmul_grouped(W, ge, gb, ng, None, flat, xs[xr.long()].contiguous(), y=z, workspace=space)
    assert torch.equal(y, z)


@pytest.mark.parametrize("tokens,top_k,experts,K", [(24, 4, 12, 256), (600, 4, 12, 256), (5, 7, 12, 1024), (100, 6, 12, 128)])
def test_grouped_malformed_lists_are_skipped(bc, tokens, top_k, experts, K):
    """A group that names no expert, one that ends behind the pairs, one that begins below them, one pair whose row does not exist, an
    empty group in between, more groups than there is room for: nothing of the bad ones is written, the rest is as it was."""
    M = 384
    w, ws = weights(experts, M, K, 9)
    x, xs = activations(tokens, K, 9)
    (ge, gb, ng, xr), groups = routed(tokens, top_k, experts, 9)
    W, space = bc.Fp8Weights(w, ws), bc.make_fp8_workspace()
    want = torch.full((tokens * top_k, M), 7.0, device="cuda")
    bc.bitcos_fp8_matmul_grouped(W, ge, gb, ng, xr, x, xs, y=want, workspace=space)
    assert bc.workspace_status(space) == 0
    P = tokens * top_k

    def run(ge, gb, ng, xr):
        y = torch.full_like(want, 7.0)
        space.zero_()
        bc.bitcos_fp8_matmul_grouped(W, ge, gb, ng, xr, x, xs, y=y, workspace=space)
        return y, bc.workspace_status(space)

    for bad in (-1, experts, 1 << 30):
        g2, w2 = ge.clone(), want.clone()
        g2[5] = bad
        w2[groups[5][1]:groups[5][1] + groups[5][2]] = 7.0
        y, status = run(g2, gb, ng, xr)
        assert torch.equal(y, w2) and status == 2
    b2, w2 = gb.clone(), want.clone()
    b2[len(groups)] = P + 1
    w2[groups[-1][1]:] = 7.0
    y, status = run(ge, b2, ng, xr)
    assert torch.equal(y, w2) and status == 2
    b2, w2 = gb.clone(), want.clone()
    b2[0] = -1
    w2[:groups[1][1]] = 7.0
    y, status = run(ge, b2, ng, xr)
    assert torch.equal(y, w2) and status == 2
    for bad in (-1, tokens, 1 << 30):
        x2, w2 = xr.clone(), want.clone()
        x2[groups[2][1] + 1] = bad
        w2[groups[2][1] + 1] = 7.0
        y, status = run(ge, gb, ng, x2)
        assert torch.equal(y, w2) and status == 2
    # group 4 gives its pairs to group 3's end: group 4 is empty
    b2 = gb.clone()
    b2[4] = b2[5]
    y, status = run(ge, b2, ng, xr)
    assert status == 0 and torch.equal(y[:groups[4][1]], want[:groups[4][1]]) and torch.equal(y[groups[5][1]:], want[groups[5][1]:])
    y, status = run(ge, gb, ng + 1000, xr)
    assert torch.equal(y, want) and status == 0
    for none in (0, -5):
        y, status = run(ge, gb, torch.full_like(ng, none), xr)
        assert (y == 7.0).all() and status == 0


def test_other_stream_graph_and_chain(bc):
    """Quantise, multiply, quantise, multiply on a stream of its own and replayed from a graph: each kernel waits for the one before."""
    K, M = 2560, 640
    w1, s1 = weights(1, M, K, 1)
    w2, s2 = weights(1, K, M, 2)
    W1, W2 = bc.Fp8Weights(w1[0], s1[0]), bc.Fp8Weights(w2[0], s2[0])
    for rows in (1, 40, 700):
        x = torch.empty(rows, K, device="cuda")

        def chain():
            q, s = bc.bitcos_fp8_quantize(x)
            h = bc.bitcos_fp8_matmul(W1, q, s, out_dtype=torch.bfloat16)
            q, s = bc.bitcos_fp8_quantize(h)
            return q, s, bc.bitcos_fp8_matmul(W2, q, s)

        x.normal_()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            chain()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                q, s, y = chain()
        for _ in range(3):
            x.normal_()
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            h = bc.bitcos_fp8_matmul(W1, *bc.bitcos_fp8_quantize(x), out_dtype=torch.bfloat16)
            qr, sr = bc.bitcos_fp8_quantize(h)
            torch.cuda.synchronize()
            assert torch.equal(q.view(torch.uint8), qr.view(torch.uint8)) and torch.equal(s, sr)
            total, mag = product_reference(w2[0], s2[0], q, s)
            check(y, total, mag, M // GROUP)


def test_a_routed_layer_of_8_bit_experts(bc):
    """Router, grouping, gate and up, activation, down, weighted sum: a prompt through an 8-bit mixture of experts, pairs and rows on the
    device throughout, and the same layer for one token."""
    H, F, E, k = 512, 256, 16, 4
    wu, su = weights(E, 2 * F, H, 3)
    wd, sd = weights(E, H, F, 4)
    U, D = bc.Fp8Weights(wu, su * 1e-3), bc.Fp8Weights(wd, sd * 1e-3)
    gen = torch.Generator(device="cuda").manual_seed(8)
    for T in (1, 300):
        x = torch.randn(T, H, generator=gen, device="cuda").to(torch.bfloat16)
        logits = torch.randn(T, E, generator=gen, device="cuda")
        expert, weight, _ = bc.bitcos_route_experts(logits, k, score="sigmoid", bias=torch.zeros(E, device="cuda"))
        ge, gb, xr, order, slot, ng = bc.bitcos_group_pairs_slots(expert, E)
        q, s = bc.bitcos_fp8_quantize(x)
        space = bc.make_fp8_workspace()
        h = bc.bitcos_fp8_matmul_grouped(U, ge, gb, ng, xr, q, s, workspace=space)
        a = torch.nn.functional.silu(h[:, :F]) * h[:, F:]
        qa, sa = bc.bitcos_fp8_quantize(a)
        y = bc.bitcos_fp8_matmul_grouped(D, ge, gb, ng, None, qa, sa, workspace=space)
        out = bc.bitcos_combine_pairs(y, slot, weight, base=x.float())
        assert bc.workspace_status(space) == 0
        # token by token from the same codes: the second product in 64 bits, then the sum
        want, size = x.double(), x.double().abs()
        for t in range(0, T, 37):
            for j in range(k):
                p, e = int(slot[t, j]), int(expert[t, j])
                total, mag = product_reference(wu[e], U.scales[e], q[t:t + 1], s[t:t + 1])
                check(h[p:p + 1], total, mag, H // GROUP)
                total, mag = product_reference(wd[e], D.scales[e], qa[p:p + 1], sa[p:p + 1])
                want[t] += total[0] * weight[t, j].double()
                size[t] += mag[0] * weight[t, j].double()
            bound = size[t] * ((132 + F // GROUP + 4 + k + 1) * 2.0 ** -24)
            assert ((out[t].double() - want[t]).abs() <= bound).all()


def test_python_refusals(bc):
    w, ws = weights(2, 256, 256, 1)
    x, xs = activations(4, 256, 1)
    W, E = bc.Fp8Weights(w[0], ws[0]), bc.Fp8Weights(w, ws)
    one = torch.zeros(2, dtype=torch.int32, device="cuda")
    for bad in (lambda: bc.Fp8Weights(w[0].float(), ws[0]), lambda: bc.Fp8Weights(w[0], ws[0, :1]), lambda: bc.Fp8Weights(w[0, :, :64].contiguous(), ws[0]),
                lambda: bc.Fp8Weights(w[0], ws[0].cpu()),
                lambda: bc.bitcos_fp8_matmul(W, x.float(), xs), lambda: bc.bitcos_fp8_matmul(W, x[:, :128].contiguous(), xs),
                lambda: bc.bitcos_fp8_matmul(W, x, xs[:, :1]), lambda: bc.bitcos_fp8_matmul(W, x, xs[:3]), lambda: bc.bitcos_fp8_matmul(E, x, xs),
                lambda: bc.bitcos_fp8_matmul(W, x, xs, out_dtype=torch.float16), lambda: bc.bitcos_fp8_matmul(W, x, xs, y=torch.empty(4, 255, device="cuda")),
                lambda: bc.bitcos_fp8_matmul(W, x[::2], xs[::2]), lambda: bc.bitcos_fp8_matmul(W, x, xs, workspace=torch.zeros(256, dtype=torch.uint8)),
                lambda: bc.bitcos_fp8_matmul_grouped(W, one, one, one, one, x, xs), lambda: bc.bitcos_fp8_matmul_grouped(E, one, one, one, one, x, xs),
                lambda: bc.bitcos_fp8_matmul_grouped(E, one[:1].long(), one, one, one, x, xs), lambda: bc.bitcos_fp8_quantize(x),
                lambda: bc.bitcos_fp8_quantize(torch.zeros(2, 256, device="cuda").t())):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(bc.BitcosError):
        bc.bitcos_fp8_quantize(torch.zeros(2, 100, device="cuda"))
    with pytest.raises(bc.BitcosError):
        bc.bitcos_fp8_matmul(W, x, xs, workspace=torch.zeros(128, dtype=torch.uint8, device="cuda"))
    assert bc.bitcos_fp8_matmul(W, x[:0], xs[:0]).shape == (0, 256)
    assert bc.bitcos_fp8_matmul_grouped(E, one[:1], one, one[:1], one[:0], x, xs).shape == (0, 256)
