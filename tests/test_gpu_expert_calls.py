"""Calls around routed experts and e4m3 products as programs may make them: two streams at once, first of all into a graph, all pairs
on one expert, many tiles per block, rows and matrices behind 32 bits.  Bounds as in test_gpu_fp8."""
import os
import subprocess
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_experts import check_route  # noqa: E402
from test_gpu_fp8 import activations, bc, check, product_reference, weights  # noqa: E402,F401


def rows_of(x, index):
    return x.view(torch.uint8)[index].view(torch.float8_e4m3fn)


@pytest.mark.parametrize("n_pairs,max_groups,M,K", [(4096, 1024, 200, 256), (24, 24, 300, 1024), (3000, 200, 200, 256), (3000, 100, 200, 256),
                                                    (3000, 12, 200, 256), (1, 1024, 129, 2560)])
@pytest.mark.parametrize("gathered", [False, True])
def test_all_pairs_on_one_expert(bc, n_pairs, max_groups, M, K, gathered):
    """The lists leave room for many groups, all pairs are one group's: the order that suits their mean is the wrong one, and right.
    Every pair reads one of three rows."""
    experts, e = 5, 3
    w, ws = weights(experts, M, K, 1)
    x, xs = activations(n_pairs if not gathered else 3, K, 2)
    ge, gb = (torch.full((max_groups + i,), 99, dtype=torch.int32, device="cuda") for i in (0, 1))
    ge[0], gb[0], gb[1] = e, 0, n_pairs
    xr = torch.arange(n_pairs, dtype=torch.int32, device="cuda") % 3 if gathered else None
    space = bc.make_fp8_workspace()
    y = bc.bitcos_fp8_matmul_grouped(bc.Fp8Weights(w, ws), ge, gb, torch.ones(1, dtype=torch.int32, device="cuda"), xr, x, xs,
                                     y=torch.empty(n_pairs, M, device="cuda"), workspace=space)
    if gathered:
        x, xs = rows_of(x, xr.long()), xs[xr.long()]
    check(y, *product_reference(w[e], ws[e], x, xs), K // 128)
    assert bc.workspace_status(space) == 0


@pytest.mark.parametrize("n_pairs,max_groups", [(40, 10), (40, 3), (60, 2), (200, 2)])
def test_pairs_without_a_list_and_without_a_row(bc, n_pairs, max_groups):
    """Pair p reads row p: those behind the last row of x are left out and marked, in every order."""
    M, K, there = 260, 512, n_pairs - 7
    w, ws = weights(2, M, K, 1)
    x, xs = activations(there, K, 2)
    ge, gb = (torch.zeros(max_groups + i, dtype=torch.int32, device="cuda") for i in (0, 1))
    half = n_pairs // 2
    ge[1], gb[1], gb[2] = 1, half, n_pairs
    space = bc.make_fp8_workspace()
    y = torch.full((n_pairs, M), 7.0, device="cuda")
    bc.bitcos_fp8_matmul_grouped(bc.Fp8Weights(w, ws), ge, gb, torch.full((1,), 2, dtype=torch.int32, device="cuda"), None, x, xs, y=y,
                                 workspace=space, n_pairs=n_pairs)
    check(y[:half], *product_reference(w[0], ws[0], x[:half], xs[:half]), K // 128)
    check(y[half:there], *product_reference(w[1], ws[1], rows_of(x, slice(half, there)), xs[half:]), K // 128)
    assert (y[there:] == 7.0).all() and bc.workspace_status(space) == 2


@pytest.mark.parametrize("rows,M", [(4096, 32768), (600, 30000), (16, 300000), (64, 100000)])
def test_many_tiles_of_one_group(bc, rows, M):
    """K = 128: blocks go through tens of tiles, each of one group of 128."""
    w, ws = weights(1, M, 128, 1)
    x, xs = activations(rows, 128, 2)
    space = bc.make_fp8_workspace()
    y = bc.bitcos_fp8_matmul(bc.Fp8Weights(w[0], ws[0]), x, xs, out_dtype=torch.bfloat16, workspace=space)
    check(y, *product_reference(w[0], ws[0], x, xs), 1)
    assert bc.workspace_status(space) == 0


@pytest.mark.parametrize("per_group,experts,M", [(8, 64, 20000), (16, 32, 20000), (30, 32, 20000), (300, 16, 30000)])
def test_many_tiles_of_routed_pairs(bc, per_group, experts, M):
    w, ws = weights(experts, M, 128, 1)
    P = per_group * experts
    x, xs = activations(50, 128, 2)
    xr = torch.randint(0, 50, (P,), dtype=torch.int32, device="cuda")
    ge = torch.arange(experts, dtype=torch.int32, device="cuda").flip(0).contiguous()
    gb = torch.arange(experts + 1, dtype=torch.int32, device="cuda") * per_group
    space = bc.make_fp8_workspace()
    y = torch.empty(P, M, dtype=torch.bfloat16, device="cuda")
    bc.bitcos_fp8_matmul_grouped(bc.Fp8Weights(w, ws), ge, gb, torch.full((1,), experts, dtype=torch.int32, device="cuda"), xr, x, xs, y=y, workspace=space)
    for i in range(experts):
        r = xr[i * per_group:(i + 1) * per_group].long()
        e = experts - 1 - i
        check(y[i * per_group:(i + 1) * per_group], *product_reference(w[e], ws[e], rows_of(x, r), xs[r]), 1)
    assert bc.workspace_status(space) == 0


@pytest.mark.parametrize("n_pairs", [5, 14, 30, 90])
def test_experts_and_rows_behind_32_bits(bc, n_pairs):
    """Weights and activations of more than 2^31 bytes each; the last expert and the last rows, in every order."""
    experts, M, K, rows = 18, 8192, 16384, 140000
    W = torch.zeros(experts, M, K, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    X = torch.zeros(rows, K, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    w, ws = weights(1, M, K, 1)
    x, xs = activations(n_pairs, K, 2)
    W.view(torch.uint8)[-1] = w[0].view(torch.uint8)
    X.view(torch.uint8)[rows - n_pairs:] = x.view(torch.uint8)
    scales = torch.ones(experts, M // 128, K // 128, device="cuda")
    scales[-1] = ws[0]
    XS = torch.ones(rows, K // 128, device="cuda")
    XS[rows - n_pairs:] = xs
    one = torch.ones(1, dtype=torch.int32, device="cuda")
    y = torch.empty(n_pairs, M, device="cuda")
    bc.bitcos_fp8_matmul_grouped(bc.Fp8Weights(W, scales), one * (experts - 1), torch.tensor([0, n_pairs], dtype=torch.int32, device="cuda"), one,
                                 torch.arange(rows - n_pairs, rows, dtype=torch.int32, device="cuda"), X, XS, y=y)
    check(y, *product_reference(w[0], ws[0], x, xs), K // 128)


def test_two_streams_at_once(bc):
    """Dense and routed products of every order from two streams, again and again, with one status word between them: the same bits as alone."""
    M, K, experts = 1024, 1024, 16
    w, ws = weights(experts, M, K, 1)
    W, one, space = bc.Fp8Weights(w, ws), bc.Fp8Weights(w[0], ws[0]), bc.make_fp8_workspace()

    def job(rows, per_group):
        P = per_group * experts
        x, xs = activations(rows, K, rows)
        gen = torch.Generator(device="cuda").manual_seed(P)
        xr = torch.randint(0, rows, (P,), generator=gen, device="cuda").int()
        ge = torch.arange(experts, dtype=torch.int32, device="cuda")
        gb = torch.arange(experts + 1, dtype=torch.int32, device="cuda") * per_group
        ng = torch.full((1,), experts, dtype=torch.int32, device="cuda")
        return lambda: (bc.bitcos_fp8_matmul(one, x, xs, workspace=space),
                        bc.bitcos_fp8_matmul_grouped(W, ge, gb, ng, xr, x, xs, y=torch.empty(P, M, device="cuda"), workspace=space))

    jobs = [job(1, 1), job(40, 6), job(20, 14), job(300, 25), job(700, 90)]
    alone = [j() for j in jobs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[], []]
    for turn in range(8):
        for s in (0, 1):
            with torch.cuda.stream(streams[s]):
                for i in range(len(jobs)):
                    i = (i + s * 2 + turn) % len(jobs)
                    got[s].append((i, jobs[i]()))
    torch.cuda.synchronize()
    for results in got:
        for i, (a, b) in results:
            assert torch.equal(a, alone[i][0]) and torch.equal(b, alone[i][1])
    assert bc.workspace_status(space) == 0


def test_groups_that_overlap_are_marked_where_blocks_share_a_tile(bc):
    """More tiles than 24 pairs can make (13 times the same group): the rest is left out and marked, nothing else is touched."""
    w, ws = weights(2, 256, 1024, 1)
    x, xs = activations(24, 1024, 2)
    ge = torch.ones(26, dtype=torch.int32, device="cuda")
    gb = torch.tensor([0, 24] * 13 + [0], dtype=torch.int32, device="cuda")
    space = bc.make_fp8_workspace()
    y = torch.full((30, 256), 7.0, device="cuda")
    bc.bitcos_fp8_matmul_grouped(bc.Fp8Weights(w, ws), ge, gb, torch.full((1,), 26, dtype=torch.int32, device="cuda"), None, x, xs, y=y[:24],
                                 workspace=space)
    check(y[:24], *product_reference(w[1], ws[1], x, xs), 8)
    assert (y[24:] == 7.0).all() and bc.workspace_status(space) == 2
    with pytest.raises(ValueError):
        bc.bitcos_fp8_matmul_grouped(bc.Fp8Weights(w, ws), ge, gb, ge, torch.zeros(24, dtype=torch.int32, device="cuda"), x, xs, n_pairs=25)


FIRST = """
import torch, paper_2609_16338_b200 as bc
torch.manual_seed(1)
E, K, M = 16, 512, 384
codes = lambda *s: (torch.randn(*s, device="cuda") * 60).clamp(-448, 448).to(torch.float8_e4m3fn)
W = bc.Fp8Weights(codes(E, M, K), torch.rand(E, M // 128, K // 128, device="cuda"))
D = bc.Fp8Weights(W.codes[0], W.scales[0])
space = bc.make_fp8_workspace()
inputs = [(torch.randn(T, K, device="cuda"), torch.randn(T, E, device="cuda"), bc.make_group_workspace(T * 4, E)) for T in (1, 30, 50, 120, 700)]
def layer(x, logits, scratch):
    expert, weight, _ = bc.bitcos_route_experts(logits, 4)
    ge, gb, xr, order, slot, ng = bc.bitcos_group_pairs_slots(expert, E, workspace=scratch)
    q, s = bc.bitcos_fp8_quantize(x)
    y = torch.zeros(x.shape[0] * 4, M, device="cuda")
    bc.bitcos_fp8_matmul_grouped(W, ge, gb, ng, xr, q, s, y=y, workspace=space)
    return bc.bitcos_combine_pairs(y, slot, weight, base=bc.bitcos_fp8_matmul(D, q, s, workspace=space))
side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
torch.cuda.synchronize()
with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
    out = [layer(*i) for i in inputs]
for turn in range(2):
    for x, logits, _ in inputs:
        x.normal_(); logits.normal_()
    torch.cuda.synchronize(); graph.replay(); torch.cuda.synchronize()
    for o, i in zip(out, inputs):
        assert torch.equal(o, layer(*i))
assert bc.workspace_status(space) == 0
print("replayed")
"""


def test_the_first_call_of_a_process_is_recorded(bc):
    """What is asked of the device once per kernel may be asked while a graph is recorded."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    run = subprocess.run([sys.executable, "-c", FIRST], cwd=root, capture_output=True, text=True, timeout=600)
    assert run.returncode == 0 and "replayed" in run.stdout, run.stderr[-2000:]


@pytest.mark.parametrize("tokens,top_k,experts", [(64, 8, 128), (513, 1, 100), (65, 8, 16), (257, 3, 1024), (1183, 32, 64), (37889, 1, 3)])
def test_pairs_around_one_block_and_a_block_each(bc, tokens, top_k, experts):
    """512 pairs and 513, chunks of 256 and the first that are longer."""
    P = tokens * top_k
    gen = torch.Generator(device="cuda").manual_seed(P)
    pe = torch.randint(-1, experts, (tokens, top_k), generator=gen, device="cuda").int()
    ge, gb, xr, order, slot, ng = (t.cpu().numpy() for t in bc.bitcos_group_pairs_slots(pe, experts))
    flat = pe.cpu().numpy().ravel()
    kept = np.flatnonzero(flat >= 0)
    want = kept[np.argsort(flat[kept], kind="stable")]
    ids, first = np.unique(flat[want], return_index=True)
    assert int(ng[0]) == ids.size and np.array_equal(ge[:ids.size], ids) and np.array_equal(gb[:ids.size + 1], np.append(first, want.size))
    assert np.array_equal(order[:want.size], want) and np.array_equal(xr[:want.size], want // top_k)
    place = np.full(P, -1)
    place[want] = np.arange(want.size)
    assert np.array_equal(slot.ravel(), place)


def test_one_row_for_every_place(bc):
    """The same row of y for several places of a token and for all tokens; a token without any."""
    y = torch.randn(3, 1000, device="cuda")
    slot = torch.ones(50, 6, dtype=torch.int32, device="cuda")
    slot[7] = -1
    weight = torch.rand(50, 6, device="cuda")
    out = bc.bitcos_combine_pairs(y, slot, weight, out_dtype=torch.float32)
    want = weight.double().sum(1, keepdim=True) * y[1].double()
    want[7] = 0
    bound = (weight.double().sum(1, keepdim=True) * y[1].double().abs()) * 7 * 2.0 ** -24 + 1e-40
    assert ((out.double() - want).abs() <= bound).all() and (out[7] == 0).all()


@pytest.mark.parametrize("experts,n_groups,top_groups", [(256, 8, 4), (1024, 32, 7), (64, 16, 3), (512, 4, 1), (32, 32, 9)])
@pytest.mark.parametrize("group_best", [1, 2])
def test_groups_that_32_bits_cannot_tell(bc, experts, n_groups, top_groups, group_best):
    """Group values that differ by less than a rounding of 32 bits, with and without ties inside the groups, masked experts, groups
    with one expert left or none: 64 bits decide."""
    if group_best > experts // n_groups:
        pytest.skip("a group has one expert")
    rng = np.random.default_rng(experts + group_best)
    z = (rng.normal(0, 1e-6, (120, experts)) - 3.0).astype(np.float32)
    z[40:80] += rng.normal(0, 1, (40, experts)).astype(np.float32) * (rng.random((40, experts)) < 0.9)
    z[60:100][rng.random((40, experts)) < 0.6] = -np.inf
    z[100:, ::2] = np.nan
    bias = (1.0 + rng.integers(-3, 4, experts) * 2.0 ** -23).astype(np.float32)
    logits = torch.from_numpy(z).cuda()
    for score in ("sigmoid", "softmax"):
        check_route(bc, logits, bias, top_k=min(8, experts), score=score, n_groups=n_groups, top_groups=top_groups, group_best=group_best)
        check_route(bc, logits, None, top_k=min(8, experts), score=score, n_groups=n_groups, top_groups=top_groups, group_best=group_best)
    check_route(bc, logits.to(torch.bfloat16), bias, top_k=4, score="sigmoid", n_groups=n_groups, top_groups=top_groups, group_best=group_best)
