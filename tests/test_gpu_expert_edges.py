"""Calls at the edge of what the entry points around routed experts and e4m3 products document: sums of choices behind the range
of 32 bits, a status word that holds something already, batches without tokens."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_experts import check_route  # noqa: E402
from test_gpu_fp8 import activations, bc, weights  # noqa: E402,F401


@pytest.mark.parametrize("experts,n_groups", [(64, 4), (60, 4), (256, 8), (12, 3)])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_group_sums_behind_the_range_of_32_bits(bc, experts, n_groups, score):
    """Biases near the type's lowest value: the sum of a group's two best choices has no finite 32-bit value, and is still more than the
    sum of a group that a mask leaves nothing (or one expert) of, and in its own order among the others."""
    lowest = np.finfo(np.float32).min
    size = experts // n_groups
    rng = np.random.default_rng(experts)
    z = rng.normal(0, 1, (9, experts)).astype(np.float32)
    z[1, :size] = -np.inf                                  # nothing left of the first group
    z[2, 1:size] = np.nan                                  # one expert of it
    z[3, :2 * size] = -np.inf
    z[4, -size:] = -np.inf
    z[5, ::2] = -np.inf
    z[6] = -np.inf
    z[6, -size:] = 1.0                                     # only the last group
    for bias in (np.full(experts, lowest, np.float32),
                 np.where(np.arange(experts) % size < 2, lowest * rng.uniform(0.6, 1.0, experts), lowest).astype(np.float32),
                 np.where(np.arange(experts) // size == n_groups - 1, 0.0, lowest).astype(np.float32),
                 np.full(experts, -lowest, np.float32)):
        for top_groups in (1, n_groups - 1):
            for dtype in (torch.float32, torch.bfloat16):
                check_route(bc, torch.from_numpy(z).cuda().to(dtype), bias, top_k=4, score=score, n_groups=n_groups, top_groups=top_groups,
                            group_best=2)


@pytest.mark.parametrize("n_pairs,max_groups", [(40, 10), (200, 2)])
def test_marks_in_the_status_word_do_not_replace_one_another(bc, n_pairs, max_groups):
    """Calls may share the word: what one of them has said of a wait that ran out stays beside what another says of its lists."""
    w, ws = weights(2, 256, 512, 1)
    x, xs = activations(n_pairs, 512, 2)
    ge, gb = (torch.zeros(max_groups + i, dtype=torch.int32, device="cuda") for i in (0, 1))
    gb[1] = n_pairs
    xr = torch.arange(n_pairs, dtype=torch.int32, device="cuda")
    bad_row = xr.clone()
    bad_row[3] = n_pairs
    one, W = torch.ones(1, dtype=torch.int32, device="cuda"), bc.Fp8Weights(w, ws)
    for lists in ((ge + 7, gb, xr), (ge, gb, bad_row)):
        for before in (0, 1, 2, 3):
            space = bc.make_fp8_workspace()
            space[0] = before
            bc.bitcos_fp8_matmul_grouped(W, lists[0], lists[1], one, lists[2], x, xs, workspace=space)
            assert bc.workspace_status(space) == (before | 2)
            bc.bitcos_fp8_matmul_grouped(W, ge, gb, one, xr, x, xs, workspace=space)
            assert bc.workspace_status(space) == (before | 2)


def test_a_layer_without_tokens(bc):
    """Every call of a routed layer takes a batch of no tokens, recorded in a graph too; a sum whose y has no rows is its base, or zero."""
    E, k, H, M = 12, 4, 256, 384
    w, ws = weights(E, M, H, 1)
    W, space = bc.Fp8Weights(w, ws), bc.make_fp8_workspace()

    def layer(x, logits):
        expert, weight, _ = bc.bitcos_route_experts(logits, k)
        ge, gb, xr, order, slot, ng = bc.bitcos_group_pairs_slots(expert, E)
        q, s = bc.bitcos_fp8_quantize(x)
        y = bc.bitcos_fp8_matmul_grouped(W, ge, gb, ng, xr, q, s, workspace=space)
        return ge, gb, xr, order, slot, ng, y, bc.bitcos_combine_pairs(y, slot, weight)

    def check_empty(ge, gb, xr, order, slot, ng, y, out):
        assert all(t.dtype == torch.int32 and t.is_cuda for t in (ge, gb, xr, order, slot, ng))
        assert (ge.shape, gb.tolist(), xr.shape, order.shape, slot.shape, ng.tolist()) == ((0,), [0], (0,), (0,), (0, k), [0])
        assert y.shape == (0, M) and out.shape == (0, M)

    x, logits = torch.empty(0, H, device="cuda"), torch.empty(0, E, device="cuda")
    check_empty(*layer(x, logits))
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        out = layer(x, logits)
    graph.replay()
    torch.cuda.synchronize()
    check_empty(*out)
    for dtype in (torch.float32, torch.bfloat16):
        y = torch.empty(0, M, dtype=dtype, device="cuda")
        slot, weight = torch.zeros(5, k, dtype=torch.int32, device="cuda"), torch.full((5, k), float("nan"), device="cuda")
        base = torch.randn(5, M, device="cuda")
        assert (bc.bitcos_combine_pairs(y, slot, weight, out_dtype=torch.float32) == 0).all()
        got = bc.bitcos_combine_pairs(y, slot, weight, base=base)
        assert torch.equal(got, base) and got.data_ptr() != base.data_ptr()
        kept = base.clone()
        assert bc.bitcos_combine_pairs(y, slot, weight, base=base, out=base) is base and torch.equal(base, kept)
    # what is refused with tokens is refused without
    empty = torch.empty(0, k, dtype=torch.int32, device="cuda")
    for bad in (0, 1025, -1):
        with pytest.raises((ValueError, bc.BitcosError)):
            bc.bitcos_group_pairs_slots(empty, bad)
    with pytest.raises((ValueError, bc.BitcosError)):
        bc.bitcos_group_pairs_slots(torch.empty(0, 0, dtype=torch.int32, device="cuda"), E)
    with pytest.raises(ValueError):
        bc.bitcos_group_pairs_slots(empty.cpu(), E)
    with pytest.raises(ValueError):
        bc.bitcos_combine_pairs(y, slot, weight, out=torch.empty(5, M, dtype=torch.float16, device="cuda"))
