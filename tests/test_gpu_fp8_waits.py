"""The give-up path of the e4m3 products: with hardly any patience the warps of a block stop wherever they stand.  The kernel waits for
what is under way (copies, products, arrivals from the other block of a pair), says so in the status word and returns; the next
calls are ordinary ones."""
import ctypes as C

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_fp8 import activations, bc, routed, weights  # noqa: E402,F401

LIMITS = (0, 3, 10, 20, 40, 80, 160, 320, 999, 1_000, 10_000, 1_000_000)       # looks, then nanoseconds
# (rows, M, K): 16, 32 and 64 tokens weights first, K whole and cut over a cluster; pairs of blocks, one tile and several, and K of few stages
DENSE = [(1, 256, 5120), (1, 20000, 1024), (20, 512, 2560), (50, 8192, 5120), (600, 300, 2560), (600, 9000, 2560), (2000, 20000, 384), (700, 512, 128)]
# (tokens, top_k, experts, M, K): K cut, one tile after another, pairs of blocks
ROUTED = [(2, 4, 16, 768, 2048), (60, 8, 16, 5000, 1024), (900, 4, 16, 1536, 2048), (2000, 4, 8, 300, 256)]


def pointer(t):
    return C.c_void_p(0 if t is None else t.data_ptr())


def stream():
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


def dense_job(bc, rows, M, K):
    w, ws = weights(1, M, K, 1)
    x, xs = activations(rows, K, 2)
    W = bc.Fp8Weights(w[0], ws[0])

    def limited(y, space, limit):
        return bc.load_library().bitcos_fp8_matmul_limited(pointer(w), pointer(ws), M, K, pointer(x), pointer(xs), rows, pointer(y), 0,
                                                           pointer(space), space.numel(), limit, stream())

    return rows, limited, lambda y, space: bc.bitcos_fp8_matmul(W, x, xs, y=y, workspace=space)


def routed_job(bc, tokens, top_k, experts, M, K, gathered):
    w, ws = weights(experts, M, K, 1)
    (ge, gb, ng, xr), _ = routed(tokens, top_k, experts, 5)
    P = tokens * top_k
    rows = tokens if gathered else P
    x, xs = activations(rows, K, 2)
    W, xr = bc.Fp8Weights(w, ws), xr if gathered else None

    def limited(y, space, limit):
        return bc.load_library().bitcos_fp8_matmul_grouped_limited(pointer(w), pointer(ws), experts, M, K, pointer(ge), pointer(gb), pointer(ng),
                                                                   ge.numel(), pointer(xr), P, pointer(x), pointer(xs), rows, pointer(y), 0,
                                                                   pointer(space), space.numel(), limit, stream())

    return P, limited, lambda y, space: bc.bitcos_fp8_matmul_grouped(W, ge, gb, ng, xr, x, xs, y=y, workspace=space, n_pairs=P)


def check_job(bc, M, rows, limited, ordinary):
    room, space = torch.full((rows + 2, M), 7.0, device="cuda"), bc.make_fp8_workspace()
    want = torch.empty(rows, M, device="cuda")
    ordinary(want, space)
    assert bc.workspace_status(space) == 0
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    for limit in LIMITS:
        gave_up = 0
        for _ in range(6):
            room.fill_(7.0)
            space.zero_()
            begin.record()
            assert limited(room[:rows], space, limit) == 0
            end.record()
            status = bc.workspace_status(space)
            assert status in (0, 1)
            gave_up += status
            # what was under way has arrived: no wait for it has run out (those take half a second)
            assert begin.elapsed_time(end) < 100.0
            assert (room[rows:] == 7.0).all()
            if status == 0:
                assert torch.equal(room[:rows], want)
            space.zero_()
            got = ordinary(torch.empty(rows, M, device="cuda"), space)
            assert bc.workspace_status(space) == 0 and torch.equal(got, want)
        if limit == 0:
            assert gave_up > 0


@pytest.mark.parametrize("rows,M,K", DENSE)
def test_dense_products_that_give_up(bc, rows, M, K):
    check_job(bc, M, *dense_job(bc, rows, M, K))


@pytest.mark.parametrize("tokens,top_k,experts,M,K", ROUTED)
@pytest.mark.parametrize("gathered", [True, False])
def test_routed_products_that_give_up(bc, tokens, top_k, experts, M, K, gathered):
    check_job(bc, M, *routed_job(bc, tokens, top_k, experts, M, K, gathered))


def test_calls_that_give_up_in_a_row_and_beside_others(bc):
    """Calls without patience follow one another on one stream while ordinary ones run on another: those are right."""
    jobs = [(M, *dense_job(bc, rows, M, K)) for rows, M, K in ((1, 4096, 2560), (700, 2048, 2560))]
    jobs += [(M, *routed_job(bc, t, 4, 16, M, 1024, g)) for t, M, g in ((30, 768, True), (700, 1024, True), (700, 1024, False))]
    want = []
    for M, rows, _, ordinary in jobs:
        want.append(ordinary(torch.empty(rows, M, device="cuda"), None))
    torch.cuda.synchronize()
    spaces = [bc.make_fp8_workspace() for _ in range(2)]
    scratch = [torch.empty(rows, M, device="cuda") for M, rows, _, _ in jobs]
    streams, got = [torch.cuda.Stream(), torch.cuda.Stream()], []
    torch.cuda.synchronize()
    for turn in range(6):
        for i, (M, rows, limited, ordinary) in enumerate(jobs):
            with torch.cuda.stream(streams[0]):
                for limit in (0, 30, 2_000):
                    assert limited(scratch[i], spaces[0], limit) == 0
            with torch.cuda.stream(streams[1]):
                got.append((i, ordinary(torch.empty(rows, M, device="cuda"), spaces[1])))
    torch.cuda.synchronize()
    assert bc.workspace_status(spaces[0]) == 1 and bc.workspace_status(spaces[1]) == 0
    for i, y in got:
        assert torch.equal(y, want[i])
