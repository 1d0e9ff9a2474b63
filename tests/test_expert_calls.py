"""What the entry points around the experts' products refuse, without a GPU: every check comes before the first CUDA call."""
import ctypes as C

import pytest

import paper_2609_16338_b200 as bc
from paper_2609_16338_b200 import build as bc_build

NULL, SHAPE, ALIGN, CAPACITY = 1, 2, 3, 6


@pytest.fixture(scope="module", autouse=True)
def built():
    bc_build.build()


def route(**kw):
    a = dict(logits=16, type=0, stride=128, bias=0, tokens=4, experts=128, score=0, n_groups=1, top_groups=1, group_best=1, top_k=8, renorm=1,
             scale=1.0, expert=16, weight=16, xrow=16)
    a.update(kw)
    v = list(a.values())
    return bc.load_library().bitcos_route_experts(*[C.c_void_p(x) if k in ("logits", "bias", "expert", "weight", "xrow") else x for k, x in a.items()], None), v


@pytest.mark.parametrize("change,want", [(dict(logits=0), NULL), (dict(expert=0), NULL), (dict(weight=0), NULL), (dict(xrow=0), NULL),
                                         (dict(tokens=-1), SHAPE), (dict(experts=0), SHAPE), (dict(experts=1025, stride=1025), SHAPE),
                                         (dict(stride=127), SHAPE), (dict(top_k=0), SHAPE), (dict(top_k=33), SHAPE),
                                         (dict(tokens=1 << 29), SHAPE), (dict(score=2), SHAPE), (dict(n_groups=0), SHAPE), (dict(n_groups=3), SHAPE),
                                         (dict(n_groups=64), SHAPE), (dict(n_groups=4, top_groups=5), SHAPE), (dict(top_groups=0), SHAPE),
                                         (dict(n_groups=4, group_best=3), SHAPE), (dict(group_best=0), SHAPE),
                                         (dict(experts=8, n_groups=8, group_best=2), SHAPE), (dict(type=3), SHAPE),
                                         (dict(logits=18), ALIGN), (dict(logits=17, type=1), ALIGN), (dict(bias=18), ALIGN), (dict(weight=18), ALIGN),
                                         (dict(tokens=0), 0)])
def test_route_refusals(change, want):
    assert route(**change)[0] == want


def group(pair_expert=16, n_pairs=100, top_k=2, experts=8, lists=(16,) * 6, ws=16, ws_bytes=256):
    p = C.c_void_p
    return bc.load_library().bitcos_group_pairs_slots(p(pair_expert), n_pairs, top_k, experts, *[p(v) for v in lists], p(ws), ws_bytes, None)


def test_group_refusals():
    assert group(pair_expert=0) == NULL and group(ws=0) == NULL
    for i in range(6):
        lists = [16] * 6
        lists[i] = 0
        assert group(lists=lists) == NULL
        lists[i] = 18
        assert group(lists=lists) == ALIGN
    assert group(n_pairs=0) == SHAPE and group(n_pairs=1 << 31) == SHAPE and group(top_k=0) == SHAPE
    assert group(experts=0) == SHAPE and group(experts=1025) == SHAPE
    need = bc.load_library().bitcos_group_workspace_bytes(1 << 20, 128)
    assert need > 256 and group(n_pairs=1 << 20, experts=128, ws_bytes=need - 1) == CAPACITY
    assert group(ws_bytes=255) == CAPACITY
    assert bc.load_library().bitcos_group_workspace_bytes(1 << 31, 128) == 0


def combine(y=16, y_type=0, n_rows=10, slot=16, weight=16, tokens=4, top_k=2, M=64, base=0, out=16, out_type=0):
    p = C.c_void_p
    return bc.load_library().bitcos_combine_pairs(p(y), y_type, n_rows, p(slot), p(weight), tokens, top_k, M, p(base), p(out), out_type, None)


def test_combine_refusals():
    for name in ("y", "slot", "weight", "out"):
        assert combine(**{name: 0}) == NULL
    for change in (dict(n_rows=0), dict(tokens=-1), dict(tokens=1 << 31), dict(top_k=0), dict(M=0), dict(M=1 << 31), dict(y_type=2), dict(out_type=2)):
        assert combine(**change) == SHAPE
    for change in (dict(y=8), dict(out=8), dict(base=8), dict(slot=18), dict(weight=18)):
        assert combine(**change) == ALIGN
    assert combine(tokens=0) == 0


def fp8(**kw):
    a = dict(W=16, w_scale=16, M=256, K=256, x=16, x_scale=16, rows=4, y=16, y_type=0, ws=0, ws_bytes=0)
    a.update(kw)
    p = C.c_void_p
    return bc.load_library().bitcos_fp8_matmul(p(a["W"]), p(a["w_scale"]), a["M"], a["K"], p(a["x"]), p(a["x_scale"]), a["rows"], p(a["y"]), a["y_type"],
                                               p(a["ws"]), a["ws_bytes"], None)


@pytest.mark.parametrize("change,want", [(dict(W=0), NULL), (dict(w_scale=0), NULL), (dict(x=0), NULL), (dict(x_scale=0), NULL), (dict(y=0), NULL),
                                         (dict(M=0), SHAPE), (dict(K=0), SHAPE), (dict(K=100), SHAPE), (dict(K=192), SHAPE), (dict(rows=-1), SHAPE),
                                         (dict(M=1 << 31), SHAPE), (dict(K=1 << 31), SHAPE), (dict(rows=1 << 31), SHAPE), (dict(y_type=2), SHAPE),
                                         (dict(W=8), ALIGN), (dict(x=8), ALIGN), (dict(y=8), ALIGN), (dict(x_scale=18), ALIGN), (dict(w_scale=18), ALIGN),
                                         (dict(ws=8, ws_bytes=256), ALIGN), (dict(ws=16, ws_bytes=255), CAPACITY), (dict(rows=0), 0)])
def test_fp8_matmul_refusals(change, want):
    assert fp8(**change) == want


def grouped(**kw):
    a = dict(W=16, w_scale=16, E=4, M=256, K=256, ge=16, gb=16, ng=16, max_groups=4, xrow=16, pairs=8, x=16, x_scale=16, xrows=4, y=16, y_type=0, ws=0, ws_bytes=0)
    a.update(kw)
    p = C.c_void_p
    return bc.load_library().bitcos_fp8_matmul_grouped(p(a["W"]), p(a["w_scale"]), a["E"], a["M"], a["K"], p(a["ge"]), p(a["gb"]), p(a["ng"]),
                                                       a["max_groups"], p(a["xrow"]), a["pairs"], p(a["x"]), p(a["x_scale"]), a["xrows"], p(a["y"]),
                                                       a["y_type"], p(a["ws"]), a["ws_bytes"], None)


@pytest.mark.parametrize("change,want", [(dict(W=0), NULL), (dict(ge=0), NULL), (dict(gb=0), NULL), (dict(ng=0), NULL), (dict(x=0), NULL), (dict(y=0), NULL),
                                         (dict(E=0), SHAPE), (dict(max_groups=0), SHAPE), (dict(max_groups=1025), SHAPE), (dict(pairs=-1), SHAPE),
                                         (dict(pairs=1 << 31), SHAPE), (dict(xrows=0), SHAPE), (dict(M=0), SHAPE), (dict(K=64), SHAPE), (dict(y_type=2), SHAPE),
                                         (dict(W=8), ALIGN), (dict(x=8), ALIGN), (dict(y=8), ALIGN), (dict(ge=18), ALIGN), (dict(xrow=18), ALIGN),
                                         (dict(ws=16, ws_bytes=255), CAPACITY), (dict(pairs=0), 0)])
def test_fp8_grouped_refusals(change, want):
    assert grouped(**change) == want


def test_fp8_quantize_refusals():
    p = C.c_void_p

    def call(x=16, x_type=0, rows=4, K=256, q=16, scale=16):
        return bc.load_library().bitcos_fp8_quantize(p(x), x_type, rows, K, p(q), p(scale), None)

    assert [call(x=0), call(q=0), call(scale=0)] == [NULL] * 3
    assert [call(x_type=2), call(rows=-1), call(K=100), call(K=0), call(rows=1 << 31)] == [SHAPE] * 5
    assert [call(x=8), call(q=8), call(scale=18)] == [ALIGN] * 3
    assert call(rows=0) == 0
