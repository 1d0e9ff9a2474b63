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
