"""Group norm at the ends of its ranges, on the GPU against float64: means whose square
leaves float32.

Bounds as in test_gpu_group_norm.py.
"""

import pytest

import test_gpu_group_norm as base

pytestmark = pytest.mark.gpu
U = base.U


@pytest.fixture(autouse=True)
def _announce(request):
    print(f"[gpu] start {request.node.name}", flush=True)
    yield


@pytest.mark.parametrize("B,S,C,groups", [
    (2, 1000, 64, 16),      # all rows in a tile: no statistics are merged
    (2, 2049, 256, 256),    # tiles of a part of the rows
    (1, 8200, 4, 4),
    (3, 1, 4160, 1),        # of a part of the channels
    (1, 9, 2051, 1),
])
def test_mean_whose_square_leaves_float32(dp, B, S, C, groups):
    # Values around 3e19 (its square is 9e38) of spread 3e16: the sum of squared deviations,
    # about 8200 x 1e33 x 3, is well inside float32.
    x, dy, gamma, beta = base._values(B, S, C, "f32", seed=S + C)
    x = x * 3e16 + 3e19
    base._check(x, dy, gamma, beta, groups, 1e-5, "none", "f32",
                base._run(dp, x, dy, gamma, beta, groups, 1e-5, "none"))
