"""Group norm at the ends of its ranges, on the GPU against float64: means whose square
leaves float32, pre-activations far from 0, the order of tiles by XCD.

Bounds as in test_gpu_group_norm.py.
"""

import numpy as np
import pytest

import test_gpu_group_norm as base
from oracle import model_oracle as mo

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


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("B,S,C,groups", [(2, 49, 30, 10), (1, 5000, 12, 4)])
def test_slope_far_from_zero(dp, B, S, C, groups, act):
    # gamma 1e20: |z| is 1e13 and more, where y is max(z, 0) and its slope 0 or 1 in float64
    # too, and z^2 leaves float32. ReLU's bounds hold then.
    x, dy, gamma, beta = base._values(B, S, C, "f32", seed=S)
    gamma = gamma * 1e20
    z = mo.group_norm(x.double().numpy(), groups, gamma.double().numpy(), beta.double().numpy(), 1e-5, "none")[0]
    assert np.abs(z).min() > 1e13 and np.abs(z).max() > 5e19
    base._check(x, dy, gamma, beta, groups, 1e-5, "relu", "f32",
                base._run(dp, x, dy, gamma, beta, groups, 1e-5, act))


@pytest.mark.parametrize("S,C", [(70, 8), (9000, 4)])
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_tails_of_the_activations(dp, S, C, act):
    # gamma 0: z is beta, exactly. y = z / (1 + exp(-w)) with w = z (SiLU) or
    # 2 sqrt(2 / pi) (z + 0.044715 z^3). Relative to y, with one u for each rounding: w is off
    # by 0 or 6 u of itself, its product with the rounded log2(e) by 1.25 u more, all of which
    # the exponential multiplies by |w|; exponential, sum, reciprocal and product add 8 u.
    import torch
    lo, hi = (-80.0, 30.0) if act == "silu" else (-9.0, 9.0)
    beta = torch.tensor(np.random.default_rng(1).uniform(lo, hi, C).astype(np.float32))
    beta[0], beta[1] = lo, hi
    x, _, _, _ = base._values(1, S, C, "f32", seed=2)
    gn_x = x.cuda()
    gn = dp.make_group_norm(gn_x, 2, torch.zeros(C, device="cuda"), beta.cuda(), 1e-5, act)
    ws = torch.empty(dp.dpsgd_group_norm_workspace_bytes(gn), dtype=torch.uint8, device="cuda")
    y = torch.full_like(gn_x, float("nan"))
    dp.dpsgd_group_norm_forward(gn, gn_x, y, workspace=ws)
    z = beta.double().numpy()
    w = z if act == "silu" else 2 * np.sqrt(2 / np.pi) * (z + 0.044715 * z ** 3)
    ref = z / (1 + np.exp(-w))
    bound = ((1.25 if act == "silu" else 7.25) * np.abs(w) + 8) * U * np.abs(ref)
    assert np.all(np.abs(y[0].cpu().double().numpy() - ref) <= bound)


@pytest.mark.parametrize("dtype,B,S", [("f32", 67, 1100), ("f32", 64, 2048), ("bf16", 67, 700), ("bf16", 71, 1300)])
def test_tiles_that_share_lines_on_one_xcd(dp, dtype, B, S):
    # Rows of 64 bytes, in the backward pass or in both, for batches that are no multiple
    # of the XCDs and one that is; outputs start as NaN.
    x, dy, gamma, beta = base._values(B, S, 64, dtype, seed=S)
    base._check(x, dy, gamma, beta, 16, 1e-5, "silu", dtype,
                base._run(dp, x, dy, gamma, beta, 16, 1e-5, "silu"))
