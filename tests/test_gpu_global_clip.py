"""One norm over many tensors, and clipping to it, on the GPU against float64.

The squares are summed in float64, so the norm is the correctly rounded one up to the
few float64 roundings: within one float32 unit, 2^-23. A scaled entry is one product
with a factor that is itself rounded once: 2^-23 of its size.
"""

import math

import numpy as np
import pytest

from oracle import model_oracle as mo

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _announce(request):
    print(f"[gpu] start {request.node.name}", flush=True)
    yield


SETS = {
    "one value": [(1, 1)],
    "odd": [(3, 5), (1, 7), (129, 1), (63, 65), (1, 4097)],
    "blocks": [(64, 64), (128, 64), (100, 1000), (1, 4096), (1, 4095)],
    "many": [(k % 7 + 1, 13 + k) for k in range(130)],       # more than two launches' tables
    "large": [(1500, 3001), (2, 2), (1024, 1024)],
}


def _tensors(shapes, seed, size=1.0):
    import torch
    rng = np.random.default_rng(seed)
    return [torch.tensor((size * rng.standard_normal(s)).astype(np.float32)).cuda() for s in shapes]


def _clip(dp, grads, max_norm, in_place=False):
    import torch
    layers = [dp.shape_layer(1, 1, g.shape[1], g.shape[0], dp.DPSGD_F32) for g in grads]
    ws = torch.full((dp.dpsgd_global_norm_workspace_bytes(layers),), 0xFF, dtype=torch.uint8,
                    device="cuda")
    outs = grads if in_place else [torch.full_like(g, float("nan")) for g in grads]
    norm, factor = (torch.full((1,), float("nan"), device="cuda") for _ in range(2))
    only = torch.full((1,), float("nan"), device="cuda")
    dp.dpsgd_global_norm_multi(layers, grads, only, workspace=ws)
    dp.dpsgd_global_clip_multi(layers, grads, outs, max_norm, norm, factor, workspace=ws)
    torch.cuda.synchronize()
    assert torch.equal(only, norm) or (math.isnan(float(only)) and math.isnan(float(norm)))
    return float(norm), float(factor), outs


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("part", [0.3, 3.0])
@pytest.mark.parametrize("name", list(SETS))
def test_norm_and_clip(dp, name, part, in_place):
    grads = _tensors(SETS[name], seed=3)
    host = [g.cpu().numpy() for g in grads]
    n0 = mo.global_clip(host, math.inf)[0]
    limit = float(np.float32(part * n0))
    ref_n, ref_c, ref = mo.global_clip(host, limit)
    norm, factor, outs = _clip(dp, grads, limit, in_place)
    assert abs(norm - ref_n) <= 2.0 ** -23 * ref_n
    assert abs(factor - ref_c) <= 2.0 ** -23 * ref_c
    for got, r, h in zip(outs, ref, host):
        got = got.cpu().numpy()
        if part > 1:
            assert factor == 1.0 and np.array_equal(got, h)
        assert np.all(np.abs(got.astype(np.float64) - r) <= 2.0 ** -23 * np.abs(r) + 1e-44)


@pytest.mark.parametrize("size", [1e-30, 1e25])
def test_squares_outside_float32(dp, size):
    grads = _tensors([(40, 50), (3, 3)], seed=4, size=size)
    ref_n, ref_c, ref = mo.global_clip([g.cpu().numpy() for g in grads], size)
    norm, factor, outs = _clip(dp, grads, size)
    assert abs(norm - ref_n) <= 2.0 ** -23 * ref_n and abs(factor - ref_c) <= 2.0 ** -22 * ref_c


def test_special_values(dp):
    import torch
    zero = [torch.zeros(5, 7, device="cuda"), torch.zeros(1, 1, device="cuda")]
    norm, factor, outs = _clip(dp, zero, 1.0)
    assert norm == 0.0 and factor == 1.0 and float(outs[0].abs().sum()) == 0.0
    tie = [torch.tensor([[3.0]], device="cuda"), torch.tensor([[4.0]], device="cuda")]
    assert _clip(dp, tie, 5.0)[:2] == (5.0, 1.0)
    grads = _tensors([(4, 5), (2, 3)], seed=5)
    keep = [g.clone() for g in grads]
    norm, factor, outs = _clip(dp, grads, math.inf)
    assert factor == 1.0 and all(torch.equal(a, b) for a, b in zip(outs, keep))
    grads[1][0, 0] = math.inf
    norm, factor, outs = _clip(dp, grads, 1.0)
    assert norm == math.inf and factor == 0.0
    assert float(outs[0].abs().sum()) == 0.0 and math.isnan(float(outs[1][0, 0]))
    grads[1][0, 0] = math.nan
    norm, factor, outs = _clip(dp, grads, 1.0)
    assert math.isnan(norm) and math.isnan(factor) and bool(torch.isnan(outs[0]).all())


def test_captured_in_a_graph(dp):
    import torch
    grads = _tensors([(300, 200), (7, 9)], seed=6)
    layers = [dp.shape_layer(1, 1, g.shape[1], g.shape[0], dp.DPSGD_F32) for g in grads]
    ws = torch.empty(dp.dpsgd_global_norm_workspace_bytes(layers), dtype=torch.uint8, device="cuda")
    outs, norm = [torch.empty_like(g) for g in grads], torch.empty(1, device="cuda")

    def step():
        dp.dpsgd_global_clip_multi(layers, grads, outs, 10.0, norm, workspace=ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(3):
        for g, n in zip(grads, _tensors([(300, 200), (7, 9)], seed=60 + k, size=0.01 * 30 ** k)):
            g.copy_(n)
        graph.replay()
        torch.cuda.synchronize()
        got = [norm.clone()] + [o.clone() for o in outs]
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, [norm] + outs))


def test_binding_refusals(dp):
    import torch
    L = [dp.shape_layer(1, 1, 4, 3, dp.DPSGD_F32)]
    g = torch.zeros(3, 4, device="cuda")
    ws = torch.empty(dp.dpsgd_global_norm_workspace_bytes(L), dtype=torch.uint8, device="cuda")
    for bad in (g.double(), g.t(), g[:2], g.cpu()):
        with pytest.raises(ValueError):
            dp.dpsgd_global_clip_multi(L, [bad], [g], 1.0, workspace=ws)
    with pytest.raises(ValueError):
        dp.dpsgd_global_clip_multi(L, [g, g], [g], 1.0, workspace=ws)
    with pytest.raises(dp.DpsgdError):
        dp.dpsgd_global_clip_multi(L, [g], [g], 0.0, workspace=ws)
    with pytest.raises(dp.DpsgdError):
        dp.dpsgd_global_clip_multi(L, [g], [g], 1.0)
