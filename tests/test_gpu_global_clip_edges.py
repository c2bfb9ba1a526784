"""One norm over many tensors, and clipping to it, at the sizes where the launches change:
tensors around one block of 8192 entries, more blocks than workgroups, outputs past the
caches. Bounds as in test_gpu_global_clip.py.
"""

import math

import numpy as np
import pytest

import test_gpu_global_clip as base
from oracle import model_oracle as mo

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _announce(request):
    print(f"[gpu] start {request.node.name}", flush=True)
    yield


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("part", [0.3, 3.0])
def test_tensors_around_a_block(dp, part, in_place, monkeypatch):
    monkeypatch.setitem(base.SETS, "around a block", [
        (1, 8191), (1, 8192), (1, 8193), (128, 64), (1, 1), (3, 5461), (1, 16384), (5, 3277), (1, 3)])
    base.test_norm_and_clip(dp, "around a block", part, in_place)


@pytest.mark.parametrize("in_place", [False, True])
def test_whole_model(dp, in_place):
    # 51.3 M entries, 205 MB: above 192 MB of outputs, and 6260 blocks over 2048 workgroups,
    # with tensors of less than a block between large ones. c is below 1.
    import torch
    shapes = [(5000, 4000), (3, 5), (1, 8191), (4099, 4097), (7, 9), (1, 8193), (3600, 4001), (1, 2)]
    assert sum(a * b for a, b in shapes) * 4 > 192 << 20
    rng = np.random.default_rng(8)
    host = [rng.standard_normal(s, dtype=np.float32) for s in shapes]
    for k in (1, 4, 7):
        host[k] *= 100.0    # the small ones count in the norm
    grads = [torch.tensor(h).cuda() for h in host]
    n0 = math.sqrt(sum(float(np.sum(h.astype(np.float64) ** 2)) for h in host))
    limit = float(np.float32(0.3 * n0))
    norm, factor, outs = base._clip(dp, grads, limit, in_place)
    c = limit / n0
    assert abs(norm - n0) <= 2.0 ** -23 * n0 and abs(factor - c) <= 2.0 ** -23 * c
    for got, h in zip(outs, host):
        want = c * h.astype(np.float64)
        assert np.all(np.abs(got.cpu().numpy() - want) <= 2.0 ** -23 * np.abs(want) + 1e-44)


@pytest.mark.parametrize("size", [1e-30, 1e25])
def test_outputs_where_squares_leave_float32(dp, size):
    # max_norm is rounded to float32 (u), the factor and the product once each: 2^-22.
    grads = base._tensors([(40, 50), (3, 3), (91, 97)], seed=4, size=size)
    host = [g.cpu().numpy() for g in grads]
    _, _, ref = mo.global_clip(host, size)
    _, factor, outs = base._clip(dp, grads, size)
    assert factor < 1.0
    for got, r in zip(outs, ref):
        assert np.all(np.abs(got.cpu().double().numpy() - r) <= 2.0 ** -22 * np.abs(r) + 1e-44)


@pytest.mark.parametrize("in_place", [False, True])
def test_norm_above_float32_and_infinite_bound(dp, in_place):
    import torch
    grads = [torch.full((100, 90), 3e38, device="cuda"), torch.full((1, 3), -1e38, device="cuda")]
    host = [g.cpu().numpy() for g in grads]
    limit = float(np.float32(1e38))
    ref_n, ref_c, ref = mo.global_clip(host, limit)      # 2.8e40
    norm, factor, outs = base._clip(dp, grads, limit, in_place)
    assert norm == math.inf and abs(factor - ref_c) <= 2.0 ** -23 * ref_c
    for got, r in zip(outs, ref):
        assert np.all(np.abs(got.cpu().double().numpy() - r) <= 2.0 ** -23 * np.abs(r))
    # No bound: nothing changes, an infinite entry neither.
    grads = [torch.tensor([[1.5, -math.inf, 3.0]], device="cuda"), torch.ones(4, 5, device="cuda")]
    keep = [g.clone() for g in grads]
    norm, factor, outs = base._clip(dp, grads, math.inf, in_place)
    assert norm == math.inf and factor == 1.0
    assert all(torch.equal(a, b) for a, b in zip(outs, keep))
