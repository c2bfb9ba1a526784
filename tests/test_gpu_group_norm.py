"""Group norm with an activation on the GPU against the float64 definitions.

Bounds, with u = 2^-24: the statistics are merged pairwise, so the mean is off by at
most K u mean|x| and the sum of squared deviations by K u of itself (and by the square
of the mean's error a value) with K = 64 for the depth of the merges here; every later
step adds a few u of its operands' sizes. The bounds below follow the formulas with
these, entry by entry; a float32 sum over S positions is off by at most (S + 16) u of the
sum of its terms' sizes. bf16 outputs add half a unit in the last place, 2^-8 of the value.
"""

import numpy as np
import pytest

from oracle import model_oracle as mo

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
K = 64.0


@pytest.fixture(autouse=True)
def _announce(request):
    print(f"[gpu] start {request.node.name}", flush=True)
    yield


def _torch():
    import torch
    return torch


SHAPES = [   # B, S, C, groups
    (1, 1, 64, 1),          # one position
    (2, 1, 12, 3),
    (1, 2, 1, 1),           # two values in a group
    (3, 5, 6, 6),           # groups of one channel
    (2, 49, 30, 10),        # groups of three, no vector divides a group
    (2, 225, 90, 10),
    (4, 64, 256, 16),
    (2, 1024, 64, 16),
    (1, 3000, 16, 16),
    (5, 7, 33, 11),         # odd channels: rows off 16 bytes
    (1, 17, 1032, 8),       # more channel vectors than threads
    (1, 4099, 24, 3),
    (70, 3, 8, 2),
    (1, 2048, 320, 32),
    (2, 40, 2, 1),
    (2, 3, 4100, 1),        # one group wider than a tile's block of channels
    (1, 9, 2051, 1),        # the same, no vectors
    (1, 40, 6200, 2),       # groups that straddle blocks
    (2, 1023, 33, 3),       # whole groups in one tile, rows not a multiple of its step
    (1, 5000, 12, 4),       # several tiles of narrow rows
    (3, 300, 144, 9),       # blocks of several groups, the last one smaller
]


def _values(B, S, C, dtype, seed, shift=0.0):
    torch = _torch()
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((B, S, C)) * np.exp(0.3 * rng.standard_normal(C)) + rng.standard_normal(C) + shift
    dy = rng.standard_normal((B, S, C))
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    x = torch.tensor(x.astype(np.float32)).to(dt)
    dy = torch.tensor(dy.astype(np.float32)).to(dt)
    gamma = torch.tensor((1 + 0.3 * rng.standard_normal(C)).astype(np.float32))
    beta = torch.tensor((0.3 * rng.standard_normal(C)).astype(np.float32))
    return x, dy, gamma, beta


def _run(dp, x, dy, gamma, beta, groups, eps, act):
    torch = _torch()
    B, C = x.shape[0], x.shape[-1]
    x, dy = x.cuda(), dy.cuda()
    gamma = None if gamma is None else gamma.cuda()
    beta = None if beta is None else beta.cuda()
    gn = dp.make_group_norm(x, groups, gamma, beta, eps, act)
    ws = torch.full((dp.dpsgd_group_norm_workspace_bytes(gn),), 0xFF, dtype=torch.uint8, device="cuda")
    y, dx = torch.full_like(x, float("nan")), torch.full_like(x, float("nan"))
    mean, rstd = (torch.full((B, groups), float("nan"), device="cuda") for _ in range(2))
    dgamma, dbeta = (torch.full((B, C), float("nan"), device="cuda") for _ in range(2))
    dp.dpsgd_group_norm_forward(gn, x, y, mean, rstd, workspace=ws)
    dp.dpsgd_group_norm_backward(gn, x, dy, mean, rstd, dx, dgamma, dbeta, workspace=ws)
    y2 = torch.empty_like(x)
    dp.dpsgd_group_norm_forward(gn, x, y2, workspace=ws)   # serving: no statistics kept
    torch.cuda.synchronize()
    assert torch.equal(y.nan_to_num(7.0), y2.nan_to_num(7.0))
    return [t.cpu().double().numpy() for t in (y, mean, rstd, dx, dgamma, dbeta)]


def _check(x, dy, gamma, beta, groups, eps, act, dtype, got):
    y, mean, rstd, dx, dgamma, dbeta = got
    x, dy = x.double().numpy(), dy.double().numpy()
    B, S, C = x.shape
    w = C // groups
    ga = np.ones(C) if gamma is None else gamma.double().numpy()
    be = np.zeros(C) if beta is None else beta.double().numpy()
    eps = float(np.float32(eps))
    ry, rmean, rrstd, xh = mo.group_norm(x, groups, ga, be, eps, act)
    rdx, rdgamma, rdbeta = mo.group_norm_backward(x, dy, groups, ga, be, eps, act)
    half = 2.0 ** -8 if dtype == "bf16" else U
    xa = np.abs(x).reshape(B, S, groups, w).mean(axis=(1, 3))
    dmean = K * U * xa
    assert np.all(np.abs(mean - rmean) <= dmean)
    # rstd: relative error of half the variance's.
    drstd = rrstd * (K * U + 0.5 * dmean ** 2 * rrstd ** 2)
    assert np.all(np.abs(rstd - rrstd) <= drstd)

    def wide(v):
        return np.repeat(v, w, axis=1)[:, None, :]

    dxh = wide(dmean * rrstd) + np.abs(xh) * wide(drstd / rrstd) + 4 * U * (np.abs(xh) + wide(rrstd * xa))
    z = ga * xh + be
    dz_z = np.abs(ga) * dxh + 4 * U * (np.abs(ga * xh) + np.abs(be))     # error of z
    # |act'| <= 1.13; its own evaluation: a few u of |z| + 1.
    assert np.all(np.abs(y - ry) <= 1.13 * dz_z + 32 * U * (np.abs(z) + np.abs(ry)) + half * np.abs(ry) + 1e-37)
    # dz = dy act'(z): |act''| <= 1.5 (SiLU 0.5, GELU 1.1). At |z| within its own error of 0 ReLU
    # may take either side: there dz is off by up to |dy|.
    slope = mo.activation_slope(z, act)
    dz = dy * slope
    e = np.abs(dy) * (1.5 * dz_z + 32 * U * (1 + np.abs(z))) if act in ("silu", "gelu") else 2 * U * np.abs(dz)
    if act == "relu":
        e = e + np.where(np.abs(z) <= dz_z, np.abs(dy), 0.0)
    n = S + 16
    eb = e.sum(1) + n * U * np.abs(dz).sum(1)
    eg = (e * np.abs(xh) + np.abs(dz) * dxh).sum(1) + n * U * np.abs(dz * xh).sum(1)
    assert np.all(np.abs(dbeta - rdbeta) <= eb + 1e-37)
    assert np.all(np.abs(dgamma - rdgamma) <= eg + 1e-37)

    def group_mean(v):   # [B, C] of sums over the positions -> group mean over all values
        return wide(v.reshape(B, groups, w).sum(2) / (S * w))

    m1, m2 = group_mean(ga * rdbeta), group_mean(ga * rdgamma)
    e1 = group_mean(np.abs(ga) * eb) + 2 * (w + 8) * U * group_mean(np.abs(ga * rdbeta))
    e2 = group_mean(np.abs(ga) * eg) + 2 * (w + 8) * U * group_mean(np.abs(ga * rdgamma))
    edx = wide(rrstd) * (np.abs(ga) * e + e1 + np.abs(xh) * e2 + dxh * np.abs(m2)
                         + 8 * U * (np.abs(ga * dz) + np.abs(m1) + np.abs(xh * m2)))
    edx += wide(drstd / rrstd) * np.abs(rdx)
    assert np.all(np.abs(dx - rdx) <= edx + half * np.abs(rdx) + 1e-37), np.max(np.abs(dx - rdx) - edx)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,S,C,groups", SHAPES)
@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu"])
def test_forward_and_backward(dp, B, S, C, groups, act, dtype):
    x, dy, gamma, beta = _values(B, S, C, dtype, seed=S * 7 + C)
    got = _run(dp, x, dy, gamma, beta, groups, 1e-5, act)
    _check(x, dy, gamma, beta, groups, 1e-5, act, dtype, got)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,S,C,groups", [(520, 8200, 1, 1), (260, 4200, 12, 3)])
def test_tiles_of_several_batches_of_rows(dp, B, S, C, groups, dtype):
    x, dy, gamma, beta = _values(B, S, C, dtype, seed=3)
    _check(x, dy, gamma, beta, groups, 1e-5, "silu", dtype, _run(dp, x, dy, gamma, beta, groups, 1e-5, "silu"))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,S,C,groups", [
    (2, 2100, 320, 32),     # rows of whole lines, groups that straddle the blocks
    (1, 2500, 324, 27),     # rows that share lines, the last block smaller
    (2, 2049, 77, 7),
    (3, 1, 4160, 1),        # one row, a group over many blocks
    (2, 2, 5001, 3),
])
def test_tiles_of_a_part_of_the_channels(dp, B, S, C, groups, dtype):
    x, dy, gamma, beta = _values(B, S, C, dtype, seed=S + C)
    _check(x, dy, gamma, beta, groups, 1e-5, "silu", dtype, _run(dp, x, dy, gamma, beta, groups, 1e-5, "silu"))


@pytest.mark.parametrize("affine", ["none", "gamma", "beta"])
def test_without_affine_parameters(dp, affine):
    x, dy, gamma, beta = _values(3, 50, 24, "f32", seed=1)
    gamma, beta = (gamma if affine == "gamma" else None), (beta if affine == "beta" else None)
    _check(x, dy, gamma, beta, 4, 1e-3, "silu", "f32", _run(dp, x, dy, gamma, beta, 4, 1e-3, "silu"))


@pytest.mark.parametrize("S,C,groups", [(1024, 64, 16), (9000, 32, 2), (33, 9, 3)])
def test_mean_far_from_zero(dp, S, C, groups):
    # Values of spread 1 around 1000: a difference of large sums would lose the variance.
    x, dy, gamma, beta = _values(2, S, C, "f32", seed=2, shift=1000.0)
    _check(x, dy, gamma, beta, groups, 1e-5, "none", "f32", _run(dp, x, dy, gamma, beta, groups, 1e-5, "none"))


def test_outlier_in_the_first_row(dp):
    x, dy, gamma, beta = _values(1, 2000, 16, "f32", seed=8)
    x[0, 0, :] = 3e4
    _check(x, dy, gamma, beta, 4, 1e-5, "none", "f32", _run(dp, x, dy, gamma, beta, 4, 1e-5, "none"))


def test_constant_rows_and_nan(dp):
    torch = _torch()
    x = torch.full((3, 70, 8), 2.5)
    x[1, 5, 3] = float("nan")
    y, mean, rstd, dx, dgamma, dbeta = _run(dp, x, torch.ones(3, 70, 8), None, None, 2, 1e-4, "relu")
    r = 1.0 / np.sqrt(np.float32(1e-4))
    assert np.all(y[0] == 0) and np.all(mean[0] == 2.5) and np.allclose(rstd[0], r, rtol=4 * U)
    assert np.all(y[2] == 0) and np.all(np.isfinite(dx[[0, 2]]))
    assert np.all(np.isnan(y[1, :, :4])) and np.all(y[1, :, 4:] == 0)   # its own group only
    assert np.all(np.isnan(dx[1, :, :4])) and np.all(np.isfinite(dx[1, :, 4:]))


def test_in_place_and_image_layout(dp):
    torch = _torch()
    x, dy, gamma, beta = _values(2, 48, 20, "f32", seed=9)
    got = _run(dp, x, dy, gamma, beta, 5, 1e-5, "gelu")
    # channels_last images: the permuted view is contiguous rows.
    img = x.view(2, 6, 8, 20).permute(0, 3, 1, 2).contiguous(memory_format=torch.channels_last).cuda()
    rows = img.permute(0, 2, 3, 1)
    gn = dp.make_group_norm(rows, 5, gamma.cuda(), beta.cuda(), 1e-5, "gelu")
    ws = torch.empty(dp.dpsgd_group_norm_workspace_bytes(gn), dtype=torch.uint8, device="cuda")
    mean, rstd = torch.empty(2, 5, device="cuda"), torch.empty(2, 5, device="cuda")
    keep = rows.clone()
    dp.dpsgd_group_norm_forward(gn, rows, rows, mean, rstd, workspace=ws)      # y over x
    assert np.array_equal(rows.reshape(2, 48, 20).cpu().double().numpy(), got[0])
    grad = dy.view(2, 6, 8, 20).cuda()
    dgamma, dbeta = torch.empty(2, 20, device="cuda"), torch.empty(2, 20, device="cuda")
    dp.dpsgd_group_norm_backward(gn, keep, grad, mean, rstd, grad, dgamma, dbeta, workspace=ws)  # dx over dy
    assert np.array_equal(grad.reshape(2, 48, 20).cpu().double().numpy(), got[3])


def test_affine_gradients_are_layers(dp):
    torch = _torch()
    x, dy, gamma, beta = _values(6, 40, 30, "f32", seed=10)
    _, _, _, _, dgamma, dbeta = _run(dp, x, dy, gamma, beta, 5, 1e-5, "silu")
    per = [torch.tensor(v, dtype=torch.float32, device="cuda") for v in (dgamma, dbeta)]
    ones = torch.ones(6, device="cuda")
    layers = [dp.affine_layer(ones, p, k) for k, p in enumerate(per)]
    buf = dp.alloc_step(layers)
    n = np.sqrt((dgamma ** 2).sum(1) + (dbeta ** 2).sum(1))
    C = float(np.median(n))
    dp.run_clipped_sum(layers, buf, C)
    torch.cuda.synchronize()
    assert np.allclose(np.sqrt(buf.norms_sq.cpu().double().numpy()), n, rtol=1e-5)
    c = np.minimum(1.0, C / n)[:, None]
    for got, p in zip(buf.grads, (dgamma, dbeta)):
        assert np.allclose(got.cpu().double().numpy()[:, 0], (c * p).sum(0), rtol=0,
                           atol=1e-5 * np.abs(c * p).sum(0).max())


def test_captured_in_a_graph(dp):
    torch = _torch()
    x, dy, gamma, beta = _values(2, 900, 48, "bf16", seed=11)
    x, dy, gamma, beta = x.cuda(), dy.cuda(), gamma.cuda(), beta.cuda()
    gn = dp.make_group_norm(x, 6, gamma, beta, 1e-5, "silu")
    ws = torch.empty(dp.dpsgd_group_norm_workspace_bytes(gn), dtype=torch.uint8, device="cuda")
    outs = [torch.empty_like(x), torch.empty(2, 6, device="cuda"), torch.empty(2, 6, device="cuda"),
            torch.empty_like(x), torch.empty(2, 48, device="cuda"), torch.empty(2, 48, device="cuda")]

    def step():
        dp.dpsgd_group_norm_forward(gn, x, outs[0], outs[1], outs[2], workspace=ws)
        dp.dpsgd_group_norm_backward(gn, x, dy, outs[1], outs[2], outs[3], outs[4], outs[5], workspace=ws)

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
        a, b, _, _ = _values(2, 900, 48, "bf16", seed=20 + k)
        x.copy_(a)
        dy.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outs]
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, outs))


def test_binding_refusals(dp):
    torch = _torch()
    x = torch.zeros(2, 5, 6, device="cuda")
    gn = dp.make_group_norm(x, 3)
    ws = torch.empty(dp.dpsgd_group_norm_workspace_bytes(gn), dtype=torch.uint8, device="cuda")
    for bad in (x.bfloat16(), x[:, :4].contiguous(), x.transpose(0, 1), x.cpu(),
                torch.zeros(2, 5, 12, device="cuda")[..., ::2]):
        with pytest.raises(ValueError):
            dp.dpsgd_group_norm_forward(gn, bad, torch.empty_like(x), workspace=ws)
    with pytest.raises(ValueError):
        dp.dpsgd_group_norm_forward(gn, x, x, torch.zeros(2, 6, device="cuda"), workspace=ws)
    with pytest.raises(dp.DpsgdError):
        dp.dpsgd_group_norm_forward(gn, x, x)
    with pytest.raises(dp.DpsgdError):
        dp.dpsgd_group_norm_forward(dp.make_group_norm(x, 4), x, x, workspace=ws)
