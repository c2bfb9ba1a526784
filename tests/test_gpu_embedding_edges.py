"""Token tables at the ends of their ranges, on the GPU against float64: scales whose square
leaves float32.

Bounds as in test_gpu_embedding.py.
"""

import numpy as np
import pytest

import test_gpu_embedding as base
from oracle import model_oracle as mo

pytestmark = pytest.mark.gpu
U = base.U


@pytest.fixture(autouse=True)
def _announce(request):
    print(f"[gpu] start {request.node.name}", flush=True)
    yield


@pytest.mark.parametrize("scale,size", [(1e-24, 1e17), (1e24, 1e-17)])
@pytest.mark.parametrize("B,T,d", [(100, 9, 16), (3, 300, 16), (2, 4200, 8)])
def test_scale_whose_square_leaves_float32(dp, B, T, d, scale, size):
    # One workgroup an example, several of them, and the list sorted by example; the first
    # example has no token, and its norm is 0 whatever the scale is.
    import torch
    rng = np.random.default_rng(T)
    ids = base._ids("padded", B, T, 40, rng)
    G = (size * rng.standard_normal((B, T, d))).astype(np.float32)
    scale = float(np.float32(scale))
    emb = dp.make_embedding(torch.tensor(ids).cuda(), (40, d), scale)
    got = torch.full((B,), float("nan"), device="cuda")
    dp.dpsgd_embedding_norms(emb, torch.tensor(G).cuda(), got, workspace=base._workspace(dp, emb))
    got, G = got.cpu().double().numpy(), G.astype(np.float64)
    ref = mo.embedding_norms_sq(ids, G, 40, scale)
    bound = (4 * T + 200) * U * ref
    for i in range(B):
        s, a = np.zeros((40, d)), np.zeros((40, d))
        at = (ids[i] >= 0) & (ids[i] < 40)
        np.add.at(s, ids[i][at], G[i][at])
        np.add.at(a, ids[i][at], np.abs(G[i][at]))
        off = np.bincount(ids[i][at], minlength=40)[:, None] * U * a
        bound[i] += scale ** 2 * np.sum(2 * np.abs(s) * off + off * off)
    assert got[0] == 0.0 and ref[0] == 0.0
    assert np.all(np.abs(got - ref) <= bound)
