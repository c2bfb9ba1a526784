"""Token tables at the ends of their ranges, on the GPU against float64: scales whose square
leaves float32, rows that the sort's and the sum's launches fill, examples that take the
most LDS.

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


def filled_from(V, d, N):
    """First row that the sort's launch fills with zeros (the sum's fills those before it)."""
    rows = ((30 << 20) + 1800 * N) // (4 * d)
    return -(-(V - rows) // 4) * 4 if rows < V else 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V,d", [(50257, 257), (50257, 260), (200003, 90)])
def test_rows_without_a_token_of_a_large_table(dp, V, d, dtype):
    import torch
    B, T = 5, 11
    first = filled_from(V, d, B * T)
    assert 0 < first < V - 64
    rng = np.random.default_rng(V + d)
    ids = rng.integers(0, V, (B, T))
    ids[0] = [0, 15, 16, 17, 63, 64, 65, V // 2, V - 2, V - 1, -1]
    ids[1] = np.arange(first - 5, first + 6)          # on both sides
    ids[2, :3] = [first, first - 1, V]
    G = torch.tensor(rng.standard_normal((B, T, d)).astype(np.float32))
    G = G.to(torch.float32 if dtype == "f32" else torch.bfloat16)
    emb = dp.make_embedding(torch.tensor(ids).cuda(), (V, d), 1.5)
    nsq = torch.tensor([0.25, 4.0, 1.0, 9.0, 2.0], device="cuda")
    C = 1.25
    n = np.sqrt(nsq.cpu().double().numpy())
    c = np.where(n > C, C / n, 1.0)
    ref, size = np.zeros((V, d)), np.zeros((V, d))
    count = np.zeros(V)
    for i in range(B):
        at = (ids[i] >= 0) & (ids[i] < V)
        g = 1.5 * c[i] * G[i].double().numpy()[at]
        np.add.at(ref, ids[i][at], g)
        np.add.at(size, ids[i][at], np.abs(g))
        np.add.at(count, ids[i][at], 1)
    for wanted in (True, False):   # with the factors' workgroups after the rows', and without
        grad = torch.full((V, d), float("nan"), device="cuda")
        fac = torch.full((B,), float("nan"), device="cuda") if wanted else None
        mask = torch.full((B,), 7, dtype=torch.uint8, device="cuda") if wanted else None
        dp.dpsgd_embedding_clip_accumulate(emb, G.cuda(), nsq, C, grad, factors_out=fac,
                                           mask_out=mask, workspace=base._workspace(dp, emb))
        got = grad.cpu().double().numpy()
        assert np.all(got[count == 0] == 0)
        assert np.all(np.abs(got - ref) <= size * ((count + 16) * U)[:, None])
        if wanted:
            assert np.allclose(fac.cpu().double().numpy(), c, rtol=8 * U)
            assert np.array_equal(mask.cpu().numpy(), (n > C).astype(np.uint8))


@pytest.mark.parametrize("B,T,V,d", [(1, 4096, 300, 768), (1, 4095, 300, 1024), (1, 4096, 70, 4096)])
def test_examples_that_take_the_most_lds(dp, B, T, V, d):
    # 127 to 131 KB: the lists of 4096 tokens and two rows of edges a part.
    base.test_norms_and_clipped_sum(dp, B, T, V, d, "words", "bf16", True)
