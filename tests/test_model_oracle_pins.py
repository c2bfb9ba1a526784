"""The float64 definitions in oracle/model_oracle.py against central differences,
torch's differentiation and closed forms (CPU)."""

import math

import numpy as np
import pytest

from oracle import model_oracle as mo


def test_embedding_gradient_is_the_derivative_of_the_lookup():
    rng = np.random.default_rng(0)
    ids = np.array([[2, 0, 2, -1], [5, 4, 2, 2]])   # 5 is outside the table of 5 rows
    table, G = rng.standard_normal((5, 3)), rng.standard_normal((2, 4, 3))
    for i in range(2):
        g = mo.embedding_example_gradient(ids[i], G[i], 5, 1.7)
        for at in np.ndindex(table.shape):
            step = np.zeros_like(table)
            step[at] = 1.0   # the lookup is linear: the difference is exact up to rounding
            d = mo.embedding_lookup(ids[i], table + step, 1.7) - mo.embedding_lookup(ids[i], table, 1.7)
            assert abs(np.sum(d * G[i]) - g[at]) < 1e-12
    assert np.array_equal(mo.embedding_lookup(ids, table, 1.0)[0, 3], np.zeros(3))
    assert np.array_equal(mo.embedding_lookup(ids, table, 1.0)[1, 0], np.zeros(3))


def test_embedding_norm_counts_equal_tokens_together():
    G = np.ones((1, 3, 4))
    assert mo.embedding_norms_sq(np.array([[1, 1, 1]]), G, 2, 1.0)[0] == 36.0
    assert mo.embedding_norms_sq(np.array([[0, 1, 1]]), G, 2, 1.0)[0] == 20.0
    assert mo.embedding_norms_sq(np.array([[0, 1, 2]]), G, 2, 2.0)[0] == 32.0


@pytest.mark.parametrize("act", ["none", "silu", "gelu", "relu"])
def test_group_norm_gradients_against_differences(act):
    rng = np.random.default_rng(3)
    B, S, C, groups, eps = 2, 5, 6, 3, 1e-5
    x, dy = rng.standard_normal((B, S, C)) + 0.5, rng.standard_normal((B, S, C))
    gamma, beta = 1.0 + 0.2 * rng.standard_normal(C), 0.3 * rng.standard_normal(C)
    dx, dgamma, dbeta = mo.group_norm_backward(x, dy, groups, gamma, beta, eps, act)
    h = 1e-6

    def loss(x, gamma, beta):   # per example
        return np.sum(mo.group_norm(x, groups, gamma, beta, eps, act)[0] * dy, axis=(1, 2))

    # Central differences: error h^2 f'''/6 + 2^-52 |f| / h, below 1e-8 here.
    for at in np.ndindex(x.shape):
        e = np.zeros_like(x)
        e[at] = h
        d = (loss(x + e, gamma, beta) - loss(x - e, gamma, beta)).sum() / (2 * h)
        assert abs(d - dx[at]) < 1e-6
    for c in range(C):
        e = np.zeros(C)
        e[c] = h
        assert np.all(np.abs((loss(x, gamma + e, beta) - loss(x, gamma - e, beta)) / (2 * h)
                             - dgamma[:, c]) < 1e-6)
        assert np.all(np.abs((loss(x, gamma, beta + e) - loss(x, gamma, beta - e)) / (2 * h)
                             - dbeta[:, c]) < 1e-6)


@pytest.mark.parametrize("act", ["none", "silu", "gelu", "relu"])
def test_group_norm_against_torch(act):
    import torch
    import torch.nn.functional as F
    rng = np.random.default_rng(4)
    B, S, C, groups = 3, 7, 8, 2
    x, dy = rng.standard_normal((B, S, C)), rng.standard_normal((B, S, C))
    gamma, beta = rng.standard_normal(C), rng.standard_normal(C)
    tx = torch.tensor(x).transpose(1, 2).contiguous().requires_grad_()
    z = F.group_norm(tx, groups, torch.tensor(gamma), torch.tensor(beta), 1e-5)
    y = {"none": lambda v: v, "relu": F.relu, "silu": F.silu,
         "gelu": lambda v: F.gelu(v, approximate="tanh")}[act](z)
    y.backward(torch.tensor(dy).transpose(1, 2).contiguous())
    ry = mo.group_norm(x, groups, gamma, beta, 1e-5, act)[0]
    rdx = mo.group_norm_backward(x, dy, groups, gamma, beta, 1e-5, act)[0]
    assert np.allclose(ry, y.detach().transpose(1, 2).numpy(), rtol=0, atol=1e-12)
    assert np.allclose(rdx, tx.grad.transpose(1, 2).numpy(), rtol=0, atol=1e-12)


def test_global_clip():
    t = [np.array([3.0, 0.0]), np.array([[4.0]])]
    norm, c, out = mo.global_clip(t, 2.5)
    assert norm == 5.0 and c == 0.5 and out[1][0, 0] == 2.0
    assert mo.global_clip(t, 5.0)[1] == 1.0   # a tie is not clipped
    assert mo.global_clip(t, math.inf)[1] == 1.0
