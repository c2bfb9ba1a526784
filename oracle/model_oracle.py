"""Plain float64 NumPy definitions of the operators around the linear layers:
token tables, group norm with an activation, one norm over many tensors.

Each function follows the operation's definition term by term (loops over
examples, tokens and groups), so that it can be read against the formulas.
"""

from __future__ import annotations

import math

import numpy as np


def embedding_lookup(ids, table, scale):
    """out[b, t] = scale * table[id], zeros where id is outside the table."""
    ids = np.asarray(ids)
    out = np.zeros(ids.shape + (table.shape[1],))
    for at in np.ndindex(ids.shape):
        if 0 <= ids[at] < table.shape[0]:
            out[at] = scale * table[ids[at]]
    return out


def embedding_example_gradient(ids_i, G_i, n_rows, scale):
    """Gradient [n_rows, d] of the table for one example: ids [T], G [T, d]."""
    g = np.zeros((n_rows, G_i.shape[1]))
    for t, v in enumerate(ids_i):
        if 0 <= v < n_rows:
            g[v] += scale * G_i[t]
    return g


def embedding_norms_sq(ids, G, n_rows, scale):
    return np.array([np.sum(embedding_example_gradient(ids[i], G[i], n_rows, scale) ** 2)
                     for i in range(len(ids))])


def embedding_clipped_sum(ids, G, n_rows, scale, factors):
    out = np.zeros((n_rows, G.shape[2]))
    for i in range(len(ids)):
        if factors[i] != 0.0:
            out += factors[i] * embedding_example_gradient(ids[i], G[i], n_rows, scale)
    return out


def activation(z, act):
    if act == "relu":
        return np.maximum(z, 0.0)
    if act == "silu":
        return z / (1.0 + np.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1.0 + np.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3)))
    return z.copy()


def activation_slope(z, act):
    if act == "relu":
        return (z > 0).astype(np.float64)
    if act == "silu":
        p = 1.0 / (1.0 + np.exp(-z))
        return p + z * p * (1.0 - p)
    if act == "gelu":
        k = math.sqrt(2.0 / math.pi)
        t = np.tanh(k * (z + 0.044715 * z ** 3))
        return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * k * (1.0 + 3 * 0.044715 * z ** 2)
    return np.ones_like(z)


def group_norm(x, groups, gamma, beta, eps, act):
    """x [B, S, C] -> (y, mean [B, groups], rstd [B, groups], xh)."""
    B, S, C = x.shape
    w = C // groups
    mean, rstd, xh = np.zeros((B, groups)), np.zeros((B, groups)), np.zeros_like(x)
    for b in range(B):
        for g in range(groups):
            part = x[b, :, g * w:(g + 1) * w]
            mean[b, g] = part.mean()
            rstd[b, g] = 1.0 / math.sqrt(np.mean((part - mean[b, g]) ** 2) + eps)
            xh[b, :, g * w:(g + 1) * w] = (part - mean[b, g]) * rstd[b, g]
    return activation(gamma * xh + beta, act), mean, rstd, xh


def group_norm_backward(x, dy, groups, gamma, beta, eps, act):
    """(dx, dgamma [B, C], dbeta [B, C]) with per-example affine gradients."""
    B, S, C = x.shape
    w = C // groups
    _, _, rstd, xh = group_norm(x, groups, gamma, beta, eps, act)
    dz = dy * activation_slope(gamma * xh + beta, act)
    dx = np.zeros_like(x)
    for b in range(B):
        for g in range(groups):
            c = slice(g * w, (g + 1) * w)
            a, h = dz[b, :, c] * gamma[c], xh[b, :, c]
            dx[b, :, c] = rstd[b, g] * (a - a.mean() - h * np.mean(a * h))
    return dx, np.sum(dz * xh, axis=1), np.sum(dz, axis=1)


def global_clip(tensors, max_norm):
    """(norm, factor, scaled tensors)."""
    norm = math.sqrt(math.fsum(float(np.sum(np.asarray(t, np.float64) ** 2)) for t in tensors))
    c = max_norm / norm if norm > max_norm else 1.0
    return norm, c, [c * np.asarray(t, np.float64) for t in tensors]
