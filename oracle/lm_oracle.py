"""Plain NumPy definitions of the operators between and behind a model's blocks: log
probabilities of tokens and the loss, residual norms (float64), and AdamW with moments
in 8 bits (float32, each operation rounded by itself, as it is defined).

Each function follows the operation's definition term by term (loops over rows), so
that it can be read against the formulas.
"""

from __future__ import annotations

import math

import numpy as np

from . import philox

# ------------------------------------------------------ log probabilities of tokens


def row_kind(z):
    """'nan', 'none' (every entry is -inf) or 'plain'."""
    if np.isnan(z).any() or (z == np.inf).any():
        return "nan"
    return "none" if (z == -np.inf).all() else "plain"


def token_row(x, scale):
    """lse, log probabilities [V] and entropy of one row of logits."""
    z = scale * x
    kind = row_kind(z)
    if kind == "nan":
        return np.nan, np.full(len(x), np.nan), np.nan
    if kind == "none":
        return -np.inf, np.full(len(x), -np.inf), 0.0
    m = z.max()
    lse = m + math.log(np.exp(z - m).sum())
    lp = z - lse
    here = lp > -np.inf
    return lse, lp, -float(np.sum(np.exp(lp[here]) * lp[here]))


def alternatives(x, scale, k):
    """The k largest logits' tokens and log probabilities; -1 where there are fewer."""
    lse, lp, _ = token_row(x, scale)
    ids, lps = np.full(k, -1, np.int64), np.full(k, -np.inf)
    if np.isnan(lse):
        lps[:] = np.nan
    elif lse > -np.inf:
        order = sorted((v for v in range(len(x)) if x[v] > -np.inf), key=lambda v: (-x[v], v))[:k]
        ids[:len(order)], lps[:len(order)] = order, lp[order]
    return ids, lps


def token_logprobs(x, targets, scale, k=0):
    """x [N, V], targets [N] or None: logprobs, lse, entropy [N], top ids and log
    probabilities [N, k]. An empty position has zeros and no alternatives."""
    N, V = x.shape
    out = [np.zeros(N), np.zeros(N), np.zeros(N), np.full((N, k), -1, np.int64),
           np.full((N, k), -np.inf)]
    for i in range(N):
        if targets is not None and not 0 <= targets[i] < V:
            continue
        lse, lp, entropy = token_row(x[i], scale)
        out[0][i] = 0.0 if targets is None else lp[targets[i]]
        out[1][i], out[2][i] = lse, entropy
        out[3][i], out[4][i] = alternatives(x[i], scale, k)
    return out


def token_gradient(x, targets, scale, g_logp=None, g_lse=None, g_entropy=None):
    """Gradient of sum g_logp logprob + g_lse lse + g_entropy entropy by x [N, V]."""
    N, V = x.shape
    out = np.zeros((N, V))
    for i in range(N):
        if targets is not None and not 0 <= targets[i] < V:
            continue
        gp, gl, ge = (0.0 if g is None else g[i] for g in (g_logp, g_lse, g_entropy))
        if gp == 0.0 and gl == 0.0 and ge == 0.0:
            continue
        lse, lp, entropy = token_row(x[i], scale)
        if np.isnan(lse):
            out[i] = np.nan
        elif lse > -np.inf:
            here = lp > -np.inf
            p, l = np.exp(lp[here]), lp[here]
            out[i, here] = p * (gl - gp - ge * (l + entropy))
            if gp != 0.0:
                out[i, targets[i]] += gp
            out[i] *= scale
    return out


# ------------------------------------------------------------------ residual norms


def norm_rows(v, kind, eps):
    """Normed rows, mean and 1 / deviation ([..., 1])."""
    mean = v.mean(-1, keepdims=True) if kind == "layer" else np.zeros(v.shape[:-1] + (1,))
    rstd = 1.0 / np.sqrt(((v - mean) ** 2).mean(-1, keepdims=True) + eps)
    return (v - mean) * rstd, mean, rstd


def _gate(gate):
    return 1.0 if gate is None else (gate[:, None, :] if gate.ndim == 2 else gate)


def _affine(vh, gamma, beta):
    return vh * (1.0 if gamma is None else gamma) + (0.0 if beta is None else beta)


def residual(x, block, kind, eps, alpha, gate=None, post=False, post_gamma=None, post_beta=None):
    """r before it is rounded, and the block's statistics."""
    zero = np.zeros(x.shape[:-1] + (1,))
    if block is None:
        return alpha * x, zero, zero
    u, mean, rstd = block, zero, zero
    if post:
        u, mean, rstd = norm_rows(block, kind, eps)
        u = _affine(u, post_gamma, post_beta)
    return alpha * x + _gate(gate) * u, mean, rstd


def normed(r, kind, eps, gamma=None, beta=None):
    vh, mean, rstd = norm_rows(r, kind, eps)
    return _affine(vh, gamma, beta), mean, rstd


def _norm_back(g, vh, rstd, kind):
    m2 = (g * vh).mean(-1, keepdims=True)
    m1 = g.mean(-1, keepdims=True) if kind == "layer" else 0.0
    return rstd * (g - m1 - vh * m2)


def residual_norm_backward(r, block, dy, dr, kind, eps, alpha, gamma=None, gate=None, post=False,
                           post_gamma=None, post_beta=None):
    """Gradients by name; those of the affine parameters per example [B, C]."""
    rh, _, rstd = norm_rows(r, kind, eps)
    out = {"dgamma": (dy * rh).sum(1), "dbeta": dy.sum(1)}
    dR = (0.0 if dr is None else dr) + _norm_back(dy * (1.0 if gamma is None else gamma), rh, rstd, kind)
    out["dx"] = alpha * dR
    if block is None:
        return out
    u, dU = block, _gate(gate) * dR
    if post:
        bh, _, brstd = norm_rows(block, kind, eps)
        u = _affine(bh, post_gamma, post_beta)
        out["dpost_gamma"], out["dpost_beta"] = (dU * bh).sum(1), dU.sum(1)
        out["dblock"] = _norm_back(dU * (1.0 if post_gamma is None else post_gamma), bh, brstd, kind)
    else:
        out["dblock"] = dU
    out["dgate"] = (dR * u).sum(1)
    return out


# ------------------------------------------------------- AdamW with 8-bit moments

BLOCK = 256
TOP = {"m": 15, "v": 31}
LOWEST = {"m": 32, "v": 48}


def block_exponents(x, which):
    """One biased exponent for every 256 entries (float32): the largest magnitude's,
    rounded up to 3 bits of fraction; 255 where that is not finite."""
    out = []
    for i in range(0, len(x), BLOCK):
        a = np.abs(x[i:i + BLOCK]).max()
        if not np.isfinite(a):
            out.append(255)
            continue
        f, e = math.frexp(float(a))                    # a = f 2^e, 1/2 <= f < 1
        k = 0 if a == 0 else e - 1 + (1 if f > 1.875 / 2 else 0) + 127
        out.append(min(255, max(LOWEST[which], k)))
    return np.array(out, np.int64)


def code_values(which):
    """The 256 (v) or 128 (m, without the sign) magnitudes of a block whose exponent
    stands for 2^0."""
    n = 128 if which == "m" else 256
    return np.array([math.ldexp(c & 7 if c < 8 else 8 + (c & 7), max(c >> 3, 1) - 3 - TOP[which])
                     for c in range(n)])


def decode(codes, exps, which):
    k = np.repeat(exps.astype(np.int64), BLOCK)[:len(codes)]
    mag = code_values(which)[codes & (127 if which == "m" else 255)] * np.exp2(k - 127.0)
    mag = np.where(k == 255, np.nan, mag)
    if which == "m":
        mag = np.where(codes & 128, -mag, mag)
    return mag.astype(np.float32)


def encode(x, exps, which, r16=None):
    """Codes of float32 moments; r16: 16 random bits an entry, or None (to nearest)."""
    k = np.repeat(exps, BLOCK)[:len(x)]
    values = code_values(which)
    with np.errstate(invalid="ignore", over="ignore"):
        mag = np.where(k < 255, np.abs(x).astype(np.float64), 0.0) * np.exp2(127.0 - k)
    c = np.searchsorted(values, mag, side="right") - 1              # the value below
    step = np.append(values[1:], 2.0 * values[-1])[c] - values[c]
    # Where between two codes, in 2^-20 (of what lies below float32's lowest, as rounded there).
    part = (mag - values[c]) / step * 2 ** 20
    part = np.where(c < 8, np.rint(part), part)
    if r16 is not None:
        c = c + (part + (r16.astype(np.int64) << 4) >= 2 ** 20)
    else:
        c = c + ((part > 2 ** 19) | ((part == 2 ** 19) & (c % 2 == 1)))
    if which == "v":
        c = np.where((c == 0) & (x > 0), 1, c)
    else:
        c = c | np.where(x < 0, 128, 0)
    return np.where(k < 255, c, 0).astype(np.uint8)


def rounding_bits(n, tensor_id, t, round_seed):
    """16 bits for m, 16 for v of each entry."""
    w = philox.philox_blocks(-(-n // 4), ~round_seed, tensor_id, t).reshape(-1)[:n]
    return w & 0xFFFF, w >> 16


def adamw8_moments(grad, m, v, opt, scale):
    """g and the new moments before they are rounded (float32 arrays, float32 operations);
    grad is the noisy sum."""
    f = np.float32
    b1, b2 = float(f(opt.beta1)), float(f(opt.beta2))
    with np.errstate(all="ignore"):
        g = f(scale) * grad
        m = f(b1) * m + f(1.0 - b1) * g
        v = f(b2) * v + f(1.0 - b2) * (g * g)
    return g, m, v


def adamw8_param(param, m, v, opt):
    f = np.float32
    b1, b2 = float(f(opt.beta1)), float(f(opt.beta2))
    lr, wd = float(f(opt.lr)), float(f(opt.weight_decay))
    with np.errstate(all="ignore"):
        denom = np.sqrt(v) * f(1.0 / math.sqrt(1.0 - b2 ** opt.t)) + f(opt.eps)
        return param * f(1.0 - lr * wd) - (m / denom) * f(lr / (1.0 - b1 ** opt.t))


def adamw8_step(grad, param, codes_m, codes_v, exps, opt, scale, tensor_id=0, round_seed=None):
    """One step without noise over a flat tensor: param, codes, exponents [blocks, 2], g."""
    m, v = decode(codes_m, exps[:, 0], "m"), decode(codes_v, exps[:, 1], "v")
    g, m, v = adamw8_moments(grad, m, v, opt, scale)
    new = adamw8_param(param, m, v, opt)
    km, kv = block_exponents(m, "m"), block_exponents(v, "v")
    rm = rv = None
    if round_seed is not None:
        rm, rv = rounding_bits(len(grad), tensor_id, opt.t, round_seed)
    return (new, encode(m, km, "m", rm), encode(v, kv, "v", rv),
            np.stack([km, kv], 1).astype(np.uint8), g)
