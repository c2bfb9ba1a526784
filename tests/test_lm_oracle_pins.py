"""Pins of the definitions of the operators between and behind the blocks (CPU only):
gradients against central differences, codes against their own rules."""

import math
from fractions import Fraction

import numpy as np
import pytest

import oracle
from oracle import lm_oracle as lo


def _differences(f, x, h=1e-6):
    g = np.zeros_like(x)
    for at in np.ndindex(x.shape):
        up, down = x.copy(), x.copy()
        up[at] += h
        down[at] -= h
        g[at] = (f(up) - f(down)) / (2 * h)
    return g


# A central difference of step h is off by h^2 / 6 of the third derivative (about 1e-12
# here) and by 2^-53 |f| / h, about 1e-9 for |f| of about 10.
DIFF = dict(rtol=0, atol=2e-8)


def test_token_gradient_is_the_slope():
    rng = np.random.default_rng(0)
    x, targets = rng.standard_normal((4, 6)) * 2, np.array([3, -1, 0, 5])
    gp, gl, ge = rng.standard_normal((3, 4))

    def f(x):
        lp, lse, h, _, _ = lo.token_logprobs(x, targets, 0.7)
        return float(gp @ lp + gl @ lse + ge @ h)

    np.testing.assert_allclose(lo.token_gradient(x, targets, 0.7, gp, gl, ge), _differences(f, x), **DIFF)


def test_token_rows_without_a_distribution():
    inf = np.inf
    x = np.array([[-inf, -inf, -inf], [0.0, -inf, 1.0], [np.nan, 0.0, 0.0], [inf, 0.0, 0.0]])
    lp, lse, h, ids, lps = lo.token_logprobs(x, np.array([1, 1, 1, 0]), 1.0, k=3)
    assert lp[0] == -inf and lse[0] == -inf and h[0] == 0 and (ids[0] == -1).all()
    assert lp[1] == -inf and ids[1].tolist() == [2, 0, -1] and lps[1, 2] == -inf
    assert math.isclose(lse[1], math.log(1 + math.e)) and h[1] > 0
    assert np.isnan(lp[2:]).all() and np.isnan(lse[2:]).all() and np.isnan(lps[2:]).all()
    g = lo.token_gradient(x, np.array([1, 1, 1, 0]), 1.0, g_logp=-np.ones(4))
    assert (g[0] == 0).all() and np.isfinite(g[1]).all() and np.isnan(g[2:]).all()


def test_alternatives_of_equal_logits_are_the_lower_tokens():
    ids, lps = lo.alternatives(np.array([1.0, 2.0, 2.0, -0.0, 0.0]), 1.0, 5)
    assert ids.tolist() == [1, 2, 0, 3, 4] and lps[0] == lps[1]


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("post", [False, True])
@pytest.mark.parametrize("gate_dim", [0, 1, 2])
def test_residual_norm_gradients_are_the_slopes(kind, post, gate_dim):
    rng = np.random.default_rng(3)
    B, S, C, eps, alpha = 2, 3, 5, 1e-3, 0.8
    x, block, dy, dr = rng.standard_normal((4, B, S, C))
    p = {n: rng.standard_normal((B, C)) for n in ("gamma", "beta", "post_gamma", "post_beta")}
    gate = {0: None, 1: rng.standard_normal(C), 2: rng.standard_normal((B, C))}[gate_dim]

    def one(i, x, block, p, gate):   # example i, with its own parameters
        r = lo.residual(x[i:i + 1], block[i:i + 1], kind, eps, alpha,
                        None if gate is None else gate, post, *((p["post_gamma"][i], p["post_beta"][i]) if post else ()))[0]
        y = lo.normed(r, kind, eps, p["gamma"][i], p["beta"][i])[0]
        return float((y * dy[i]).sum() + (r * dr[i]).sum())

    for i in range(B):
        g = gate if gate is None or gate.ndim == 1 else gate[i]
        r = lo.residual(x[i:i + 1], block[i:i + 1], kind, eps, alpha, g, post,
                        *((p["post_gamma"][i], p["post_beta"][i]) if post else ()))[0]
        got = lo.residual_norm_backward(
            r, block[i:i + 1], dy[i:i + 1], dr[i:i + 1], kind, eps, alpha, p["gamma"][i], g, post,
            *((p["post_gamma"][i], p["post_beta"][i]) if post else ()))
        for name, value in (("dx", x), ("dblock", block)):
            ref = _differences(lambda v: one(i, *((v, block) if name == "dx" else (x, v)), p, g), value)[i]
            np.testing.assert_allclose(got[name][0], ref, **DIFF)
        names = ["gamma", "beta"] + (["post_gamma", "post_beta"] if post else [])
        for name in names:
            ref = _differences(lambda v: one(i, x, block, {**p, name: v}, g), p[name])[i]
            np.testing.assert_allclose(got["d" + name][0], ref, **DIFF)
        if g is not None:
            ref = _differences(lambda v: one(i, x, block, p, v), g)
            np.testing.assert_allclose(got["dgate"][0], ref, **DIFF)


@pytest.mark.parametrize("which", ["m", "v"])
def test_codes(which):
    values = lo.code_values(which)
    assert values[0] == 0 and (np.diff(values) > 0).all() and values[-1] == 1.875
    # Each value is its own code, at several block exponents, whatever the random bits.
    for k in (lo.LOWEST[which], 127, 254):
        x = (values * 2.0 ** (k - 127)).astype(np.float32)
        exps = lo.block_exponents(x, which)
        assert exps.tolist() == [k]
        for r in (None, np.full(len(x), 65535)):
            assert lo.encode(x, exps, which, r).tolist() == list(range(len(x)))
        assert (lo.decode(np.arange(len(x), dtype=np.uint8), exps, which) == x).all()


@pytest.mark.parametrize("which", ["m", "v"])
def test_rounding_is_to_the_nearest_or_a_neighbour(which):
    rng = np.random.default_rng(5)
    x = np.exp(rng.uniform(-12, 2, 4096)).astype(np.float32) * np.float32(1e-5)
    exps = lo.block_exponents(x, which)
    values = np.unique(np.concatenate([v * 2.0 ** (exps - 127) for v in lo.code_values(which)[:, None]]))
    got = lo.decode(lo.encode(x, exps, which), exps, which).astype(np.float64)
    for i in range(0, 4096, 37):
        own = lo.code_values(which) * 2.0 ** (exps[i // 256] - 127.0)
        near = np.abs(own - x[i]).min()
        if which == "v" and got[i] == own[1] and x[i] < own[1]:
            continue   # never 0
        assert abs(got[i] - x[i]) <= near
    # Stochastic: a neighbour, and the mean over all random bits is the value (to 2^-16 of a step).
    y = x[:256]
    e = lo.block_exponents(y, which)
    for i in (0, 17, 99):
        z = np.full(65536, y[i], np.float32)
        c = lo.encode(z, np.repeat(e, 256), which, np.arange(65536)).astype(np.int64)
        assert c.max() - c.min() <= 1
        own = [Fraction(float(v)) for v in lo.code_values(which) * 2.0 ** (e[0] - 127.0)]
        mean = sum(own[int(v)] * int(n) for v, n in zip(*np.unique(c, return_counts=True))) / 65536
        step = own[int(c.min()) + 1] - own[int(c.min())]
        if not (which == "v" and c.min() <= 1):
            assert abs(mean - Fraction(float(y[i]))) <= step / 65536
    assert values[0] == 0


def test_block_exponents_of_what_is_not_finite_and_of_nothing():
    x = np.zeros(700, np.float32)
    x[300] = np.inf
    x[600] = np.nan
    assert lo.block_exponents(x, "m").tolist() == [32, 255, 255]
    assert np.isnan(lo.decode(np.zeros(700, np.uint8), np.array([32, 255, 32]), "m"))[256:512].all()
    x = np.full(1, 1.8751 * 2.0 ** 127, np.float32)
    assert lo.block_exponents(x, "m").tolist() == [255]
    # A subnormal largest magnitude.
    x = np.full(1, 1e-40, np.float32)
    assert lo.block_exponents(x, "v").tolist() == [48]
    assert lo.encode(x, np.array([48]), "v").tolist() == [1]


def test_adamw8_step_is_adamw_between_the_codes():
    """Where the moments before and after are values of codes, the step is the float64 one."""
    rng = np.random.default_rng(6)
    n = 700
    cfg = oracle.AdamWConfig(lr=1e-3, beta1=0.5, beta2=0.75, eps=1e-8, weight_decay=0.1, t=3)
    param, grad = rng.standard_normal(n).astype(np.float32), rng.standard_normal(n).astype(np.float32)
    cm, cv = rng.integers(0, 256, n).astype(np.uint8), rng.integers(8, 256, n).astype(np.uint8)
    exps = np.array([[120, 110]] * 3, np.uint8)
    m, v = lo.decode(cm, exps[:, 0], "m"), lo.decode(cv, exps[:, 1], "v")
    new, qm, qv, e, g = lo.adamw8_step(grad, param, cm, cv, exps, cfg, 0.5)
    g64 = 0.5 * grad.astype(np.float64)
    m64, v64 = 0.5 * m + 0.5 * g64, 0.75 * v + 0.25 * g64 * g64
    th = param * (1 - 1e-3 * 0.1) - 1e-3 * (m64 / (1 - 0.5 ** 3)) / (np.sqrt(v64 / (1 - 0.75 ** 3)) + 1e-8)
    # A dozen float32 roundings of the update (at most 1e-3 m / sqrt(v)) and one of the parameter.
    tol = 2.0 ** -24 * (2 * np.abs(th) + 12 * np.abs(th - param) + 2e-4 * np.abs(param)) + 1e-12
    assert (np.abs(new - th) <= tol).all()
    back = lo.decode(qm, e[:, 0], "m")
    assert (np.abs(back - m64) <= np.maximum(2.0 ** -4 * np.abs(m64), 2.0 ** -17 * np.abs(m64).max())).all()
    assert np.array_equal(g, (0.5 * grad).astype(np.float32))
