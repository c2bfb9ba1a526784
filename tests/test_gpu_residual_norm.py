"""The residual sum with the norms on both sides of it, and its gradients, on the GPU
against the float64 definitions.

Bounds, with u = 2^-24: a mean over C values adds them over at most 16 a thread and then
over threads and waves, so it is off by at most 32 u of the mean of their sizes; the sum
of squared deviations by 36 u of itself (and the mean's error squared); rstd by half of
that and a few roundings, 24 u. r is one rounding of its dtype after three of float32, and
y is formed from the r that was stored, which the tests read back. The backward pass is
bounded term by term from the same parts: a normed value is off by e1 = 32 u (|mean part|
+ |value|), a row mean of products by 40 u of the mean of their sizes, and a sum over S
positions by (S + 16) u of the sum of its terms' sizes. bf16 outputs add 2^-8 of the value.
"""

import numpy as np
import pytest

from oracle import lm_oracle as lo

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
AFFINE = ("gamma", "beta", "gate", "post_gamma", "post_beta")


@pytest.fixture(autouse=True)
def _announce(request):
    print(f"[gpu] start {request.node.name}", flush=True)
    yield


def _torch():
    import torch
    return torch


def _tensor(x, dtype="f32"):
    torch = _torch()
    return torch.from_numpy(np.ascontiguousarray(x, np.float32)).to(
        {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]).cuda()


def _wide(t):
    return None if t is None else t.double().cpu().numpy()


def _half(dtype, v):
    return 2.0 ** -8 * np.abs(v) if dtype == "bf16" else 0.0


def _case(B, S, C, dtype, seed, gate, post, beta=True, shift=0.0):
    rng = np.random.default_rng(seed)
    c = {"x": _tensor(rng.standard_normal((B, S, C)) + shift, dtype),
         "block": _tensor(0.7 * rng.standard_normal((B, S, C)) - 0.5 * shift, dtype),
         "dy": _tensor(rng.standard_normal((B, S, C)), dtype),
         "dr": _tensor(rng.standard_normal((B, S, C)), dtype)}
    p = {n: _tensor(1.0 + 0.3 * rng.standard_normal(C)) for n in ("gamma", "post_gamma")}
    p |= {n: _tensor(0.3 * rng.standard_normal(C)) for n in ("beta", "post_beta")}
    p["gate"] = None if gate == 0 else _tensor(0.5 + 0.3 * rng.standard_normal((B, C) if gate == 2 else C))
    if not post:
        p["post_gamma"] = p["post_beta"] = None
    if not beta:
        p["beta"] = p["post_beta"] = None
    return c, p


def _desc(dp, c, p, kind, post, alpha=0.8, eps=1e-5):
    return dp.make_residual_norm(c["x"], kind=kind, post=post, residual_scale=alpha, eps=eps, **p)


def _forward(dp, c, desc, block=True, stats=True):
    torch = _torch()
    r, y = torch.full_like(c["x"], 7.0), torch.full_like(c["x"], 7.0)
    st = torch.full((desc.B, desc.S, 4), 7.0, device="cuda") if stats else None
    dp.dpsgd_residual_norm_forward(desc, c["x"], c["block"] if block else None, r, y, st)
    torch.cuda.synchronize()
    return r, y, st


def _norm_parts(v, kind, eps):
    """The normed rows, rstd, and the bound of a normed value's error."""
    vh, mean, rstd = lo.norm_rows(v, kind, eps)
    em = (32 * U * np.abs(v).mean(-1, keepdims=True) + U * np.abs(mean)) if kind == "layer" else 0.0
    e = (em + 2 * U * (np.abs(v) + np.abs(mean))) * rstd + (26 * U + (em * rstd) ** 2) * np.abs(vh)
    return vh, mean, rstd, e, em


def check_forward(c, p, kind, post, got, dtype, block=True, alpha=0.8, eps=1e-5):
    r, y, st = got
    a, f = float(np.float32(alpha)), {n: _wide(v) for n, v in p.items()}
    eps = float(np.float32(eps))
    x, b = _wide(c["x"]), _wide(c["block"]) if block else None
    ref, pm, pr = lo.residual(x, b, kind, eps, a, f["gate"], post, f["post_gamma"], f["post_beta"])
    gate = np.abs(lo._gate(f["gate"]))
    tol = 2 * U * np.abs(a * x)
    if block:
        u, eu = b, 0.0
        if post:
            vh, _, rstd, e, em = _norm_parts(b, kind, eps)
            u = lo._affine(vh, f["post_gamma"], f["post_beta"])
            eu = e * (1.0 if f["post_gamma"] is None else np.abs(f["post_gamma"])) + 2 * U * np.abs(u)
            assert (np.abs(_wide(st)[..., 2:3] - pm) <= em).all()
            assert (np.abs(_wide(st)[..., 3:4] / pr - 1) <= 26 * U + (em * rstd) ** 2).all()
        tol = tol + gate * eu + 2 * U * (gate * np.abs(u) + np.abs(ref))
    if st is not None and not post:
        assert bool((st[..., 2:] == 0).all())
    tol = tol + _half(dtype, np.abs(ref) + tol)
    assert (np.abs(_wide(r) - ref) <= tol).all(), f"r: {np.max(np.abs(_wide(r) - ref) / tol)}"
    yref, mean, rstd = lo.normed(_wide(r), kind, eps, f["gamma"], f["beta"])
    vh, _, _, e, em = _norm_parts(_wide(r), kind, eps)
    tol = e * (1.0 if f["gamma"] is None else np.abs(f["gamma"])) + 3 * U * np.abs(yref)
    tol = tol + _half(dtype, np.abs(yref) + tol) + 1e-38
    assert (np.abs(_wide(y) - yref) <= tol).all(), f"y: {np.max(np.abs(_wide(y) - yref) / tol)}"
    if st is not None:
        assert (np.abs(_wide(st)[..., 0:1] - mean) <= em).all()
        assert (np.abs(_wide(st)[..., 1:2] / rstd - 1) <= 26 * U + (em * rstd) ** 2).all()


def _backward(dp, c, desc, r, st, names, block=True, with_dr=True, dx=True, in_place=False):
    torch = _torch()
    ws = torch.empty(dp.dpsgd_residual_norm_workspace_bytes(desc), dtype=torch.uint8, device="cuda")
    dy, dr = c["dy"].clone(), c["dr"].clone() if with_dr else None
    out = {"d" + n: torch.full((desc.B, desc.C), 7.0, device="cuda") for n in names}
    if dx:
        out["dx"] = dr if in_place else torch.full_like(r, 7.0)
    if block:
        out["dblock"] = dy if in_place else torch.full_like(r, 7.0)
    dp.dpsgd_residual_norm_backward(desc, c["block"] if block else None, r, dy, dr, st, workspace=ws, **out)
    torch.cuda.synchronize()
    return out


def _d_bound(g, eg, vh, eh, rstd, kind):
    """Bound of the error of D(g, vh) = rstd (g - mean g - vh mean(g vh)) for errors eg, eh."""
    gv = g * vh
    e2 = (eg * np.abs(vh) + np.abs(g) * eh).mean(-1, keepdims=True) + 40 * U * np.abs(gv).mean(-1, keepdims=True)
    m2 = gv.mean(-1, keepdims=True)
    e1 = eg.mean(-1, keepdims=True) + 40 * U * np.abs(g).mean(-1, keepdims=True) if kind == "layer" else 0.0
    m1 = g.mean(-1, keepdims=True) if kind == "layer" else 0.0
    size = np.abs(g) + np.abs(m1) + np.abs(vh * m2)
    return rstd * (eg + e1 + eh * np.abs(m2) + np.abs(vh) * e2 + 32 * U * size)


def check_backward(c, p, kind, post, r, out, dtype, block=True, with_dr=True, alpha=0.8, eps=1e-5):
    a, f = float(np.float32(alpha)), {n: _wide(v) for n, v in p.items()}
    eps = float(np.float32(eps))
    r, dy = _wide(r), _wide(c["dy"])
    b, dr = _wide(c["block"]) if block else None, _wide(c["dr"]) if with_dr else None
    ref = lo.residual_norm_backward(r, b, dy, dr, kind, eps, a, f["gamma"], f["gate"], post,
                                    f["post_gamma"], f["post_beta"])
    one = lambda v: 1.0 if v is None else v  # noqa: E731
    S = r.shape[1]

    def sums(terms, errors):
        return errors.sum(1) + (S + 16) * U * np.abs(terms).sum(1)

    rh, _, rstd, eh, _ = _norm_parts(r, kind, eps)
    g = dy * one(f["gamma"])
    eR = _d_bound(g, U * np.abs(g), rh, eh, rstd, kind)
    dR = ref["dx"] / a
    eR = eR + 3 * U * np.abs(dR) + (0.0 if dr is None else U * np.abs(dr))
    tol = {"dgamma": sums(dy * rh, np.abs(dy) * eh), "dbeta": sums(dy, 0.0 * dy), "dx": np.abs(a) * eR + 2 * U * np.abs(ref["dx"])}
    if block:
        gate = lo._gate(f["gate"])
        dU, eU = gate * dR, np.abs(gate) * (eR + U * np.abs(dR))
        u, eu = b, np.zeros_like(b)
        if post:
            bh, _, brstd, be, _ = _norm_parts(b, kind, eps)
            u = lo._affine(bh, f["post_gamma"], f["post_beta"])
            eu = np.abs(one(f["post_gamma"])) * be + 2 * U * np.abs(u)
            h = dU * one(f["post_gamma"])
            tol["dblock"] = _d_bound(h, np.abs(one(f["post_gamma"])) * eU + U * np.abs(h), bh, be, brstd, kind)
            tol["dpost_gamma"] = sums(dU * bh, eU * np.abs(bh) + np.abs(dU) * be)
            tol["dpost_beta"] = sums(dU, eU)
        else:
            tol["dblock"] = eU
        tol["dgate"] = sums(dR * u, eR * np.abs(u) + np.abs(dR) * eu)
    for name, t in out.items():
        bound = tol[name]
        if name in ("dx", "dblock"):
            bound = bound + _half(dtype, np.abs(ref[name]) + bound)
        err = np.abs(_wide(t) - ref[name])
        assert (err <= bound + 1e-38).all(), f"{name}: {np.max(err / (bound + 1e-38))}"


SHAPES = [   # B, S, C
    (1, 1, 1), (2, 1, 2), (1, 3, 3), (3, 5, 8), (2, 7, 30), (8, 1, 768), (1, 9, 63), (2, 65, 64),
    (5, 3, 100), (37, 61, 250), (2, 130, 513), (1, 300, 1024), (3, 4, 1032), (2, 33, 2051),
    (1, 17, 4096), (2, 3, 4100), (1, 5, 8192), (1, 3, 8200), (2, 2, 12289), (1, 3, 16383), (2, 3, 16384),
    (300, 2, 48), (3000, 1, 16), (1, 2100, 24), (70, 40, 768),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("at", range(len(SHAPES)))
def test_forward_and_backward(dp, at, dtype):
    """Every size; norms, gates and biases in turn."""
    B, S, C = SHAPES[at]
    for turn in (at, at + 5):
        kind, post, gate = ("layer", "rms")[turn % 2], turn // 2 % 2 == 0, turn % 3
        c, p = _case(B, S, C, dtype, turn, gate, post, beta=turn % 5 != 0)
        desc = _desc(dp, c, p, kind, post)
        got = _forward(dp, c, desc)
        check_forward(c, p, kind, post, got, dtype)
        names = [n for n in AFFINE if (post or not n.startswith("post"))]
        out = _backward(dp, c, desc, got[0], got[2], names)
        check_backward(c, p, kind, post, got[0], out, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("post", [False, True])
@pytest.mark.parametrize("gate", [0, 1, 2])
def test_every_combination(dp, kind, post, gate, dtype):
    c, p = _case(3, 21, 96, dtype, 5, gate, post, shift=3.0)
    desc = _desc(dp, c, p, kind, post, alpha=-1.25)
    got = _forward(dp, c, desc)
    check_forward(c, p, kind, post, got, dtype, alpha=-1.25)
    names = [n for n in AFFINE if (post or not n.startswith("post"))]
    for with_dr in (True, False):
        out = _backward(dp, c, desc, got[0], got[2], names, with_dr=with_dr)
        check_backward(c, p, kind, post, got[0], out, dtype, with_dr=with_dr, alpha=-1.25)
    out = _backward(dp, c, desc, got[0], got[2], names, in_place=True)
    check_backward(c, p, kind, post, got[0], out, dtype, alpha=-1.25)
    # Frozen parameters, and each gradient alone.
    for some in ([], *([n] for n in names)):
        alone = _backward(dp, c, desc, got[0], got[2], some, dx=False)
        for n, t in alone.items():
            assert _torch().equal(t, out[n]), n


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("form", ["bare", "gated", "post"])
@pytest.mark.parametrize("C", [8200, 12292, 16382, 16383, 16384])
def test_widest_rows(dp, C, form, dtype):
    """Rows of 1024 threads whose sums are in LDS: every vector width; three workgroups an
    example with two rows each, the last with one."""
    B, S = 40, 5
    post, gate, kind = form == "post", {"bare": 0, "gated": 2, "post": 1}[form], ("layer", "rms")[C % 4 == 0]
    c, p = _case(B, S, C, dtype, C, gate, post)
    desc = _desc(dp, c, p, kind, post)
    got = _forward(dp, c, desc)
    check_forward(c, p, kind, post, got, dtype)
    names = [n for n in AFFINE if (post or not n.startswith("post")) and (gate or n != "gate")]
    for in_place in (False, True):
        out = _backward(dp, c, desc, got[0], got[2], names, in_place=in_place)
        check_backward(c, p, kind, post, got[0], out, dtype)
    if form == "bare":
        got = _forward(dp, c, desc, block=False)
        out = _backward(dp, c, desc, got[0], got[2], ["gamma", "beta"], block=False, with_dr=False)
        check_backward(c, p, kind, post, got[0], out, dtype, block=False, with_dr=False)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,S,C", [(2, 9, 40), (4, 33, 768), (1, 2, 5000)])
def test_without_a_block(dp, B, S, C, dtype):
    """The first norm of a model: r is x (scaled), nothing is added."""
    torch = _torch()
    c, p = _case(B, S, C, dtype, 9, 0, False)
    for alpha in (1.0, 0.5):
        desc = _desc(dp, c, p, "layer", False, alpha=alpha)
        got = _forward(dp, c, desc, block=False)
        check_forward(c, p, "layer", False, got, dtype, block=False, alpha=alpha)
        out = _backward(dp, c, desc, got[0], got[2], ["gamma", "beta"], block=False)
        check_backward(c, p, "layer", False, got[0], out, dtype, block=False, alpha=alpha)
    desc = _desc(dp, c, p, "layer", False, alpha=1.0)
    r, y, _ = _forward(dp, c, desc, block=False)
    assert torch.equal(r, c["x"])
    again = torch.empty_like(y)
    dp.dpsgd_residual_norm_forward(desc, c["x"], None, None, again, None)
    assert torch.equal(again, y)


def test_in_place_and_without_stats(dp):
    torch = _torch()
    c, p = _case(3, 17, 260, "bf16", 4, 1, True)
    desc = _desc(dp, c, p, "rms", True)
    r, y, _ = _forward(dp, c, desc)
    x, block = c["x"].clone(), c["block"].clone()
    dp.dpsgd_residual_norm_forward(desc, x, block, x, block, None)
    assert torch.equal(x, r) and torch.equal(block, y)


def test_more_axes_than_three(dp):
    c, p = _case(2, 12, 36, "f32", 4, 2, True)
    desc = _desc(dp, c, p, "layer", True)
    r, y, st = _forward(dp, c, desc)
    c4 = {n: v.view(2, 3, 4, 36) for n, v in c.items()}
    desc4 = _desc(dp, c4, p, "layer", True)
    r4, y4, st4 = _forward(dp, c4, desc4)
    assert _torch().equal(r4.view(2, 12, 36), r) and _torch().equal(y4.view(2, 12, 36), y)


def test_rows_of_one_value_and_of_nan(dp):
    """A row without spread is beta; a row with a NaN is NaN, and only that row; an
    example's gradients are its own."""
    torch = _torch()
    c, p = _case(3, 6, 129, "f32", 8, 0, False)
    c["x"][0, 1], c["block"][0, 1] = 2.0, 0.5
    c["x"][1, 2, 7] = float("nan")
    desc = _desc(dp, c, p, "layer", False, alpha=1.0)
    r, y, st = _forward(dp, c, desc)
    assert float((y[0, 1] - p["beta"]).abs().max()) <= 1e-4
    assert bool(torch.isnan(y[1, 2]).all())
    y[1, 2] = 0.0
    assert bool(torch.isfinite(y).all())
    out = _backward(dp, c, desc, r, st, ["gamma", "beta"])
    assert bool(torch.isnan(out["dgamma"][1]).all())
    for i in (0, 2):
        assert all(bool(torch.isfinite(out[n][i]).all()) for n in out)
    assert bool(torch.isnan(out["dx"][1, 2]).all())


@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_rows_of_extreme_sizes(dp, kind):
    """Rows whose squares leave float32 at either end: the norm's 1 / sqrt is 0 (of
    infinity) or that of eps, never NaN."""
    torch = _torch()
    c, p = _case(1, 4, 96, "f32", 8, 0, False, beta=False)
    sign = torch.ones(96, device="cuda")
    sign[1::2] = -1.0
    for row, size in enumerate((1e25, 1e-25, 1e-42, 1.0)):
        c["x"][0, row], c["block"][0, row] = sign * size, 0.0
    desc = _desc(dp, c, p, kind, False, alpha=1.0, eps=1e-40)
    r, y, st = _forward(dp, c, desc)
    assert torch.equal(r, c["x"]) and bool(torch.isfinite(y).all())
    gamma = p["gamma"]
    assert bool((st[0, 0, 1] == 0).all()) and bool((y[0, 0] == 0).all())
    # The squares of 1e-25 and below are 0 beside eps in float32.
    for row, size in ((1, 1e-25), (2, 1e-42)):
        ref = sign * float(np.float32(size)) * 1e20 * gamma
        assert float(((y[0, row] - ref).abs() / ref.abs()).max()) <= 1e-3
    assert float((y[0, 3] - sign * gamma).abs().max()) <= 32 * U


def test_same_bits_on_another_stream_and_in_a_graph(dp):
    torch = _torch()
    c, p = _case(3, 200, 768, "bf16", 2, 2, True)
    desc = _desc(dp, c, p, "rms", True)
    names = list(AFFINE)
    r, y, st = _forward(dp, c, desc)
    out = _backward(dp, c, desc, r, st, names)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        r2, y2, st2 = _forward(dp, c, desc)
        out2 = _backward(dp, c, desc, r2, st2, names)
    assert torch.equal(r, r2) and torch.equal(y, y2) and torch.equal(st, st2)
    assert all(torch.equal(out[n], out2[n]) for n in out)
    torch.cuda.current_stream().wait_stream(side)
    ws = torch.empty(dp.dpsgd_residual_norm_workspace_bytes(desc), dtype=torch.uint8, device="cuda")

    def both():
        dp.dpsgd_residual_norm_forward(desc, c["x"], c["block"], r2, y2, st2)
        dp.dpsgd_residual_norm_backward(desc, c["block"], r2, c["dy"], c["dr"], st2, workspace=ws, **out2)

    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for seed in range(3):
        new, _ = _case(3, 200, 768, "bf16", 60 + seed, 2, True)
        for n in c:
            c[n].copy_(new[n])
        for t in (r2, y2, st2, *out2.values()):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (r2, y2, st2, *out2.values())]
        both()
        torch.cuda.synchronize()
        for a, b in zip(got, (r2, y2, st2, *out2.values())):
            assert torch.equal(a, b)


def test_per_example_gradients_go_through_the_norm_and_clip(dp):
    """dgamma and dgate as layers: their norms and clipped sums."""
    torch = _torch()
    c, p = _case(5, 11, 72, "f32", 3, 1, False)
    desc = _desc(dp, c, p, "layer", False)
    r, y, st = _forward(dp, c, desc)
    out = _backward(dp, c, desc, r, st, ["gamma", "gate"])
    ones = torch.ones(5, device="cuda")
    Ls = [dp.affine_layer(ones, out["dgamma"], 0), dp.affine_layer(ones, out["dgate"], 1)]
    buf = dp.alloc_step(Ls)
    dp.run_clipped_sum(Ls, buf, 6.0)
    torch.cuda.synchronize()
    both = torch.cat([out["dgamma"], out["dgate"]], 1).double()
    n = both.norm(dim=1)
    f = torch.clamp(6.0 / n, max=1.0)
    ref = (both * f[:, None]).sum(0)
    got = torch.cat([buf.grads[0].view(-1), buf.grads[1].view(-1)]).double()
    assert float((buf.norms_sq.double().sqrt() / n - 1).abs().max()) <= 200 * U
    assert float((got - ref).abs().max()) <= 400 * U * float((both.abs() * f[:, None]).sum(0).max())
