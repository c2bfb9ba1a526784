"""Log probabilities of tokens, their gradient, and the loss on the GPU against the
float64 definitions.

Bounds, with u = 2^-24, zm the largest finite |scale x| of a row and n its length. z is
one rounding (u zm), z - m carries two of them and its own (u 2 zm), and the exponential's
argument and value are off by 2 u 2 zm + 4 u relative to the exponential: R = (10 zm + 4) u
at most. A sum of n positive terms over threads and waves adds (n / 64 + 32) u. So S is off
by K u of itself with K = 10 zm + n / 64 + 40, ln S by that absolutely, and lse and logprob
by that and a few roundings of values of at most 3 zm + ln n: L = K + 8 zm + 8 ln n + 8.
The entropy's sum has terms p |z - m| of at most 2 zm in all (and at most 1 + ln n on
average weight): E = L (2 + ln n) bounds it. A gradient entry is p off by 2 K u of itself,
times a factor, and a few roundings of the factor's terms. bf16 gradients add 2^-8 of the
value.
"""

import math

import numpy as np
import pytest

from oracle import lm_oracle as lo

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(autouse=True)
def _announce(request):
    print(f"[gpu] start {request.node.name}", flush=True)
    yield


def _torch():
    import torch
    return torch


def _tensor(x, dtype):
    torch = _torch()
    return torch.from_numpy(np.ascontiguousarray(x, np.float32)).to(
        {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]).cuda()


def _wide(t):
    return t.double().cpu().numpy()


def _bounds(x, scale):
    """Per row: K, L, E of the module's text, in u."""
    n = x.shape[1]
    z = np.where(np.isfinite(x), np.abs(scale * x), 0.0).max(1)
    K = 10 * z + n / 64 + 40
    L = K + 8 * z + 8 * math.log(n) + 8
    return K, L, L * (2 + math.log(n))


def _close(got, ref, tol, what):
    got, ref = np.asarray(got, np.float64), np.asarray(ref, np.float64)
    same = (got == ref) | (np.isnan(got) & np.isnan(ref))
    with np.errstate(invalid="ignore"):
        ok = same | (np.abs(got - ref) <= tol)
    assert ok.all(), f"{what}: {np.argwhere(~ok)[:4].tolist()}, {got[~ok][:4]} for {ref[~ok][:4]}"


def _logits(B, T, V, dtype, seed, spread=2.5):
    rng = np.random.default_rng(seed)
    return _tensor(rng.standard_normal((B, T, V)) * spread, dtype)


def _targets(B, T, V, seed, ragged):
    rng = np.random.default_rng(seed + 1)
    t = rng.integers(0, V, (B, T))
    if ragged:
        t = np.where(rng.random((B, T)) < 0.3, rng.choice([-1, V, -2 ** 31, 2 ** 31 - 1], (B, T)), t)
    return t


def _ws(dp, desc, k=0):
    torch = _torch()
    return torch.empty(dp.dpsgd_token_workspace_bytes(desc, k), dtype=torch.uint8, device="cuda")


def run_logprobs(dp, x, targets, scale, k):
    torch = _torch()
    B, T, _ = x.shape
    desc = dp.make_logits(x, targets, scale)
    out = {n: torch.full((B, T), 7.0, device="cuda") for n in ("lse", "entropy")}
    if targets is not None:
        out["logprobs"] = torch.full((B, T), 7.0, device="cuda")
    if k:
        out["top_ids"] = torch.full((B, T, k), 7, dtype=torch.int64, device="cuda")
        out["top_logprobs"] = torch.full((B, T, k), 7.0, device="cuda")
    dp.dpsgd_token_logprobs(desc, x, workspace=_ws(dp, desc, k), **out)
    torch.cuda.synchronize()
    return desc, out


def check_logprobs(x, targets, scale, k, out):
    N, V = x.shape[0] * x.shape[1], x.shape[2]
    x64 = _wide(x).reshape(N, V)
    s = float(np.float32(scale))
    t = None if targets is None else targets.reshape(-1)
    lp, lse, h, ids, lps = lo.token_logprobs(x64, t, s, k)
    _, L, E = _bounds(x64, s)
    if t is not None:
        _close(_wide(out["logprobs"]).reshape(N), lp, L * U, "logprobs")
    _close(_wide(out["lse"]).reshape(N), lse, L * U, "lse")
    _close(_wide(out["entropy"]).reshape(N), h, E * U, "entropy")
    if k:
        assert np.array_equal(out["top_ids"].cpu().numpy().reshape(N, k), ids)
        _close(_wide(out["top_logprobs"]).reshape(N, k), lps, L[:, None] * U, "top_logprobs")


SHAPES = [   # B, T, V, k
    (1, 1, 1, 1), (3, 2, 2, 5), (128, 1, 4, 2), (2, 3, 7, 64), (5, 1, 63, 3), (4, 2, 64, 64),
    (3, 1, 65, 8), (2, 2, 255, 5), (2, 3, 1000, 20), (70, 1, 1000, 0), (2, 1, 1023, 63),
    (1, 2, 4099, 33), (3, 2, 8191, 1), (2, 1, 32003, 20), (1, 3, 50257, 5), (1, 1, 65537, 64),
    (1, 2, 131072, 20), (1, 1, 131077, 9), (2, 1, 300001, 64), (600, 2, 130, 3),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,T,V,k", SHAPES)
def test_logprobs(dp, B, T, V, k, dtype):
    torch = _torch()
    x = _logits(B, T, V, dtype, V + k)
    targets = _targets(B, T, V, V, ragged=V % 2 == 1)
    wide = torch.from_numpy(targets).cuda()
    desc, out = run_logprobs(dp, x, wide if V % 3 else wide.to(torch.int32), 0.75, k)
    check_logprobs(x, targets, 0.75, k, out)


def special_rows(V, rng):
    """Rows where a distribution is at an end of its range, and what they are."""
    inf, base = np.inf, rng.standard_normal(V)
    rows = {"masked": np.full(V, -inf), "equal": np.full(V, 1.5), "zeros": np.where(np.arange(V) % 2, 0.0, -0.0),
            "lowest": np.full(V, -3.0e38), "one left": np.full(V, -inf), "one high": np.full(V, -3.0e38),
            "nan": base.copy(), "all nan": np.full(V, np.nan), "inf": base.copy(),
            "nan among masked": np.full(V, -inf), "ascending": np.linspace(-8, 8, V),
            "descending": np.linspace(8, -8, V), "far": 80.0 * base, "ties": np.round(2 * base),
            "half masked": np.where(rng.random(V) < 0.5, -inf, base), "few left": np.full(V, -inf)}
    at = int(rng.integers(V))
    rows["one left"][at] = -5.0
    rows["one high"][at] = 3.0
    rows["nan"][at] = np.nan
    rows["inf"][at] = inf
    rows["nan among masked"][at] = np.nan
    rows["few left"][rng.integers(0, V, 3)] = 2.0
    # The largest ones near each other, and in steps that one thread's entries may have.
    near = base.copy()
    near[:min(V, 70)] += 9.0
    strided = base.copy()
    strided[::256] += 9.0
    return {**rows, "near": near, "strided": strided}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [5, 64, 1000, 8200, 33000, 140001])
def test_special_rows(dp, V, dtype):
    torch = _torch()
    rng = np.random.default_rng(V)
    rows = special_rows(V, rng)
    x = _tensor(np.stack(list(rows.values()))[None], dtype)
    # A target that the row has masked, and one that it has not.
    targets = rng.integers(0, V, (1, len(rows)))
    for k in (0, 5, 64):
        desc, out = run_logprobs(dp, x, torch.from_numpy(targets).cuda(), 0.75, k)
        check_logprobs(x, targets, 0.75, k, out)
    w = np.full((1, len(rows)), 0.5)
    check_loss(dp, x, targets, w, 0.75)
    check_backward(dp, x, targets, 0.75, 1)


@pytest.mark.parametrize("V", [7, 900, 9001, 140001])
def test_scales_that_leave_float32(dp, V):
    """z = scale x beyond float32: +inf makes a row NaN, -inf is a masked token, and a row
    of nothing else has no distribution; products far from 0 keep their order."""
    torch = _torch()
    rng = np.random.default_rng(V)
    base = rng.standard_normal(V).astype(np.float32)
    rows = {"over": base.copy(), "under": base * np.float32(0.1), "all under": np.full(V, -2.0e38, np.float32),
            "all under but one": np.full(V, -2.0e38, np.float32), "zeros": np.zeros(V, np.float32),
            "large": base * np.float32(3.0e35)}
    rows["over"][V // 2] = 2.0e38
    rows["under"][V // 3] = -2.0e38
    rows["all under but one"][1] = -1.0e37
    x = _tensor(np.stack(list(rows.values()))[None], "f32")
    targets = np.full((1, len(rows)), V // 3)
    for scale in (8.0, 1.0):
        # The products in float32, as they are defined.
        with np.errstate(over="ignore"):
            z = np.float32(scale) * x.cpu().numpy()[0]
        for k in (0, 3):
            _, out = run_logprobs(dp, x, torch.from_numpy(targets).cuda(), scale, k)
            lp, lse, h, ids, lps = lo.token_logprobs(z.astype(np.float64), targets[0], 1.0, k)
            _, L, E = _bounds(z.astype(np.float64), 1.0)
            _close(_wide(out["logprobs"])[0], lp, L * U, "logprobs")
            _close(_wide(out["lse"])[0], lse, L * U, "lse")
            _close(_wide(out["entropy"])[0], h, E * U, "entropy")
            if k:
                for i, name in enumerate(rows):
                    if name not in ("under", "all under but one"):   # whose z are -inf where x is not
                        assert np.array_equal(out["top_ids"].cpu().numpy()[0, i], ids[i]), name
        desc = dp.make_logits(x, torch.from_numpy(targets).cuda(), scale)
        dx = torch.empty_like(x)
        dp.dpsgd_token_loss(desc, x, dx, workspace=_ws(dp, desc))
        with np.errstate(over="ignore"):
            ref = scale * lo.token_gradient(z.astype(np.float64), targets[0], 1.0, g_logp=-np.ones(len(rows)))
        got = _wide(dx)[0]
        for i, name in enumerate(rows):
            K, L, _ = _bounds(z[i:i + 1].astype(np.float64), 1.0)
            p = np.abs(ref[i]) + (np.arange(V) == V // 3) * scale
            _close(got[i], ref[i], p * (2 * (K + L) + 8) * U, name)


def test_no_targets(dp):
    x = _logits(2, 3, 517, "bf16", 3)
    _, out = run_logprobs(dp, x, None, 1.0, 4)
    check_logprobs(x, None, 1.0, 4, out)


def _gradient_close(got, x64, t, s, factors, ref, dtype):
    """factors: the sizes of the three upstream gradients [N]."""
    K, L, E = _bounds(x64, s)
    p = np.zeros_like(x64)
    for i, row in enumerate(x64):
        lse, lp, _ = lo.token_row(row, s)
        p[i] = np.exp(lp) if np.isfinite(lse) else 0.0
    gp, gl, ge = (np.abs(f)[:, None] for f in factors)
    l = np.where(p > 0, -np.log(np.maximum(p, 1e-300)), 0.0)
    H = np.array([abs(lo.token_row(row, s)[2]) for row in x64])[:, None]
    H = np.where(np.isfinite(H), H, 0.0)
    size = gp + gl + ge * (l + H)
    tol = s * U * (p * size * (2 * (K + L)[:, None] + 8) + p * ge * 2 * (L + E)[:, None] + 4 * gp * (ref != 0))
    if dtype == "bf16":
        tol = tol + 2.0 ** -8 * np.where(np.isfinite(ref), np.abs(ref) + tol, 0.0)
    # Below float32's normal numbers, a step of its or bf16's grid.
    _close(got, ref, tol + 1e-38, "gradient")


def check_loss(dp, x, targets, weights, scale, in_place=False, dlogits=None):
    torch = _torch()
    B, T, V = x.shape
    x64, s = _wide(x).reshape(B * T, V), float(np.float32(scale))
    desc = dp.make_logits(x, torch.from_numpy(targets).cuda(), scale)
    w = None if weights is None else _tensor(weights, "f32")
    dlogits = x if in_place else (torch.full_like(x, 7.0) if dlogits is None else dlogits)
    losses, logprobs = torch.full((B,), 7.0, device="cuda"), torch.full((B, T), 7.0, device="cuda")
    dp.dpsgd_token_loss(desc, x, dlogits, losses=losses, weights=w, logprobs=logprobs,
                        workspace=_ws(dp, desc))
    torch.cuda.synchronize()
    t = targets.reshape(-1)
    w64 = np.ones(B * T) if weights is None else weights.astype(np.float32).astype(np.float64).reshape(-1)
    w64 = np.where((t >= 0) & (t < V), w64, 0.0)
    lp = lo.token_logprobs(x64, t, s)[0]
    _, L, _ = _bounds(x64, s)
    _close(_wide(logprobs).reshape(-1), lp, L * U, "logprobs")
    with np.errstate(invalid="ignore"):
        terms = np.where(w64 != 0.0, -w64 * lp, 0.0).reshape(B, T)
        tol = (np.abs(w64) * L * U).reshape(B, T).sum(1) + (T / 64 + 16) * U * np.where(
            np.isfinite(terms), np.abs(terms), 0.0).sum(1)
        _close(_wide(losses), terms.sum(1), tol, "losses")
    ref = lo.token_gradient(x64, t, s, g_logp=-w64)
    dtype = "bf16" if x.dtype == torch.bfloat16 else "f32"
    zero = np.zeros(B * T)
    _gradient_close(_wide(dlogits).reshape(B * T, V), x64, t, s, (w64, zero, zero), ref, dtype)
    return losses, dlogits


def check_backward(dp, x, targets, scale, seed, parts="ple", in_place=False):
    torch = _torch()
    B, T, V = x.shape
    x64, s = _wide(x).reshape(B * T, V), float(np.float32(scale))
    rng = np.random.default_rng(seed)
    g = {n: (rng.standard_normal((B, T)) if n in parts else None) for n in "ple"}
    for v in g.values():
        if v is not None and T > 1:
            v[:, -1] = 0.0
    dev = torch.from_numpy(targets).cuda()
    desc, out = run_logprobs(dp, x, dev, scale, 0)
    dx = x if in_place else torch.full_like(x, 7.0)
    up = {n: None if v is None else _tensor(v, "f32") for n, v in g.items()}
    dp.dpsgd_token_logprobs_backward(desc, x, out["lse"], dx, entropy=out["entropy"],
                                     grad_logprobs=up["p"], grad_lse=up["l"], grad_entropy=up["e"])
    torch.cuda.synchronize()
    f = [np.zeros(B * T) if g[n] is None else np.float32(g[n]).astype(np.float64).reshape(-1) for n in "ple"]
    t = targets.reshape(-1)
    ref = lo.token_gradient(x64, t, s, *f)
    _gradient_close(_wide(dx).reshape(B * T, V), x64, t, s, f, ref,
                    "bf16" if x.dtype == torch.bfloat16 else "f32")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,T,V,k", SHAPES)
def test_loss(dp, B, T, V, k, dtype):
    x = _logits(B, T, V, dtype, V + 3)
    targets = _targets(B, T, V, V + 3, ragged=V % 2 == 1)
    rng = np.random.default_rng(V)
    w = rng.standard_normal((B, T))
    w[rng.random((B, T)) < 0.2] = 0.0
    check_loss(dp, x, targets, w if V % 3 else None, 0.75)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("parts", ["p", "l", "e", "ple"])
@pytest.mark.parametrize("B,T,V", [(2, 3, 5), (3, 2, 1001), (1, 2, 50257), (1, 2, 131079)])
def test_backward(dp, B, T, V, parts, dtype):
    x = _logits(B, T, V, dtype, V + 9)
    check_backward(dp, x, _targets(B, T, V, V + 9, True), 1.3, V, parts)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [3, 130, 8193, 32003, 140003])
def test_gradient_in_place(dp, V, dtype):
    targets = _targets(3, 2, V, V, True)
    check_loss(dp, _logits(3, 2, V, dtype, 1), targets, None, 1.0, in_place=True)
    check_backward(dp, _logits(3, 2, V, dtype, 2), targets, 1.0, 3, in_place=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V,pad,first", [(5, 3, 1), (1000, 1, 0), (1001, 6, 3), (32003, 61, 1), (131075, 2, 5)])
def test_strides_and_offsets(dp, V, pad, first, dtype):
    """Rows of a wider table, off 16 bytes; what lies between them is not touched."""
    torch = _torch()
    B, T = 2, 3
    stride = first + V + pad
    buf = _logits(B, T, stride, dtype, V)
    buf[..., :first] = float("nan")
    buf[..., first + V:] = float("nan")
    x = buf[..., first:first + V]
    targets = _targets(B, T, V, V, True)
    dev = torch.from_numpy(targets).cuda()
    k = 7
    _, out = run_logprobs(dp, x, dev, 1.0, k)
    check_logprobs(x, targets, 1.0, k, out)
    grad = torch.full((B, T, stride + 5), 7.0, dtype=x.dtype, device="cuda")
    check_loss(dp, x, targets, None, 1.0, dlogits=grad[..., 2:2 + V])
    assert bool((grad[..., :2] == 7).all()) and bool((grad[..., 2 + V:] == 7).all())
    # The last position of each example.
    last = x[:, -1:]
    _, out = run_logprobs(dp, last, dev[:, -1:].contiguous(), 1.0, k)
    check_logprobs(last, targets[:, -1:], 1.0, k, out)


def test_positions_of_weight_0_are_not_looked_at(dp):
    torch = _torch()
    x = _logits(2, 3, 300, "f32", 5)
    targets = np.array([[1, 2, 3], [4, -1, 5]])
    w = np.array([[0.5, 0.0, 1.0], [0.0, 3.0, 2.0]])
    x[0, 1] = float("nan")
    x[1, 0] = float("inf")
    x[1, 1] = float("nan")   # an empty position
    losses, dlogits = check_loss(dp, x, targets, w, 1.0)
    assert bool(torch.isfinite(losses).all()) and bool(torch.isfinite(dlogits).all())


def test_same_inputs_same_bits_and_other_streams(dp):
    torch = _torch()
    x = _logits(4, 8, 50257, "bf16", 6)
    targets = torch.from_numpy(_targets(4, 8, 50257, 6, True)).cuda()
    _, a = run_logprobs(dp, x, targets, 0.9, 20)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _, b = run_logprobs(dp, x, targets, 0.9, 20)
    for n in a:
        assert torch.equal(a[n], b[n]), n


@pytest.mark.parametrize("V", [130, 32003, 140001])
def test_graph_replays(dp, V):
    """A captured loss and captured log probabilities, replayed on other inputs with eager
    calls between, equal the eager results bit for bit."""
    torch = _torch()
    B, T, k = 2, 4, 9
    x, targets = _logits(B, T, V, "bf16", 1), torch.from_numpy(_targets(B, T, V, 1, True)).cuda()
    desc = dp.make_logits(x, targets, 1.0)
    ws = _ws(dp, desc, k)
    dlogits, losses = torch.empty_like(x), torch.empty(B, device="cuda")
    ids = torch.empty(B, T, k, dtype=torch.int64, device="cuda")
    lps, lse = torch.empty(B, T, k, device="cuda"), torch.empty(B, T, device="cuda")

    def both():
        dp.dpsgd_token_logprobs(desc, x, lse=lse, top_ids=ids, top_logprobs=lps, workspace=ws)
        dp.dpsgd_token_loss(desc, x, dlogits, losses=losses, workspace=ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for seed in range(3):
        x.copy_(_logits(B, T, V, "bf16", 40 + seed))
        targets.copy_(torch.from_numpy(_targets(B, T, V, 40 + seed, True)).cuda())
        for t in (dlogits, losses, ids, lps, lse):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (dlogits, losses, ids, lps, lse)]
        both()
        torch.cuda.synchronize()
        for a, b in zip(got, (dlogits, losses, ids, lps, lse)):
            assert torch.equal(a, b)


def test_many_rows(dp):
    """More rows than workgroups of a launch."""
    torch = _torch()
    B, T, V = 1100, 1000, 3
    x = _logits(B, T, V, "bf16", 8)
    targets = _targets(B, T, V, 8, True)
    _, out = run_logprobs(dp, x, torch.from_numpy(targets).cuda(), 1.0, 0)
    lp = torch.log_softmax(x.double(), -1)
    ids = torch.from_numpy(targets).cuda()
    there = (ids >= 0) & (ids < V)
    ref = torch.where(there, lp.gather(2, ids.clamp(0, V - 1).unsqueeze(-1)).squeeze(-1), 0.0)
    assert float((out["logprobs"].double() - ref).abs().max()) <= 250 * U


def test_rows_past_2_to_the_31(dp):
    """The last rows of logits of more than 2^32 bytes."""
    torch = _torch()
    B, T, V = 3, 1, 1001
    stride = (1 << 31) - 3
    buf = torch.empty(2 * stride + V, dtype=torch.bfloat16, device="cuda")
    x = buf.as_strided((B, T, V), (stride, stride, 1))
    x.copy_(_logits(B, T, V, "bf16", 4))
    targets = _targets(B, T, V, 4, False)
    _, out = run_logprobs(dp, x, torch.from_numpy(targets).cuda(), 1.0, 6)
    check_logprobs(x, targets, 1.0, 6, out)
    check_loss(dp, x, targets, None, 1.0, in_place=True)
