"""The gradient of the token log probabilities where all logits of a row have a common
offset, which the distribution does not depend on, against the float64 definition and by its
sum over a row; and the loss's and the entropy of such rows.

Bound, with u = 2^-24, d = m - z >= 0 an entry's distance from the row's largest, range the
largest d of a row, n its length. d is off by 3 u d (the scale times log2 e is two roundings,
the multiply-add one; the rounding of the product that is common to a row is taken back to
u / 16), the exponential by 2 u beside that, so e^-d by (3 d + 3) u of itself. The sum S
adds the terms' own errors, on average over p (3 (1 + ln n) + 3) u, since sum p d = H - ln S
<= ln n, and (n / 64 + 32) u of summing; where a row is summed in one pass the terms are
rescaled: 2 range u in all, as the steps have one sign, and 3 u a step of at most n / 1024 +
8. The quotient and the factors add 8 u. So p is off by K(d) u of itself with

    K(d) = 3 d + 3 ln n + 2 range + n / 32 + 80.

Rows whose lse is within 32 of 0 (1024 in bf16) take p from it: half a step of it is 16 u (512
u), z - lse is one rounding more, and its values one of 2 u: 64 + 2 d (576 + 2 d) more, at
most. ln p is off by K(d) u, the entropy by E u, E = K(0) + sum p d (K(d) + K(0) + 4) + H. bf16
adds 2^-8 of a value.
"""

import math

import numpy as np
import pytest

from oracle import lm_oracle as lo

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
BF16 = 2.0 ** -8


@pytest.fixture(autouse=True)
def _announce(request):
    print(f"[gpu] start {request.node.name}", flush=True)
    yield


def _tensor(x, dtype):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x, np.float32)).to(
        {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]).cuda()


def _wide(t):
    return t.double().cpu().numpy()


def _row(x, s, dtype):
    """p, ln p, entropy and the bounds K(d), E of one row, in u."""
    z = s * x
    d, n = z.max() - z, len(x)
    there = np.isfinite(d)
    e = np.where(there, np.exp(-np.where(there, d, 0.0)), 0.0)
    p, log_S = e / e.sum(), math.log(e.sum())
    d = np.where(there, d, 0.0)
    lse = abs(z.max() + log_S)
    near = 0.0
    if lse < (1025 if dtype == "bf16" else 32.1):
        near = 2 * d + (576 if dtype == "bf16" else 64)
    K = 3 * d + 3 * math.log(n) + 2 * d.max() + n / 32 + 80 + near
    K0 = K[d == 0].min()
    H = log_S + float((p * d).sum())
    return p, np.where(there, -d - log_S, 0.0), H, K, K0 + float((p * d * (K + K0 + 4)).sum()) + H


def _check(got, x64, t, s, g, dtype):
    """g: the factors of logprob, lse and entropy, [N] each."""
    ref = lo.token_gradient(x64, t, s, *g)
    for i, row in enumerate(x64):
        if not np.isfinite(ref[i]).all() or not ref[i].any():
            assert np.array_equal(got[i], ref[i], equal_nan=True), i
            continue
        gp, gl, ge = (abs(f[i]) for f in g)
        p, l, H, K, E = _row(row, s, dtype)
        tol = s * U * (p * (gp + gl + ge * (abs(l) + H)) * (K + 8) + p * ge * (K + E + 4 * (abs(l) + H)))
        tol += 4 * U * s * gp * (ref[i] != 0)
        if dtype == "bf16":
            tol = tol + BF16 * (np.abs(ref[i]) + tol)
        off = np.abs(got[i] - ref[i])
        bad = off > tol + 1e-38
        assert not bad.any(), f"row {i}: {got[i][bad][:4]} for {ref[i][bad][:4]}, within {tol[bad][:4]}"


def _backward(dp, x, targets, s, g, in_place=False):
    import torch
    B, T, _ = x.shape
    desc = dp.make_logits(x, torch.from_numpy(targets).cuda(), s)
    lse, entropy = torch.empty(2, B, T, device="cuda").unbind(0)
    ws = torch.empty(dp.dpsgd_token_workspace_bytes(desc), dtype=torch.uint8, device="cuda")
    dp.dpsgd_token_logprobs(desc, x, lse=lse, entropy=entropy, workspace=ws)
    dx = x if in_place else torch.full_like(x, 7.0)
    up = [None if f is None else _tensor(f.reshape(B, T), "f32") for f in g]
    dp.dpsgd_token_logprobs_backward(desc, x, lse, dx, entropy=entropy, grad_logprobs=up[0],
                                     grad_lse=up[1], grad_entropy=up[2])
    torch.cuda.synchronize()
    return desc, ws, dx


# By waves, by workgroups of each size, and what none holds; few rows, in parts.
SHAPES = [(65, 1, 1000), (33, 2, 1001), (65, 1, 5003), (70, 1, 20011), (13, 5, 40000), (5, 13, 65536), (66, 1, 66001),
          (2, 33, 131081), (3, 2, 1000), (2, 3, 9001), (2, 3, 50257), (1, 2, 140001)]
OFFSETS = [0.0, -40.0, 300.0, 20000.0, -1.0e6]


def _case(B, T, V, dtype, offset, seed, masked=True):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((B, T, V)) * 2.5 + offset
    if masked:   # some tokens, in one row all, and a row with a NaN
        x[rng.random((B, T, V)) < 0.05] = -np.inf
        x[0, 0] = -np.inf
        x[-1, -1, V // 2] = np.nan
    targets = rng.integers(0, V, (B, T))
    targets[-1, 0] = -1
    x = _tensor(x, dtype)
    return x, _wide(x).reshape(B * T, V), targets, rng


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("offset", OFFSETS)
@pytest.mark.parametrize("B,T,V", SHAPES)
def test_gradient_of_rows_with_an_offset(dp, B, T, V, offset, dtype):
    # A scale that is not a power of two where the products are taken exactly.
    s = 1.0 if abs(offset) > 1e5 else 0.75
    x, x64, targets, rng = _case(B, T, V, dtype, offset, V)
    g = [np.float32(rng.standard_normal(B * T)).astype(np.float64) for _ in range(3)]
    if offset == 300.0:
        g[2] = np.zeros(B * T)
    _, _, dx = _backward(dp, x, targets, s, [g[0], g[1], None if offset == 300.0 else g[2]], 
                         in_place=offset in (-40.0, 20000.0))
    _check(_wide(dx).reshape(B * T, V), x64, targets.reshape(-1), s, g, dtype)


@pytest.mark.parametrize("offset", OFFSETS)
@pytest.mark.parametrize("B,T,V", SHAPES)
def test_gradient_sums_to_zero(dp, B, T, V, offset):
    s = 1.0 if abs(offset) > 1e5 else 0.75
    x, x64, targets, _ = _case(B, T, V, "f32", offset, V + 1, masked=False)
    N, t = B * T, targets.reshape(-1)
    _, _, dx = _backward(dp, x, targets, s, [-np.ones(N), None, None])
    got = _wide(dx).reshape(N, V)
    for i in range(N):
        if t[i] < 0:
            assert not got[i].any()
            continue
        p, _, _, K, _ = _row(x64[i], s, "f32")
        tol = s * U * (p * (K + 8) + 4 * (np.arange(V) == t[i]))
        assert abs(got[i].sum()) <= tol.sum() + 1e-38 * V, (i, got[i].sum(), tol.sum())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("offset", OFFSETS)
@pytest.mark.parametrize("B,T,V", SHAPES + [(1, 3, 300007)])
def test_loss_and_entropy_of_rows_with_an_offset(dp, B, T, V, offset, dtype):
    """Rows in parts among them: their join adds (3 D + 3) u to a part's share, D the distance
    of its largest entry from the row's, so no more than 3 d u of any entry in it: on average
    over p (3 ln n + 3) u, and 16 u of summing."""
    import torch
    s = 1.0 if abs(offset) > 1e5 else 0.75
    x, x64, targets, _ = _case(B, T, V, dtype, offset, V + 1, masked=False)
    N, t = B * T, targets.reshape(-1)
    desc = dp.make_logits(x, torch.from_numpy(targets).cuda(), s)
    ws = torch.empty(dp.dpsgd_token_workspace_bytes(desc), dtype=torch.uint8, device="cuda")
    dl, entropy = torch.full_like(x, 7.0), torch.empty(B, T, device="cuda")
    dp.dpsgd_token_loss(desc, x, dl, workspace=ws)
    dp.dpsgd_token_logprobs(desc, x, entropy=entropy, workspace=ws)
    got, H_got = _wide(dl).reshape(N, V), _wide(entropy).reshape(N)
    ref = lo.token_gradient(x64, t, s, -np.ones(N))
    for i in range(N):
        if t[i] < 0:
            assert not got[i].any() and H_got[i] == 0.0
            continue
        p, _, H, K, E = _row(x64[i], s, dtype)
        more = 3 * math.log(V) + 20
        tol = s * U * (p * (K + more + 8) + 4 * (np.arange(V) == t[i]))
        if dtype == "f32":
            assert abs(got[i].sum()) <= tol.sum() + 1e-38 * V, (i, got[i].sum(), tol.sum())
        else:
            tol = tol + BF16 * (np.abs(ref[i]) + tol)
        assert (np.abs(got[i] - ref[i]) <= tol + 1e-38).all(), i
        assert abs(H_got[i] - H) <= (E + more * (2 + 2 * H)) * U, (i, H_got[i], H)


@pytest.mark.parametrize("offset", [-40.0, 1000.0, 3000.0, -2.0e5])
@pytest.mark.parametrize("B,T,V,k", [(2, 3, 1000, 64), (2, 2, 5003, 20), (70, 1, 20011, 64), (2, 1, 40000, 5),
                                     (1, 2, 70001, 64), (2, 1, 300007, 20), (3, 1, 700, 1)])
def test_alternatives_of_rows_with_an_offset(dp, B, T, V, k, offset):
    """float32 logits whose upper bits are alike, ties among them: the tokens are the exact
    ones, in order."""
    import torch
    x, x64, _, _ = _case(B, T, V, "f32", offset, V + k)
    desc = dp.make_logits(x)
    ids = torch.full((B, T, k), 7, dtype=torch.int64, device="cuda")
    ws = torch.empty(dp.dpsgd_token_workspace_bytes(desc, k), dtype=torch.uint8, device="cuda")
    dp.dpsgd_token_logprobs(desc, x, top_ids=ids, workspace=ws)
    want = [lo.alternatives(row, 1.0, k)[0] for row in x64]
    assert np.array_equal(ids.cpu().numpy().reshape(B * T, k), np.stack(want))
