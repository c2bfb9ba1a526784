"""Token tables on the GPU against the float64 definitions.

Bounds, with u = 2^-24 and n the number of terms of a float32 sum: a sum is off by at
most n u sum|terms|, in any order; a product or a rounded factor adds u of its size
each. The lookup is one product and one rounding, so it is compared bit for bit.
"""

import math

import numpy as np
import pytest

from oracle import model_oracle as mo

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(autouse=True)
def _announce(request):
    print(f"[gpu] start {request.node.name}", flush=True)
    yield


def _torch():
    import torch
    return torch


def _ids(kind, B, T, V, rng):
    if kind == "uniform":
        return rng.integers(0, V, (B, T))
    if kind == "words":      # a few tokens are most of the text
        return np.minimum((np.exp(rng.random((B, T)) * math.log(V + 1)) - 1).astype(np.int64), V - 1)
    if kind == "one":        # one token everywhere
        return np.full((B, T), V // 2)
    if kind == "position":
        return np.broadcast_to(np.arange(T) % V, (B, T)).copy()
    ids = rng.integers(0, V, (B, T))   # "padded": ends of examples empty, one example all empty
    for i in range(B):
        ids[i, rng.integers(0, T + 1):] = [-1, -100, V, V + 7][i % 4]
    ids[0] = -1
    return ids


def _data(B, T, V, d, dtype, kind, seed):
    torch = _torch()
    rng = np.random.default_rng(seed)
    ids = _ids(kind, B, T, V, rng)
    G = torch.tensor(rng.standard_normal((B, T, d)).astype(np.float32)).to(dtype)
    empty = (ids < 0) | (ids >= V)
    poisoned = G.clone()
    poisoned[torch.tensor(empty)] = float("nan")   # rows of empty positions are not read
    return ids, G.double().numpy(), poisoned.cuda()


def _workspace(dp, emb):
    # Poisoned scratch: what it holds on entry does not matter.
    torch = _torch()
    return torch.full((dp.dpsgd_embedding_workspace_bytes(emb),), 0xFF, dtype=torch.uint8,
                      device="cuda")


SHAPES = [   # B, T, V, d, ids
    (1, 1, 1, 1, "uniform"),
    (3, 1, 7, 5, "uniform"),
    (2, 37, 11, 6, "uniform"),
    (5, 64, 300, 64, "words"),
    (4, 33, 50, 24, "padded"),
    (3, 700, 5, 12, "uniform"),         # every row longer than a chunk of the sorted list
    (2, 515, 9, 132, "one"),            # one row over many chunks
    (9, 130, 130, 40, "position"),
    (6, 257, 4099, 257, "words"),       # odd width, more than one column block
    (3, 90, 131100, 16, "padded"),      # more keys than 256 workgroups hold at 512 each
    (2, 1100, 40, 520, "words"),
    (300, 4, 33, 8, "padded"),          # more examples than workgroups of the sort
    (1, 4500, 700, 24, "words"),        # one long example
    (1, 4096, 900, 128, "words"),       # the longest that is sorted in LDS, and the most of it
    (2, 4097, 3, 72, "uniform"),        # the shortest that is not; few tokens, each most of a part
    (3, 2500, 2, 136, "padded"),
]


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,T,V,d,kind", SHAPES)
def test_norms_and_clipped_sum(dp, B, T, V, d, kind, dtype, wide):
    torch = _torch()
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    ids, G, dG = _data(B, T, V, d, dt, kind, seed=B * 1000 + T)
    scale = np.float32(1.5)
    dids = torch.tensor(ids, dtype=torch.int64 if wide else torch.int32).cuda()
    emb = dp.make_embedding(dids, (V, d), float(scale))
    ws = _workspace(dp, emb)
    start = torch.rand(B, device="cuda")
    got = torch.full((B,), float("nan"), device="cuda")
    more = start.clone()
    dp.dpsgd_embedding_norms(emb, dG, got, workspace=ws)
    dp.dpsgd_embedding_norms(emb, dG, more, accumulate=True, workspace=ws)
    torch.cuda.synchronize()

    ref, bound = np.zeros(B), np.zeros(B)
    for i in range(B):
        groups = {}
        for t in range(T):
            if 0 <= ids[i, t] < V:
                groups.setdefault(ids[i, t], []).append(G[i, t])
        for rows in groups.values():
            s, a = np.sum(rows, axis=0), np.sum(np.abs(rows), axis=0)
            off = len(rows) * U * a
            ref[i] += float(scale) ** 2 * np.sum(s * s)
            bound[i] += float(scale) ** 2 * np.sum(2 * np.abs(s) * off + off * off)
    assert np.allclose(ref, mo.embedding_norms_sq(ids, G, V, float(scale)), rtol=1e-12)
    # A lane adds at most 4 squares a row; then its wave, parts and blocks add up.
    bound += (4 * T + 200) * U * ref
    got, more = got.cpu().double().numpy(), more.cpu().double().numpy()
    assert np.all(np.abs(got - ref) <= bound), np.max(np.abs(got - ref) - bound)
    s0 = start.cpu().double().numpy()
    assert np.all(np.abs(more - (ref + s0)) <= bound + 2 * U * (ref + s0))
    assert np.all(got[ref == 0] == 0)

    # The clipped sum, from given norms: half of the examples over the bound.
    nsq = torch.tensor((0.25 + np.arange(B) % 4).astype(np.float32), device="cuda")
    C = 1.25
    n = np.sqrt(nsq.cpu().double().numpy())
    c = np.where(n > C, C / n, 1.0)
    ref = mo.embedding_clipped_sum(ids, G, V, float(scale), c)
    size = mo.embedding_clipped_sum(ids, np.abs(G), V, float(scale), c)
    count = np.zeros(V)
    at = (ids >= 0) & (ids < V)
    np.add.at(count, ids[at], 1)
    bound = size * ((count + 16) * U)[:, None]   # the factor: three roundings of at most 2 u
    grad = torch.full((V, d), float("nan"), device="cuda")
    fac, mask = torch.empty(B, device="cuda"), torch.empty(B, dtype=torch.uint8, device="cuda")
    dp.dpsgd_embedding_clip_accumulate(emb, dG, nsq, C, grad, factors_out=fac, mask_out=mask,
                                       workspace=ws)
    g1 = grad.cpu().double().numpy()
    assert np.all(np.abs(g1 - ref) <= bound)
    assert np.all(g1[count == 0] == 0)
    assert np.allclose(fac.cpu().double().numpy(), c, rtol=8 * U)
    assert np.array_equal(mask.cpu().numpy(), (n > C).astype(np.uint8))
    again = torch.empty_like(grad)
    dp.dpsgd_embedding_clip_accumulate(emb, dG, nsq, C, again, workspace=ws)
    assert torch.equal(again, grad)   # bit for bit: no order is left open
    first = torch.rand(V, d, device="cuda")
    grad = first.clone()
    dp.dpsgd_embedding_clip_accumulate(emb, dG, nsq, C, grad, accumulate=True, workspace=ws)
    f = first.cpu().double().numpy()
    assert np.all(np.abs(grad.cpu().double().numpy() - (f + ref)) <= bound + 2 * U * (np.abs(f) + size))
    # No norms: the plain gradient.
    dp.dpsgd_embedding_clip_accumulate(emb, dG, None, 0.0, grad, workspace=ws)
    ref = mo.embedding_clipped_sum(ids, G, V, float(scale), np.ones(B))
    size = mo.embedding_clipped_sum(ids, np.abs(G), V, float(scale), np.ones(B))
    assert np.all(np.abs(grad.cpu().double().numpy() - ref) <= size * ((count + 4) * U)[:, None])


@pytest.mark.parametrize("to", ["f32", "bf16"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,T,V,d,kind", SHAPES + [(8, 1, 1000, 768, "uniform"),
                                                    (3, 5, 20, 2052, "padded")])
def test_lookup_bit_for_bit(dp, B, T, V, d, kind, dtype, to):
    torch = _torch()
    dts = {"f32": torch.float32, "bf16": torch.bfloat16}
    rng = np.random.default_rng(5)
    ids = _ids(kind, B, T, V, rng)
    table = torch.tensor(rng.standard_normal((V, d)).astype(np.float32)).to(dts[dtype])
    scale = np.float32(27.712812)
    at = torch.tensor((ids >= 0) & (ids < V))
    ref = torch.zeros(B, T, d)
    ref[at] = table.float()[torch.tensor(ids)[at]] * torch.tensor(scale)
    ref = ref.to(dts[to])
    for wide in (torch.int32, torch.int64):
        out = torch.full((B, T, d), float("nan"), dtype=dts[to], device="cuda")
        emb = dp.make_embedding(torch.tensor(ids, dtype=wide).cuda(), (V, d), float(scale))
        dp.dpsgd_embedding_lookup(emb, table.cuda(), out)
        assert torch.equal(out.cpu(), ref)


def test_ids_beyond_32_bits_are_empty(dp):
    torch = _torch()
    ids = torch.tensor([[0, 1 << 32, (1 << 32) + 1, -(1 << 40)]]).cuda()
    table = torch.ones(2, 8, device="cuda")
    out = torch.full((1, 4, 8), float("nan"), device="cuda")
    emb = dp.make_embedding(ids, (2, 8), 3.0)
    dp.dpsgd_embedding_lookup(emb, table, out)
    assert torch.equal(out[0, 0].cpu(), torch.full((8,), 3.0)) and float(out[0, 1:].abs().sum()) == 0
    ws, nsq = _workspace(dp, emb), torch.empty(1, device="cuda")
    dp.dpsgd_embedding_norms(emb, torch.ones(1, 4, 8, device="cuda"), nsq, workspace=ws)
    assert float(nsq) == 72.0


def test_factor_zero_reads_nothing_and_nan_norm_spreads(dp):
    torch = _torch()
    ids = torch.tensor([[0, 1, 1], [1, 2, 2], [3, 3, 3]], dtype=torch.int32).cuda()
    G = torch.ones(3, 3, 4, device="cuda")
    G[1] = float("nan")
    emb = dp.make_embedding(ids, (5, 4), 1.0)
    ws = _workspace(dp, emb)
    nsq = torch.tensor([1.0, float("inf"), float("nan")], device="cuda")
    grad = torch.empty(5, 4, device="cuda")
    dp.dpsgd_embedding_clip_accumulate(emb, G, nsq, 2.0, grad, workspace=ws)
    g = grad.cpu()
    assert torch.equal(g[:3], torch.tensor([1.0, 2.0, 0.0]).view(3, 1).expand(3, 4))
    assert torch.isnan(g[3]).all() and float(g[4].abs().sum()) == 0
    # A NaN row makes its example's norm NaN, and no other's.
    out = torch.empty(3, device="cuda")
    dp.dpsgd_embedding_norms(emb, G, out, workspace=ws)
    out = out.cpu()
    assert float(out[0]) == 20.0 and math.isnan(float(out[1])) and float(out[2]) == 36.0


def test_calls_on_another_stream(dp):
    torch = _torch()
    ids, G, dG = _data(6, 257, 4099, 64, torch.float32, "words", 11)
    dids = torch.tensor(ids).cuda()
    emb = dp.make_embedding(dids, (4099, 64), 0.5)
    ws = _workspace(dp, emb)
    nsq, grad = torch.empty(6, device="cuda"), torch.empty(4099, 64, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    dp.dpsgd_embedding_norms(emb, dG, nsq, workspace=ws, stream=side)
    dp.dpsgd_embedding_clip_accumulate(emb, dG, nsq, 1.0, grad, workspace=ws, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    n = np.sqrt(mo.embedding_norms_sq(ids, G, 4099, 0.5))
    assert np.allclose(np.sqrt(nsq.cpu().double().numpy()), n, rtol=1e-4)
    ref = mo.embedding_clipped_sum(ids, G, 4099, 0.5, np.minimum(1.0, 1.0 / n))
    assert np.allclose(grad.cpu().double().numpy(), ref, rtol=0, atol=1e-4 * np.abs(ref).max())


def test_captured_in_a_graph(dp):
    torch = _torch()
    ids, G, dG = _data(4, 300, 500, 48, torch.bfloat16, "words", 12)
    dids = torch.tensor(ids).cuda()
    emb = dp.make_embedding(dids, (500, 48), 2.0)
    ws = _workspace(dp, emb)
    nsq, grad = torch.empty(4, device="cuda"), torch.empty(500, 48, device="cuda")

    def step():
        dp.dpsgd_embedding_norms(emb, dG, nsq, workspace=ws)
        dp.dpsgd_embedding_clip_accumulate(emb, dG, nsq, 3.0, grad, workspace=ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(3):   # new contents in the same buffers between the replays
        rng = np.random.default_rng(40 + k)
        dids.copy_(torch.tensor(_ids("padded", 4, 300, 500, rng)))
        dG.copy_(torch.tensor(rng.standard_normal((4, 300, 48)), dtype=torch.bfloat16))
        graph.replay()
        torch.cuda.synchronize()
        got = (nsq.clone(), grad.clone())
        step()
        torch.cuda.synchronize()
        assert torch.equal(got[0], nsq) and torch.equal(got[1], grad)


def test_binding_refusals(dp):
    torch = _torch()
    ids = torch.zeros(2, 3, dtype=torch.int64, device="cuda")
    emb = dp.make_embedding(ids, (4, 8), 1.0)
    ws = _workspace(dp, emb)
    table, out = torch.zeros(4, 8, device="cuda"), torch.zeros(2, 3, 8, device="cuda")
    for bad in (table.double(), table[:3], table.cpu(), table.t()):
        with pytest.raises(ValueError):
            dp.dpsgd_embedding_lookup(emb, bad, out)
    with pytest.raises(ValueError):
        dp.dpsgd_embedding_lookup(emb, table, torch.zeros(2, 3, 16, device="cuda")[..., ::2])
    with pytest.raises(ValueError):
        dp.make_embedding(ids[:, ::2], (4, 8))
    with pytest.raises(ValueError):
        dp.dpsgd_embedding_norms(emb, out, torch.zeros(3, device="cuda"), workspace=ws)
    with pytest.raises(dp.DpsgdError):
        dp.dpsgd_embedding_norms(emb, out, torch.zeros(2, device="cuda"))          # no workspace
    with pytest.raises(ValueError):
        dp.dpsgd_embedding_clip_accumulate(emb, out, None, 1.0, table.bfloat16(), workspace=ws)
