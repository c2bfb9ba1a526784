"""The ends of the ranges of the operators between and behind the blocks, and calls at the
same time: offsets past 32 bits, the largest vocabulary, two streams."""

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(autouse=True)
def _announce(request):
    print(f"[gpu] start {request.node.name}", flush=True)
    yield


def _bytes(n):
    import torch
    return torch.empty(n, dtype=torch.uint8, device="cuda")


def test_largest_vocabulary(dp):
    """2^24 tokens: sums in parts, alternatives joined from 2048 or 4096 of them."""
    import torch
    V = 1 << 24
    gen = torch.Generator(device="cuda").manual_seed(3)
    for dtype in (torch.float32, torch.bfloat16):
        x = torch.randn(1, 2, V, generator=gen, device="cuda").to(dtype)
        targets = torch.tensor([[V - 1, 12345]], device="cuda")
        desc = dp.make_logits(x, targets, 1.0)
        out = {n: torch.empty(1, 2, device="cuda") for n in ("logprobs", "lse", "entropy")}
        out["top_ids"] = torch.empty(1, 2, 64, dtype=torch.int64, device="cuda")
        out["top_logprobs"] = torch.empty(1, 2, 64, device="cuda")
        dp.dpsgd_token_logprobs(desc, x, workspace=_bytes(dp.dpsgd_token_workspace_bytes(desc, 64)), **out)
        dx = torch.empty_like(x)
        dp.dpsgd_token_loss(desc, x, dx, workspace=_bytes(dp.dpsgd_token_workspace_bytes(desc)))
        lp = torch.log_softmax(x.double(), -1)
        # ln S is off by K u, K = 10 max |x| (at most 6.5) + the adds of a thread, of the waves
        # and of the parts (32 + 16 + 24 in a row); entries of logprob and lse by a few u of 22.
        L = (65 + 72 + 8 * 22) * U
        assert float((out["logprobs"].double() - lp.gather(2, targets.unsqueeze(-1)).squeeze(-1)).abs().max()) <= L
        assert float((out["lse"].double() - torch.logsumexp(x.double(), -1)).abs().max()) <= L
        assert float((out["entropy"].double() + (lp.exp() * lp).sum(-1)).abs().max()) <= L * (2 + 17)
        ids = torch.sort(x, dim=-1, descending=True, stable=True)[1][..., :64]
        assert torch.equal(out["top_ids"], ids)
        assert float((out["top_logprobs"].double() - lp.gather(2, ids)).abs().max()) <= L
        ref = lp.exp()
        ref.scatter_add_(2, targets.unsqueeze(-1), torch.full((1, 2, 1), -1.0, dtype=torch.float64, device="cuda"))
        half = 2.0 ** -8 if dtype == torch.bfloat16 else 0.0
        tol = ref.abs() * (2 * L + 8 * U + half * 1.01) + 1e-38
        assert bool(((dx.double() - ref).abs() <= tol).all())
        del lp, ref, tol, dx, x
        torch.cuda.empty_cache()


def test_tokens_far_apart_in_int32(dp):
    """int32 targets, more rows than a launch has workgroups of whole rows."""
    import torch
    B, T, V = 2, 600_000, 5
    x = torch.randn(B, T, V, device="cuda")
    targets = torch.randint(-1, V, (B, T), device="cuda", dtype=torch.int32)
    desc = dp.make_logits(x, targets, 2.0)
    losses, dx = torch.empty(B, device="cuda"), torch.empty_like(x)
    w = torch.rand(B, T, device="cuda") / T
    dp.dpsgd_token_loss(desc, x, dx, losses=losses, weights=w,
                        workspace=_bytes(dp.dpsgd_token_workspace_bytes(desc)))
    there = targets >= 0
    lp = torch.log_softmax(2.0 * x.double(), -1)
    at = lp.gather(2, targets.clamp(min=0).long().unsqueeze(-1)).squeeze(-1)
    terms = torch.where(there, -w.double() * at, 0.0)
    # A thread adds 2344 positions, each off by a hundred u of it at most.
    assert float(((losses.double() - terms.sum(1)) / terms.sum(1)).abs().max()) <= (2344 + 116) * U
    ref = lp.exp()
    ref.scatter_add_(2, targets.clamp(min=0).long().unsqueeze(-1), torch.full((B, T, 1), -1.0, dtype=torch.float64, device="cuda"))
    ref *= torch.where(there, 2.0 * w.double(), 0.0).unsqueeze(-1)
    size = torch.where(there, 2.0 * w.double(), 0.0).unsqueeze(-1)
    assert bool(((dx.double() - ref).abs() <= size * 600 * U).all())


@pytest.mark.parametrize("C", [4096, 5])
def test_residual_norm_past_2_to_the_31(dp, C):
    """The last rows of more than 2^31 elements are those of a call on them alone."""
    import torch
    rows = (1 << 31) // C + 3000
    B, S = 2, (rows + 1) // 2
    x = torch.zeros(B, S, C, dtype=torch.bfloat16, device="cuda")
    block, dy = torch.zeros_like(x), torch.zeros_like(x)
    n = 700
    gen = torch.Generator(device="cuda").manual_seed(1)
    for t in (x, block, dy):
        t[-1, -n:] = torch.randn(n, C, generator=gen, device="cuda").to(t.dtype)
    gamma, gate = torch.rand(C, device="cuda"), torch.rand(C, device="cuda")
    small = [t[-1:, -n:].clone() for t in (x, block, dy)]
    kw = dict(kind="rms", gamma=gamma, gate=gate, post=True, residual_scale=0.5)
    results = []
    for a, b, d in ((x, block, dy), small):
        desc = dp.make_residual_norm(a, **kw)
        st = torch.empty(*a.shape[:2], 4, device="cuda")
        y = torch.empty_like(a)
        dp.dpsgd_residual_norm_forward(desc, a, b, a, y, st)
        ws = _bytes(dp.dpsgd_residual_norm_workspace_bytes(desc))
        dg = torch.empty(a.shape[0], C, device="cuda")
        dp.dpsgd_residual_norm_backward(desc, b, a, d, None, st, dx=y, dblock=d, dgate=dg, workspace=ws)
        torch.cuda.synchronize()
        results.append([t[-1, -n:].clone() for t in (a, y, d, st)] + [dg[-1].clone()])
        del y, ws
    for p, q in zip(results[0][:4], results[1][:4]):
        assert torch.equal(p, q)
    # Sums in another order: at most the adds of a thread and of the joins, of their sizes.
    a, b = results[0][4].double(), results[1][4].double()
    assert float((a - b).abs().max()) <= 300 * U * n
    torch.cuda.empty_cache()


def test_adamw8_past_2_to_the_31(dp):
    """The last blocks of a tensor of more than 2^31 entries are those of a tensor of them."""
    import torch
    rows, cols = 3, 715_828_140
    n, tail = rows * cols, 4 * 256 + rows * cols % 256
    assert n > 1 << 31 and (n - tail) % 256 == 0
    gen = torch.Generator(device="cuda").manual_seed(1)
    layers = [dp.shape_layer(1, 1, cols, rows, dp.DPSGD_F32, 0)]
    big = [torch.zeros(rows, cols, device="cuda") for _ in range(2)]
    for t in big:
        t.view(-1)[-tail:] = torch.randn(tail, generator=gen, device="cuda")
    m, v, exps = dp.make_states8(layers)
    small = [t.view(-1)[-tail:].clone().view(1, tail) for t in big]
    one = [dp.shape_layer(1, 1, tail, 1, dp.DPSGD_F32, 0)]
    sm, sv, se = dp.make_states8(one)
    opt = dp.make_adamw(1e-2, t=2)
    for _ in range(2):
        dp.dpsgd_noise_adamw8_multi(layers, big[:1], big[1:], m, v, exps, 0.0, 1.0, 0, 0, 1.0, opt)
        dp.dpsgd_noise_adamw8_multi(one, small[:1], small[1:], sm, sv, se, 0.0, 1.0, 0, 0, 1.0, opt)
    torch.cuda.synchronize()
    assert torch.equal(big[1].view(-1)[-tail:], small[1].view(-1))
    assert torch.equal(m[0].view(-1)[-tail:], sm[0].view(-1)) and torch.equal(v[0].view(-1)[-tail:], sv[0].view(-1))
    assert torch.equal(exps[0][-len(se[0]):], se[0])
    assert bool((m[0].view(-1)[:4096] == 0).all()) and bool((sm[0] != 0).any())
    torch.cuda.empty_cache()


def test_two_streams_at_once(dp):
    """Calls on two streams, each with a workspace of its own, give what they give alone."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(9)

    def make(seed):
        x = torch.randn(8, 4, 50257, generator=gen, device="cuda").to(torch.bfloat16)
        t = torch.randint(0, 50257, (8, 4), generator=gen, device="cuda")
        desc = dp.make_logits(x, t, 1.0)
        r = torch.randn(6, 300, 768, generator=gen, device="cuda").to(torch.bfloat16)
        b, dy = torch.randn_like(r), torch.randn_like(r)
        gamma = torch.rand(768, device="cuda")
        norm = dp.make_residual_norm(r, gamma=gamma)
        return dict(x=x, desc=desc, r=r, b=b, dy=dy, norm=norm,
                    ws=_bytes(dp.dpsgd_token_workspace_bytes(desc, 9)),
                    ws2=_bytes(dp.dpsgd_residual_norm_workspace_bytes(norm)),
                    ids=torch.empty(8, 4, 9, dtype=torch.int64, device="cuda"), dx=torch.empty_like(x),
                    losses=torch.empty(8, device="cuda"), out=torch.empty_like(r), y=torch.empty_like(r),
                    st=torch.empty(6, 300, 4, device="cuda"), dg=torch.empty(6, 768, device="cuda"),
                    dr=torch.empty_like(r), db=torch.empty_like(r))

    def run(s):
        dp.dpsgd_token_logprobs(s["desc"], s["x"], top_ids=s["ids"], workspace=s["ws"])
        dp.dpsgd_token_loss(s["desc"], s["x"], s["dx"], losses=s["losses"], workspace=s["ws"])
        dp.dpsgd_residual_norm_forward(s["norm"], s["r"], s["b"], s["out"], s["y"], s["st"])
        dp.dpsgd_residual_norm_backward(s["norm"], s["b"], s["out"], s["dy"], None, s["st"], dx=s["dr"],
                                        dblock=s["db"], dgamma=s["dg"], workspace=s["ws2"])

    names = ("ids", "dx", "losses", "out", "y", "st", "dg", "dr", "db")
    states = [make(k) for k in range(2)]
    alone = []
    for s in states:
        run(s)
        torch.cuda.synchronize()
        alone.append([s[n].clone() for n in names])
        for n in names:
            s[n].zero_()
    streams = [torch.cuda.Stream() for _ in states]
    torch.cuda.synchronize()
    for _ in range(3):
        for stream, s in zip(streams, states):
            with torch.cuda.stream(stream):
                run(s)
    torch.cuda.synchronize()
    for s, ref in zip(states, alone):
        for n, r in zip(names, ref):
            assert torch.equal(s[n], r), n


def test_two_graphs_share_a_workspace(dp):
    """Two captured calls with one workspace, replayed in turn, give what each gives alone."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(4)
    xs = [torch.randn(2, 3, V, generator=gen, device="cuda").to(torch.bfloat16) for V in (200_003, 50_001)]
    targets = torch.tensor([[1, -1, 7], [2, 3, 4]], device="cuda")
    descs = [dp.make_logits(x, targets, 1.0) for x in xs]
    ws = _bytes(max(dp.dpsgd_token_workspace_bytes(d, 30) for d in descs))
    ids = [torch.empty(2, 3, 30, dtype=torch.int64, device="cuda") for _ in xs]
    grads, losses = [torch.empty_like(x) for x in xs], [torch.empty(2, device="cuda") for _ in xs]

    def run(k):
        dp.dpsgd_token_logprobs(descs[k], xs[k], top_ids=ids[k], workspace=ws)
        dp.dpsgd_token_loss(descs[k], xs[k], grads[k], losses=losses[k], workspace=ws)

    for k in range(2):
        run(k)
    torch.cuda.synchronize()
    graphs = []
    for k in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            run(k)
        graphs.append(g)
    for turn in range(3):
        for x in xs:
            x.copy_(torch.randn(x.shape, generator=gen, device="cuda").to(x.dtype))
        for k in range(2):
            graphs[k].replay()
        torch.cuda.synchronize()
        got = [(ids[k].clone(), grads[k].clone(), losses[k].clone()) for k in range(2)]
        for k in range(2):
            run(k)
            torch.cuda.synchronize()
            for a, b in zip(got[k], (ids[k], grads[k], losses[k])):
                assert torch.equal(a, b), (turn, k)
