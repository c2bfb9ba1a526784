"""The noise + AdamW step with 8-bit moments on the GPU against its definition: codes,
exponents and parameters are compared bit for bit (every operation of the definition is a
float32 operation that is rounded by itself). Where noise is added its normals are the
library's own, read back from the call's noisy output."""

import numpy as np
import pytest

import oracle
from oracle import lm_oracle as lo

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _announce(request):
    print(f"[gpu] start {request.node.name}", flush=True)
    yield


def _torch():
    import torch
    return torch


def _dev(x):
    return _torch().from_numpy(np.ascontiguousarray(x)).cuda()


def _cfg(t=5, **kw):
    d = dict(lr=4e-4, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=1e-2, t=t)
    return oracle.AdamWConfig(**{**d, **kw})


def _opt(dp, cfg):
    return dp.make_adamw(lr=cfg.lr, beta1=cfg.beta1, beta2=cfg.beta2, eps=cfg.eps,
                         weight_decay=cfg.weight_decay, t=cfg.t)


def _state(shape, seed, fresh=False, spread=1.0):
    """A gradient, a parameter and moments of different sizes, packed by the definition."""
    rng = np.random.default_rng(seed)
    n = shape[0] * shape[1]
    size = np.exp(spread * rng.standard_normal(n))
    grad = (rng.standard_normal(n) * size).astype(np.float32)
    param = rng.standard_normal(n).astype(np.float32)
    m = np.zeros(n, np.float32) if fresh else (rng.standard_normal(n) * size * 1e-2).astype(np.float32)
    v = np.zeros(n, np.float32) if fresh else (rng.random(n) * size * size * 1e-4).astype(np.float32)
    km, kv = lo.block_exponents(m, "m"), lo.block_exponents(v, "v")
    exps = np.stack([km, kv], 1).astype(np.uint8)
    if fresh:
        exps[:] = 0
    return grad, param, lo.encode(m, km, "m"), lo.encode(v, kv, "v"), exps


class Tensors:
    """Device tensors of several states."""

    def __init__(self, dp, shapes, states):
        self.shapes = shapes
        self.layers = [dp.shape_layer(1, 1, s[1], s[0], dp.DPSGD_F32, 11 + 3 * k) for k, s in enumerate(shapes)]
        self.grads, self.params, self.m, self.v = ([_dev(st[i].reshape(s)) for st, s in zip(states, shapes)]
                                                   for i in range(4))
        self.exps = [_dev(st[4]) for st in states]

    def lists(self):
        return self.grads, self.params, self.m, self.v, self.exps

    def numpy(self, k):
        return tuple(a[k].cpu().numpy().reshape(-1) for a in (self.params, self.m, self.v)) + (self.exps[k].cpu().numpy(),)


def _same(got, ref, what):
    a, b = got, ref
    if a.dtype == np.float32:
        bad = ~((a.view(np.uint32) == b.view(np.uint32)) | (np.isnan(a) & np.isnan(b)))
    else:
        bad = a != b
    assert not bad.any(), f"{what}: {np.argwhere(bad)[:4].tolist()}: {a[bad][:4]} for {b[bad][:4]}"


def _check(t, states, cfg, scale, round_seed, noisy=None):
    for k, st in enumerate(states):
        tid = 11 + 3 * k
        grad, s = st[0], scale
        if noisy is not None:   # g as the call has it
            grad, s = noisy[k].cpu().numpy().reshape(-1), 1.0
        new, qm, qv, exps, _ = lo.adamw8_step(grad, st[1], st[2], st[3], st[4], cfg, s, tid, round_seed)
        got = t.numpy(k)
        for name, a, b in zip(("param", "m", "v", "exponents"), got, (new, qm, qv, exps)):
            _same(a, b, f"tensor {k}, {name}")


SHAPES = [[(1, 1)], [(1, 3), (7, 13), (1, 255), (256, 1), (1, 257)], [(64, 64), (4, 768)], [(300, 77)],
          [(128, 256), (1, 4096), (3, 1365), (5, 821)], [(3, k + 1) for k in range(60)]]


@pytest.mark.parametrize("round_seed", [None, 0, 2 ** 63 + 12345])
@pytest.mark.parametrize("at", range(len(SHAPES)))
def test_step_is_the_definition(dp, at, round_seed):
    torch = _torch()
    states = [_state(s, 10 * at + k, fresh=at == 3) for k, s in enumerate(SHAPES[at])]
    t = Tensors(dp, SHAPES[at], states)
    cfg = _cfg(t=1 if at == 3 else 40 + at)
    dp.dpsgd_noise_adamw8_multi(t.layers, *t.lists(), 0.0, 1.0, 9, 4, 0.125, _opt(dp, cfg), round_seed=round_seed)
    torch.cuda.synchronize()
    _check(t, states, cfg, 0.125, round_seed)


def test_many_steps(dp):
    """Ten steps, each from the codes that the one before has left."""
    torch = _torch()
    shapes = [(37, 53), (2, 300)]
    states = [_state(s, k, fresh=True) for k, s in enumerate(shapes)]
    t = Tensors(dp, shapes, states)
    m, v, exps = dp.make_states8(t.layers)
    assert all(torch.equal(a, b) for x, y in ((m, t.m), (v, t.v), (exps, t.exps)) for a, b in zip(x, y))
    for step in range(1, 11):
        cfg = _cfg(t=step)
        grads = [np.random.default_rng(100 * step + k).standard_normal(len(s[0])).astype(np.float32)
                 for k, s in enumerate(states)]
        for k, g in enumerate(grads):
            t.grads[k].copy_(_dev(g.reshape(shapes[k])))
        dp.dpsgd_noise_adamw8_multi(t.layers, *t.lists(), 0.0, 1.0, 9, 4, 0.5, _opt(dp, cfg), round_seed=77)
        torch.cuda.synchronize()
        states = [(g, *s[1:]) for g, s in zip(grads, states)]
        _check(t, states, cfg, 0.5, 77)
        states = [(s[0], *t.numpy(k)) for k, s in enumerate(states)]


@pytest.mark.parametrize("round_seed", [None, 5])
def test_with_noise(dp, round_seed):
    """The noisy gradient is dpsgd_noise_adamw's bit for bit, and the step the definition's
    on it."""
    torch = _torch()
    shapes = [(37, 53), (64, 256), (1, 3)]
    states = [_state(s, 20 + k) for k, s in enumerate(shapes)]
    t = Tensors(dp, shapes, states)
    cfg, noise = _cfg(t=3), (0.8, 1.5, 42, 6, 0.03125)
    noisy = [torch.empty(s, device="cuda") for s in shapes]
    wide = [torch.empty(s, device="cuda") for s in shapes]
    zeros = [[torch.zeros(s, device="cuda") for s in shapes] for _ in range(3)]
    dp.dpsgd_noise_adamw_multi(t.layers, t.grads, *zeros, *noise, _opt(dp, cfg), noisy_outs=wide)
    dp.dpsgd_noise_adamw8_multi(t.layers, *t.lists(), *noise, _opt(dp, cfg), round_seed=round_seed,
                                noisy_outs=[noisy[0], noisy[1], noisy[2]])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(noisy, wide))
    _check(t, states, cfg, None, round_seed, noisy)
    again = Tensors(dp, shapes, states)
    dp.dpsgd_noise_adamw8_multi(again.layers, *again.lists(), *noise, _opt(dp, cfg), round_seed=round_seed,
                                noisy_outs=[None, torch.empty(shapes[1], device="cuda"), None])
    torch.cuda.synchronize()
    assert all(np.array_equal(a, b) for k in range(3) for a, b in zip(t.numpy(k), again.numpy(k)))


def test_what_is_not_finite(dp):
    """A NaN or infinite moment makes its block NaN, and leaves the others; the parameters
    of its own entry alone are NaN in that step."""
    torch = _torch()
    shapes = [(3, 400)]
    grad, param, m, v, exps = _state(shapes[0], 2)
    grad[300], grad[900], grad[1100] = np.nan, np.inf, 1e30
    states = [(grad, param, m, v, exps)]
    t = Tensors(dp, shapes, states)
    cfg = _cfg()
    dp.dpsgd_noise_adamw8_multi(t.layers, *t.lists(), 0.0, 1.0, 0, 0, 1.0, _opt(dp, cfg))
    torch.cuda.synchronize()
    _check(t, states, cfg, 1.0, None)
    p = t.params[0].view(-1)
    assert bool(torch.isnan(p[300])) and int(torch.isnan(p).sum()) == 2   # inf / inf too
    back = [[torch.empty(shapes[0], device="cuda")] for _ in range(2)]
    dp.dpsgd_adamw8_unpack_multi(t.layers, t.m, t.v, t.exps, *back)
    bad = torch.isnan(back[0][0].view(-1))
    blocks = bad.view(-1)[:1024].view(4, 256)
    assert bool(blocks[1].all()) and bool(blocks[3].all()) and not bool(blocks[0].any()) and not bool(blocks[2].any())
    # 1e30 squared is beyond float32: v's block alone.
    assert not bool(bad[1024:].any()) and bool(torch.isnan(back[1][0].view(-1)[1024:]).all())


def test_small_moments(dp):
    """Gradients down to where squares leave float32: nothing is divided by a v that was
    lost, and a v above 0 stays above 0."""
    torch = _torch()
    shapes = [(8, 256)]
    rng = np.random.default_rng(4)
    n = 2048
    grad = (rng.standard_normal(n) * 10.0 ** np.repeat([-25, -20, -15, -10, -5, 0, 5, 10], 256)).astype(np.float32)
    grad[::7] *= np.float32(1e-6)
    states = [(grad, np.ones(n, np.float32), np.zeros(n, np.uint8), np.zeros(n, np.uint8), np.zeros((8, 2), np.uint8))]
    t = Tensors(dp, shapes, states)
    for step in (1, 2, 3):
        cfg = _cfg(t=step, eps=1e-12)
        dp.dpsgd_noise_adamw8_multi(t.layers, *t.lists(), 0.0, 1.0, 0, 0, 1.0, _opt(dp, cfg), round_seed=3)
        torch.cuda.synchronize()
        _check(t, states, cfg, 1.0, 3)
        states = [(grad, *t.numpy(0))]
    v = t.v[0].view(-1).cpu().numpy()
    with np.errstate(under="ignore"):
        assert (v[(np.float32(0.001) * (grad * grad)) > 0] > 0).all()


@pytest.mark.parametrize("n", [1, 255, 256, 257, 5000])
def test_pack_and_unpack(dp, n):
    torch = _torch()
    rng = np.random.default_rng(n)
    size = 10.0 ** rng.uniform(-30, 4, n)
    m, v = (rng.standard_normal(n) * size).astype(np.float32), (rng.random(n) * size).astype(np.float32)
    if n > 300:
        v[5], v[600], m[900], m[2000], v[1400] = -1.0, np.inf, np.nan, -np.inf, -0.0
    L = [dp.shape_layer(1, 1, n, 1, dp.DPSGD_F32, 0)]
    ms, vs, exps = dp.make_states8(L)
    dp.dpsgd_adamw8_pack_multi(L, [_dev(m)], [_dev(v)], ms, vs, exps)
    km, kv = lo.block_exponents(m, "m"), lo.block_exponents(v, "v")
    for i in np.flatnonzero(v < 0):
        kv[i // 256] = 255
    torch.cuda.synchronize()
    _same(exps[0].cpu().numpy(), np.stack([km, kv], 1).astype(np.uint8), "exponents")
    qm, qv = lo.encode(m, km, "m"), lo.encode(v, kv, "v")
    _same(ms[0].view(-1).cpu().numpy(), qm, "m")
    _same(vs[0].view(-1).cpu().numpy(), qv, "v")
    for dtype in (torch.float32, torch.bfloat16):
        out = [[torch.empty(1, n, dtype=dtype, device="cuda")] for _ in range(2)]
        dp.dpsgd_adamw8_unpack_multi(L, ms, vs, exps, *out)
        torch.cuda.synchronize()
        _same(out[0][0].float().view(-1).cpu().numpy(), lo.decode(qm, km, "m"), "m read back")
        _same(out[1][0].float().view(-1).cpu().numpy(), lo.decode(qv, kv, "v"), "v read back")


def test_every_code(dp):
    """Every code at low, middle and high exponents, read back in both types."""
    torch = _torch()
    ks = [0, 1, 31, 32, 48, 100, 127, 200, 254, 255]
    codes = np.tile(np.arange(256, dtype=np.uint8), len(ks))
    exps = np.array([[k, k] for k in ks], np.uint8)
    L = [dp.shape_layer(1, 1, 256, len(ks), dp.DPSGD_F32, 0)]
    for dtype in (torch.float32, torch.bfloat16):
        out = [[torch.empty(len(ks), 256, dtype=dtype, device="cuda")] for _ in range(2)]
        dp.dpsgd_adamw8_unpack_multi(L, [_dev(codes)], [_dev(codes)], [_dev(exps)], *out)
        torch.cuda.synchronize()
        for o, which in zip(out, "mv"):
            ref = lo.decode(codes, exps[:, 0], which)
            keep = np.ones(len(ref), bool) if dtype == torch.float32 else np.repeat(np.array(ks) >= 32, 256)
            if dtype == torch.bfloat16 and which == "v":
                keep = np.repeat(np.array(ks) >= 48, 256)
            _same(o[0].float().view(-1).cpu().numpy()[keep], ref[keep], which)


def test_neighbours_are_not_touched(dp):
    """Tensors of odd sizes inside larger buffers: what lies behind them stays."""
    torch = _torch()
    n = 259
    state = _state((1, n), 1)
    bufs = [torch.full((n + 64,), 7.0, device="cuda") for _ in range(2)] + [
        torch.full((n + 64,), 7, dtype=torch.uint8, device="cuda") for _ in range(3)]
    views = [b[:n].view(1, n) for b in bufs[:4]] + [bufs[4][:4].view(2, 2)]
    for view, x in zip(views, state):
        view.copy_(_dev(x).view(view.shape))
    L = [dp.shape_layer(1, 1, n, 1, dp.DPSGD_F32, 11)]
    cfg = _cfg()
    dp.dpsgd_noise_adamw8_multi(L, *[[v] for v in views], 0.0, 1.0, 0, 0, 1.0, _opt(dp, cfg), round_seed=8)
    torch.cuda.synchronize()
    new, qm, qv, exps, _ = lo.adamw8_step(*state, cfg, 1.0, 11, 8)
    for view, ref in zip(views[1:], (new, qm, qv, exps)):
        _same(view.cpu().numpy().reshape(-1), ref.reshape(-1), "state")
    assert all(bool((b[n:] == 7).all()) for b in bufs[:4]) and bool((bufs[4][4:] == 7).all())


def test_graph_replays(dp):
    """A captured step, replayed: every replay is a step with the same t and random bits."""
    torch = _torch()
    shapes = [(64, 40), (9, 111)]
    states = [_state(s, 50 + k) for k, s in enumerate(shapes)]
    t, eager = Tensors(dp, shapes, states), Tensors(dp, shapes, states)
    cfg = _cfg()

    def step(x):
        dp.dpsgd_noise_adamw8_multi(x.layers, *x.lists(), 0.5, 1.0, 3, 4, 0.5, _opt(dp, cfg), round_seed=6)

    step(t)
    step(eager)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(t)
    for _ in range(3):
        graph.replay()
        step(eager)
        torch.cuda.synchronize()
        assert all(np.array_equal(a, b) for k in range(2) for a, b in zip(t.numpy(k), eager.numpy(k)))


def test_mean_of_stochastic_rounding(dp):
    """v's slow decay is kept on average: from one code's value, with gradients of zero, the
    mean over the entries follows beta2^t, where rounding to nearest does not move."""
    torch = _torch()
    n, steps = 1 << 18, 20
    L = [dp.shape_layer(1, 1, n, 1, dp.DPSGD_F32, 0)]
    zero = torch.zeros(1, n, device="cuda")
    means = {}
    for seed in (None, 9):
        m, v, exps = dp.make_states8(L)
        dp.dpsgd_adamw8_pack_multi(L, [zero], [torch.ones(1, n, device="cuda")], m, v, exps)
        p = torch.zeros(1, n, device="cuda")
        for t in range(1, steps + 1):
            dp.dpsgd_noise_adamw8_multi(L, [zero], [p], m, v, exps, 0.0, 1.0, 0, 0, 1.0,
                                        dp.make_adamw(1e-3, t=t), round_seed=seed)
        out = [[torch.empty(1, n, device="cuda")] for _ in range(2)]
        dp.dpsgd_adamw8_unpack_multi(L, m, v, exps, *out)
        means[seed] = float(out[1][0].double().mean())
    assert means[None] == 1.0
    # An entry's deviation is below a step of 1/8 each time it moves: after 20 steps its
    # standard deviation is below 0.1, the mean's below 2e-4; six of them.
    assert abs(means[9] - 0.999 ** steps) <= 1.2e-3


def test_binding_refuses_wrong_tensors(dp):
    torch = _torch()
    shapes = [(8, 16), (3, 5)]
    t = Tensors(dp, shapes, [_state(s, k) for k, s in enumerate(shapes)])

    def call(at, k, tensor):
        lists = [list(x) for x in t.lists()]
        lists[at][k] = tensor
        dp.dpsgd_noise_adamw8_multi(t.layers, *lists, 0.0, 1.0, 0, 0, 1.0, dp.make_adamw(1e-3))

    before = t.numpy(0) + t.numpy(1)
    wrong = [(0, 1, torch.zeros(3, 4, device="cuda")), (0, 0, torch.zeros(8, 16)),
             (1, 0, torch.zeros(16, 8, device="cuda").t()), (1, 1, torch.zeros(3, 5, dtype=torch.bfloat16, device="cuda")),
             (2, 0, torch.zeros(8, 16, device="cuda")), (3, 1, torch.zeros(3, 6, dtype=torch.uint8, device="cuda")),
             (4, 0, torch.zeros(2, 2, dtype=torch.uint8, device="cuda"))]
    for at, k, tensor in wrong:
        with pytest.raises(ValueError):
            call(at, k, tensor)
    with pytest.raises(ValueError):
        dp.dpsgd_adamw8_unpack_multi(t.layers, t.m, t.v, t.exps, t.params[:1], t.params)
    with pytest.raises(dp.DpsgdError):   # off 16 bytes
        call(0, 1, torch.zeros(17, device="cuda")[1:16].view(3, 5))
    torch.cuda.synchronize()
    assert all(np.array_equal(a, b) for a, b in zip(before, t.numpy(0) + t.numpy(1)))
