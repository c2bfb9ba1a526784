"""The text classifier's private step on the GPU against float64: per-example gradients of
the same model by torch's differentiation on the CPU, one example at a time, then the
oracle's clip, noise and AdamW.

Tolerances: the library's float32 bounds of this suite (norms 1e-4; sums 1e-4 of a
tensor's norm); torch's float32 products of at most 768 terms add about 1e-6.
"""

import math

import numpy as np
import pytest

import oracle
from oracle import model_oracle as mo

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _announce(request):
    print(f"[gpu] start {request.node.name}", flush=True)
    yield


def _example_gradients(cfg, params, ids, label):
    """Gradients by name of one example's loss, float64 on the CPU."""
    import torch
    import torch.nn.functional as F
    p = {k: v.clone().requires_grad_() for k, v in params.items()}
    there = ids >= 0
    x = p["table"][ids.clamp(min=0)] * math.sqrt(cfg.d) * there.unsqueeze(-1)
    for k in range(cfg.blocks):
        q = F.pad(x, (0, 0, 1, 1))
        y = F.linear(torch.cat([q[:-2], q[1:-1], q[2:]], dim=1), p[f"conv{k}"])
        z = F.group_norm(y.t().unsqueeze(0), cfg.groups, p[f"gamma{k}"].view(-1),
                         p[f"beta{k}"].view(-1), cfg.eps)[0].t()
        x = F.silu(z)
    pooled = (x * there.unsqueeze(-1)).sum(0) / there.sum().clamp(min=1)
    logits = F.linear(pooled, p["head"], p["bias"].view(-1))
    loss = F.cross_entropy(logits.unsqueeze(0), label.unsqueeze(0))
    loss.backward()
    return float(loss.detach()), {k: v.grad.numpy() for k, v in p.items()}


def test_step_against_float64(dp):
    import torch
    from paper_2609_20532_amd import text_conv as tc
    cfg = tc.TextConvConfig(vocab=211, d=24, channels=48, groups=6, blocks=2, classes=3)
    model = tc.TextConv(cfg, seed=3)
    B, T, sigma, seed, max_norm, lr, wd = 6, 29, 0.3, 77, 0.05, 1e-2, 0.02
    ids, labels = tc.synthetic_texts(cfg, B, T, 5, "cuda")
    ids[2] = -1                      # an example with no token
    host = {k: v.cpu().double() for k, v in model.params.items()}
    each = [_example_gradients(cfg, host, ids[i].cpu(), labels[i].cpu()) for i in range(B)]
    names = list(model.params)
    n = np.array([math.sqrt(sum(np.sum(g[k] ** 2) for k in names)) for _, g in each])
    C = float(np.median(n))
    c = np.minimum(1.0, C / n)
    sums = {k: sum(c[i] * each[i][1][k] for i in range(B)) for k in names}

    trainer = tc.PrivateTrainer(model, C, sigma, seed, lr, max_norm, wd)
    losses, norms_sq, factors = trainer.sums(ids, labels)
    torch.cuda.synchronize()
    assert np.allclose(losses.cpu().double().numpy(), [e[0] for e in each], rtol=1e-5)
    assert np.allclose(np.sqrt(norms_sq.cpu().double().numpy()), n, rtol=1e-4)
    assert np.allclose(factors.cpu().double().numpy(), c, rtol=1e-4)
    for k, g in zip(names, trainer.grads):
        err = np.linalg.norm(g.cpu().double().numpy() - sums[k])
        assert err <= 1e-4 * np.linalg.norm(sums[k]), (k, err)

    before = [p.cpu().double().numpy() for p in model.params.values()]
    trainer.step(ids, labels)
    torch.cuda.synchronize()
    noisy = [oracle.add_noise(sums[k], sigma, C, seed, i, 0, 1.0 / B) for i, k in enumerate(names)]
    norm, factor, noisy = mo.global_clip(noisy, max_norm)
    assert factor < 1.0 and abs(float(trainer.norm) - norm) <= 1e-4 * norm
    opt = oracle.AdamWConfig(lr=lr, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=wd, t=1)
    for i, (k, g) in enumerate(zip(names, trainer.grads)):
        got = g.cpu().double().numpy()
        assert np.linalg.norm(got - noisy[i]) <= 1e-4 * np.linalg.norm(noisy[i]), k
        # AdamW on the gradient that the GPU has (its first step takes the sign of an entry,
        # which a rounding may decide).
        want = oracle.adamw_step(before[i], np.zeros_like(got), np.zeros_like(got), got, opt)[0]
        now = model.params[k].cpu().double().numpy()
        assert np.allclose(now, want, rtol=0, atol=1e-5 * lr + 1e-6 * np.abs(want).max()), k


def test_training_lowers_the_loss(dp):
    import torch
    from paper_2609_20532_amd import text_conv as tc
    cfg = tc.TextConvConfig(vocab=500, d=32, channels=64, groups=8, blocks=1, classes=4)
    trainer = tc.PrivateTrainer(tc.TextConv(cfg, seed=1), C=1.0, sigma=0.2, seed=9, lr=3e-3, max_norm=1.0)
    ids, labels = tc.synthetic_texts(cfg, 64, 40, 11, "cuda")
    losses = [float(trainer.step(ids, labels).mean()) for _ in range(25)]
    assert all(math.isfinite(v) for v in losses)
    assert losses[-1] < 0.7 * losses[0]
