"""The capture's residual norms on the GPU with parameters that are trained."""

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _announce(request):
    print(f"[gpu] start {request.node.name}", flush=True)
    yield


def _model(device, dtype):
    import torch
    from paper_2609_20532_amd import capture as cap
    cfg = cap.GPT2Config(n_layer=2, n_embd=96, n_head=4, vocab=331, n_ctx=64, r=4)
    model = cap.GPT2LoRA(cfg, seed=3).to(dtype)
    norms = [ln for blk in model.blocks for ln in (blk.ln1, blk.ln2)] + [model.ln_f]
    gen = torch.Generator().manual_seed(5)
    with torch.no_grad():
        for ln in norms:
            ln.weight.copy_(1 + 0.2 * torch.randn(96, generator=gen))
            ln.bias.copy_(0.2 * torch.randn(96, generator=gen))
    for ln in norms:
        ln.weight.requires_grad_(True)
        ln.bias.requires_grad_(True)
    return cap, cfg, model.to(device), [p for ln in norms for p in (ln.weight, ln.bias)]


@pytest.mark.parametrize("B,T", [(3, 17), (2, 64)])
def test_unfrozen_norms_have_gradients(dp, B, T):
    """As near to the float64 model's as torch's own float32 ones, within a factor for
    another order of sums."""
    import torch
    grads, tokens = {}, None
    for name, device, dtype, own in (("own", "cuda", torch.float32, True), ("torch", "cuda", torch.float32, False),
                                     ("exact", "cpu", torch.float64, False)):
        cap, cfg, model, params = _model(device, dtype)
        if tokens is None:
            tokens = cap.synthetic_tokens(cfg, B, T, seed=T, device="cuda")
        cap.capture(model, tokens.to(device), own=own)
        grads[name] = [p.grad for p in params]
    for mine, torchs, exact in zip(*(grads[n] for n in ("own", "torch", "exact"))):
        assert mine is not None

        def off(g):
            return float((g.double().cpu() - exact).norm() / exact.norm())

        assert off(mine) <= 4 * off(torchs) + 4 * 2.0 ** -24


def test_gradients_of_bf16_rows(dp):
    """bf16 rows have float32 parameters, and their gradients are float32. Against float64 on
    the r that is stored: gradients of rows are rounded to bf16 once, 2^-8 of them at most and
    2^-12 for what is formed in float32. A parameter's gradient is a float32 sum of 150 terms,
    each off by 16 u of |dy| (|vh| + 1) (u = 2^-24: mean, deviation and product), and adds
    150 u of the terms' magnitudes."""
    import torch
    from paper_2609_20532_amd import capture as cap
    gen = torch.Generator().manual_seed(4)
    x, b, wy = (torch.randn(3, 50, 96, generator=gen).to(torch.bfloat16) for _ in range(3))
    gamma, beta = 1 + 0.2 * torch.randn(96, generator=gen), 0.2 * torch.randn(96, generator=gen)
    leaves = [t.cuda().requires_grad_(True) for t in (x, b, gamma, beta)]
    _, y = cap._ResidualNorm.apply(*leaves, 1e-5)
    y.backward(wy.cuda())
    # The stored r, so that its rounding is not counted again.
    r = (x.float() + b.float()).to(torch.bfloat16).double().requires_grad_(True)
    g64, b64 = gamma.double().requires_grad_(True), beta.double().requires_grad_(True)
    torch.nn.functional.layer_norm(r, (96,), g64, b64, 1e-5).backward(wy.double())
    assert leaves[2].grad.dtype == leaves[3].grad.dtype == torch.float32
    r64 = r.detach()
    vh = (r64 - r64.mean(-1, keepdim=True)) / torch.sqrt(r64.var(-1, unbiased=False, keepdim=True) + 1e-5)
    terms = (wy.double().abs() * (vh.abs() + 1)).sum((0, 1))
    for got in (leaves[0].grad, leaves[1].grad):
        assert float((got.double().cpu() - r.grad).norm() / r.grad.norm()) <= 2.0 ** -8 + 2.0 ** -12
    for got, want in ((leaves[2].grad, g64.grad), (leaves[3].grad, b64.grad)):
        assert bool(((got.double().cpu() - want).abs() <= 166 * 2.0 ** -24 * terms).all())
