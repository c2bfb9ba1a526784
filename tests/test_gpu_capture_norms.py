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
