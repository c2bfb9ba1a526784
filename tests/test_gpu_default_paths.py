"""Which of the library's calls the paths with options make: without an option the loss,
norms and moments are torch's and the float32 step's, and with it they are not. (That the
default step's results are right, float64 says elsewhere in this suite.)"""

import pytest

pytestmark = pytest.mark.gpu

LOSS, STEP, STEP8, NORM = ("dpsgd_token_loss", "dpsgd_noise_adamw_multi", "dpsgd_noise_adamw8_multi",
                           "dpsgd_residual_norm_forward")


@pytest.fixture
def calls(monkeypatch, dp):
    """Names of the library's calls, in order."""
    import torch
    made = []

    def record(module, name):
        f = getattr(module, name)

        def call(*a, **kw):
            made.append(name)
            return f(*a, **kw)
        monkeypatch.setattr(module, name, call)

    for name in (LOSS, STEP, STEP8, NORM):
        record(dp, name)
    record(torch.nn.functional, "cross_entropy")
    print("[gpu] start", flush=True)
    return made


@pytest.mark.parametrize("options,want", [
    ({}, ["cross_entropy", STEP]), ({"own_loss": True}, [LOSS, STEP]), ({"moments": "8bit"}, ["cross_entropy", STEP8]),
    ({"own_loss": True, "moments": "8bit"}, [LOSS, STEP8])])
def test_calls_of_a_private_step(calls, options, want):
    import torch
    from paper_2609_20532_amd import text_conv as tc
    cfg = tc.TextConvConfig(vocab=101, d=24, channels=48, groups=6, blocks=1, classes=3)
    t = tc.PrivateTrainer(tc.TextConv(cfg, seed=2), C=0.7, sigma=0.4, seed=9, max_norm=5.0, **options)
    for k in range(2):
        losses = t.step(*tc.synthetic_texts(cfg, 4, 30, k, "cuda"))
    torch.cuda.synchronize()
    assert bool(torch.isfinite(losses).all()) and calls == 2 * want


@pytest.mark.parametrize("options,want", [({}, ["cross_entropy"]), ({"own": True}, [NORM] * 5 + [LOSS])])
def test_calls_of_a_capture(calls, options, want):
    from paper_2609_20532_amd import capture as cap
    cfg = cap.GPT2Config(n_layer=2, n_embd=32, n_head=2, vocab=61, n_ctx=16, r=2)
    model = cap.GPT2LoRA(cfg, seed=3).to("cuda")
    cap.capture(model, cap.synthetic_tokens(cfg, 2, 9, seed=1, device="cuda"), **options)
    assert calls == want
