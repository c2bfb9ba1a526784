"""The autograd node of the capture's residual norms on the CPU, with the library's calls
replaced by their formulas in float64: what it saves, returns and refuses."""

from types import SimpleNamespace

import pytest
import torch

from paper_2609_20532_amd import capture as cap
from paper_2609_20532_amd import dpsgd


def _normed(v, eps):
    d = v - v.mean(-1, keepdim=True)
    rstd = 1 / torch.sqrt((d * d).mean(-1, keepdim=True) + eps)
    return d * rstd, rstd


def _make(x, kind, gamma, beta, eps):
    assert kind == "layer" and x.is_contiguous()
    return SimpleNamespace(B=x.shape[0], S=x.numel() // (x.shape[0] * x.shape[-1]), C=x.shape[-1],
                           gamma=gamma, beta=beta, eps=eps)


def _forward(desc, x, block, r, y, stats):
    total = x if block is None else x + block
    if r is not None:
        r.copy_(total)
    y.copy_(_normed(total, desc.eps)[0] * desc.gamma + desc.beta)


@torch.no_grad()   # as the library's
def _backward(desc, block, r, dy, dr, stats, dx=None, dblock=None, dgamma=None, dbeta=None, workspace=None):
    assert (block is None) == (dblock is None) and any(t is not None for t in (dx, dblock, dgamma, dbeta))
    vh, rstd = _normed(r, desc.eps)
    g = dy * desc.gamma
    dR = rstd * (g - g.mean(-1, keepdim=True) - vh * (g * vh).mean(-1, keepdim=True))
    if dr is not None:
        dR = dR + dr
    each = lambda t: t.reshape(desc.B, -1, desc.C).sum(1)
    for to, value in ((dx, lambda: dR), (dblock, lambda: dR), (dgamma, lambda: each(dy * vh)), (dbeta, lambda: each(dy))):
        if to is not None:
            to.copy_(value())


@pytest.fixture(autouse=True)
def formulas(monkeypatch):
    monkeypatch.setattr(dpsgd, "make_residual_norm", _make)
    monkeypatch.setattr(dpsgd, "dpsgd_residual_norm_forward", _forward)
    monkeypatch.setattr(dpsgd, "dpsgd_residual_norm_backward", _backward)
    monkeypatch.setattr(dpsgd, "dpsgd_residual_norm_workspace_bytes", lambda desc: 16)


def _inputs(needs):
    gen = torch.Generator().manual_seed(1)
    x, block = (torch.randn(3, 4, 6, generator=gen, dtype=torch.float64) for _ in range(2))
    gamma, beta = (torch.randn(6, generator=gen, dtype=torch.float64) for _ in range(2))
    for name, t in zip("xbgB", (x, block, gamma, beta)):
        t.requires_grad_(name in needs)
    return x, block, gamma, beta


@pytest.mark.parametrize("needs", ["xbgB", "xb", "x", "b", "gB", "g", "B", "xg", "bB"])
def test_gradients_of_the_residual_norm(needs):
    """Every input that asks for a gradient gets it, against torch's own node and differences."""
    args = _inputs(needs)
    r, y = cap._ResidualNorm.apply(*args, 1e-5)
    wr, wy = torch.randn(2, 3, 4, 6, dtype=torch.float64, generator=torch.Generator().manual_seed(2))
    ((r * wr).sum() + (y * wy).sum()).backward()
    same = [t.detach().clone().requires_grad_(t.requires_grad) for t in args]
    r2 = same[0] + same[1]
    y2 = torch.nn.functional.layer_norm(r2, (6,), same[2], same[3], 1e-5)
    ((r2 * wr).sum() + (y2 * wy).sum()).backward()
    for t, u in zip(args, same):
        assert (t.grad is None) == (u.grad is None)
        if t.grad is not None:
            assert torch.allclose(t.grad, u.grad, rtol=1e-12, atol=1e-12)
    assert torch.autograd.gradcheck(lambda *a: cap._ResidualNorm.apply(*a, 1e-5), args)


@pytest.mark.parametrize("needs", ["xgB", "x", "gB", "g"])
def test_gradients_of_the_first_norm(needs):
    x, _, gamma, beta = _inputs(needs)
    assert torch.autograd.gradcheck(lambda a, c, d: cap._ResidualNorm.apply(a, None, c, d, 1e-5),
                                    (x, gamma, beta))


@pytest.mark.parametrize("which", [2, 3])
def test_parameters_changed_before_the_backward_pass_are_noticed(which):
    args = _inputs("xbgB")
    r, y = cap._ResidualNorm.apply(*args, 1e-5)
    with torch.no_grad():
        args[which].mul_(2.0)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        (r.sum() + y.square().sum()).backward()


def test_a_second_derivative_is_refused():
    x, block, gamma, beta = _inputs("xbgB")
    _, y = cap._ResidualNorm.apply(x, block, gamma, beta, 1e-5)
    gx, = torch.autograd.grad(y.square().sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        ((gx * gx).sum() + (x * x).sum()).backward()


@pytest.mark.parametrize("used", [0, 1])
def test_one_output_alone(used):
    """The gradient of the output that nothing uses is none."""
    assert torch.autograd.gradcheck(lambda *a: cap._ResidualNorm.apply(*a, 1e-5)[used], _inputs("xbgB"))
