"""A text classifier trained privately from end to end by the library: every trainable
tensor, not only the linear layers' weights, enters the per-example norm, the clipped
sum, the noise and the optimizer step.

The model: token embedding (scaled by sqrt(d), padding is id -1), blocks of a
convolution over the sequence (a linear layer over unfolded rows, kernel 3), group norm
and SiLU over channels-last rows, the mean over the positions, a linear classifier with
a bias. Group norm acts within an example, so that per-example gradients exist (Section
2.2 of the paper); every parameter is trained:

* the token table, through ``dpsgd_embedding_norms`` and
  ``dpsgd_embedding_clip_accumulate``;
* convolution and classifier weights, as layers of captured activations and output
  gradients;
* the group norms' gamma and beta and the classifier's bias, whose per-example
  gradients [B, C] are layers with activations of 1 (``affine_layer``).

A step is the paper's: norms over all of it, clipped sums, noise and the average; then
one norm over the noisy gradient bounds it (``dpsgd_global_clip_multi``) and AdamW takes
it. torch runs the convolutions' and the classifier's products and their backward; the
lookup, group norms and everything after the backward are the library's. Weights and
texts are random (no dataset here).
"""

from __future__ import annotations

import math
from dataclasses import dataclass

import torch
import torch.nn.functional as F

from . import dpsgd


@dataclass
class TextConvConfig:
    vocab: int = 32003
    d: int = 128           # width of the token table
    channels: int = 256
    groups: int = 16
    blocks: int = 2
    classes: int = 4
    eps: float = 1e-5


class _Lookup(torch.autograd.Function):
    """Rows of the token table; the gradient of the rows is left in `record`."""

    @staticmethod
    def forward(ctx, table, emb, record):
        out = torch.empty(emb.B, emb.T, emb.d, device=table.device)
        dpsgd.dpsgd_embedding_lookup(emb, table, out)
        ctx.record = record
        return out

    @staticmethod
    def backward(ctx, grad):
        ctx.record["rows"] = grad.contiguous()
        return None, None, None


class _GroupNormAct(torch.autograd.Function):
    """Group norm and SiLU; per-example gradients of gamma and beta are left in `record`."""

    @staticmethod
    def forward(ctx, x, gamma, beta, groups, eps, record):
        x = x.contiguous()
        gn = dpsgd.make_group_norm(x, groups, gamma, beta, eps, "silu")
        y = torch.empty_like(x)
        mean, rstd = (torch.empty(x.shape[0], groups, device=x.device) for _ in range(2))
        ctx.ws = torch.empty(dpsgd.dpsgd_group_norm_workspace_bytes(gn), dtype=torch.uint8,
                             device=x.device)
        dpsgd.dpsgd_group_norm_forward(gn, x, y, mean, rstd, workspace=ctx.ws)
        ctx.save_for_backward(x, mean, rstd)
        ctx.gn, ctx.record = gn, record
        return y

    @staticmethod
    def backward(ctx, dy):
        x, mean, rstd = ctx.saved_tensors
        dx = torch.empty_like(x)
        dgamma, dbeta = (torch.empty(x.shape[0], x.shape[-1], device=x.device) for _ in range(2))
        dpsgd.dpsgd_group_norm_backward(ctx.gn, x, dy.contiguous(), mean, rstd, dx, dgamma, dbeta,
                                        workspace=ctx.ws)
        ctx.record["gamma"], ctx.record["beta"] = dgamma, dbeta
        return dx, None, None, None, None, None


def unfold(x):
    """[B, T, C] -> [B, T, 3 C]: each position with its neighbours (zeros outside)."""
    p = F.pad(x, (0, 0, 1, 1))
    return torch.cat([p[:, :-2], p[:, 1:-1], p[:, 2:]], dim=2).contiguous()


class TextConv:
    """Parameters (float32, on the device) by name, in a fixed order. Vectors are [n, 1],
    the shape of their layers."""

    def __init__(self, cfg: TextConvConfig = TextConvConfig(), seed: int = 0, device="cuda"):
        gen = torch.Generator().manual_seed(seed)
        self.cfg = cfg
        self.params: dict[str, torch.Tensor] = {
            "table": torch.randn(cfg.vocab, cfg.d, generator=gen) * 0.02}
        c = cfg.d
        for k in range(cfg.blocks):
            self.params[f"conv{k}"] = (torch.randn(cfg.channels, 3 * c, generator=gen)
                                       * math.sqrt(2.0 / (3 * c)))
            self.params[f"gamma{k}"] = torch.ones(cfg.channels, 1)
            self.params[f"beta{k}"] = torch.zeros(cfg.channels, 1)
            c = cfg.channels
        self.params["head"] = torch.randn(cfg.classes, c, generator=gen) / math.sqrt(c)
        self.params["bias"] = torch.zeros(cfg.classes, 1)
        self.params = {k: v.to(device) for k, v in self.params.items()}

    def embedding(self, ids) -> dpsgd.dpsgd_embedding:
        return dpsgd.make_embedding(ids, self.params["table"].shape, math.sqrt(self.cfg.d))

    def backward(self, ids, labels):
        """Losses [B], and what the step needs of one backward pass of their sum: the
        layers (name, activations, output gradients) and the rows' gradients."""
        cfg, p = self.cfg, self.params
        B = ids.shape[0]
        record = {"rows": {}}
        # The lookup has no gradient of its own: its output starts the graph.
        x = _Lookup.apply(p["table"].detach().requires_grad_(), self.embedding(ids), record["rows"])
        there = (ids >= 0).unsqueeze(-1).to(x.dtype)
        layers = []
        for k in range(cfg.blocks):
            a = unfold(x)
            y = F.linear(a, p[f"conv{k}"])
            layers.append((f"conv{k}", a.detach(), _tap(y)))
            record[k] = {}
            x = _GroupNormAct.apply(y, p[f"gamma{k}"].view(-1), p[f"beta{k}"].view(-1),
                                    cfg.groups, cfg.eps, record[k])
        pooled = (x * there).sum(1) / there.sum(1).clamp(min=1.0)
        logits = F.linear(pooled, p["head"], p["bias"].view(-1))
        head = _tap(logits)
        losses = F.cross_entropy(logits, labels, reduction="none")
        losses.sum().backward()
        ones = torch.ones(B, device=ids.device)
        out = []
        for k, (name, a, g) in enumerate(layers):
            out.append((name, a, g[0].contiguous()))
            out.append((f"gamma{k}", ones.view(B, 1, 1), record[k]["gamma"].view(B, 1, -1)))
            out.append((f"beta{k}", ones.view(B, 1, 1), record[k]["beta"].view(B, 1, -1)))
        out.append(("head", pooled.detach().view(B, 1, -1), head[0].contiguous().view(B, 1, -1)))
        out.append(("bias", ones.view(B, 1, 1), head[0].contiguous().view(B, 1, -1)))
        return losses.detach(), out, record["rows"]["rows"]


def _tap(t):
    """A list that the backward pass leaves t's gradient in."""
    got = []
    t.register_hook(lambda g: got.append(g.detach()))
    return got


class PrivateTrainer:
    """The private step over a TextConv's parameters, its buffers and AdamW's moments."""

    def __init__(self, model: TextConv, C: float, sigma: float, seed: int, lr: float = 1e-3,
                 max_norm: float = math.inf, weight_decay: float = 0.01):
        dpsgd.load()
        self.model, self.C, self.sigma, self.seed = model, C, sigma, seed
        self.lr, self.max_norm, self.weight_decay = lr, max_norm, weight_decay
        self.names = list(model.params)
        self.shapes = [dpsgd.shape_layer(1, 1, p.shape[1], p.shape[0], dpsgd.DPSGD_F32, k)
                       for k, p in enumerate(model.params.values())]
        dev = model.params["table"].device
        self.grads, self.m, self.v = ([torch.zeros_like(p) for p in model.params.values()]
                                      for _ in range(3))
        self.norm = torch.empty(1, device=dev)   # of the noisy gradient, before clipping
        self.clip_ws = torch.empty(dpsgd.dpsgd_global_norm_workspace_bytes(self.shapes),
                                   dtype=torch.uint8, device=dev)
        self.t = 0

    def sums(self, ids, labels):
        """Losses, squared per-example norms over every parameter, clip factors; the
        clipped sums are in self.grads."""
        losses, layers, rows = self.model.backward(ids, labels)
        by_name = dict(zip(self.names, range(len(self.names))))
        Ls = [dpsgd.make_layer(A, G, by_name[name]) for name, A, G in layers]
        dev, B = ids.device, ids.shape[0]

        def ws(n):
            return torch.empty(max(n, 1), dtype=torch.uint8, device=dev)

        norms_sq, factors = torch.empty(B, device=dev), torch.empty(B, device=dev)
        emb = self.model.embedding(ids)
        emb_ws = ws(dpsgd.dpsgd_embedding_workspace_bytes(emb))
        dpsgd.dpsgd_per_example_norms_multi(Ls, dpsgd.DPSGD_NORM_AUTO, norms_sq,
                                            workspace=ws(dpsgd.dpsgd_norms_workspace_bytes(Ls)))
        dpsgd.dpsgd_embedding_norms(emb, rows, norms_sq, accumulate=True, workspace=emb_ws)
        dpsgd.dpsgd_clip_accumulate_multi(Ls, norms_sq, self.C,
                                          [self.grads[by_name[n]] for n, _, _ in layers],
                                          factors_out=factors,
                                          workspace=ws(dpsgd.dpsgd_clip_workspace_bytes(Ls)))
        dpsgd.dpsgd_embedding_clip_accumulate(emb, rows, norms_sq, self.C,
                                              self.grads[by_name["table"]], workspace=emb_ws)
        return losses, norms_sq, factors

    def step(self, ids, labels):
        """One step: clipped sums, noise and average, one norm over the noisy gradient,
        AdamW. Returns the losses (before the step)."""
        losses, _, _ = self.sums(ids, labels)
        dpsgd.dpsgd_add_noise_multi(self.shapes, self.grads, self.sigma, self.C, self.seed, self.t,
                                    1.0 / ids.shape[0])
        dpsgd.dpsgd_global_clip_multi(self.shapes, self.grads, self.grads, self.max_norm, self.norm,
                                      workspace=self.clip_ws)
        self.t += 1
        opt = dpsgd.make_adamw(self.lr, weight_decay=self.weight_decay, t=self.t)
        # The noise is in the gradient already: sigma 0 adds none.
        dpsgd.dpsgd_noise_adamw_multi(self.shapes, self.grads, list(self.model.params.values()),
                                      self.m, self.v, 0.0, self.C, self.seed, self.t, 1.0, opt)
        return losses


def synthetic_texts(cfg: TextConvConfig, B: int, T: int, seed: int, device):
    """Texts of random words (frequency 1 / rank) and lengths, padded with -1, whose class
    decides where in the vocabulary every fourth word is from."""
    gen = torch.Generator().manual_seed(seed)
    labels = torch.randint(0, cfg.classes, (B,), generator=gen)
    u = torch.rand(B, T, generator=gen, dtype=torch.float64)
    ids = (torch.exp(u * math.log(cfg.vocab + 1)) - 1).long().clamp_(0, cfg.vocab - 1)
    topic = torch.rand(B, T, generator=gen) < 0.25
    ids = torch.where(topic, cfg.vocab - 1 - (labels.unsqueeze(1) * 8 + ids % 8), ids)
    n = torch.randint(max(1, T // 2), T + 1, (B, 1), generator=gen)
    ids = torch.where(torch.arange(T) < n, ids, -1)
    return ids.to(device), labels.to(device)


def bench(B: int = 128, T: int = 256, steps: int = 20, sigma: float = 0.5) -> dict:
    """Trains on cuda:0; returns the first and the last loss and the time of a step."""
    cfg = TextConvConfig()
    trainer = PrivateTrainer(TextConv(cfg), C=1.0, sigma=sigma, seed=7, max_norm=1.0)
    batches = [synthetic_texts(cfg, B, T, k, "cuda") for k in range(4)]
    losses = [float(trainer.step(*batches[0]).mean())]
    torch.cuda.synchronize()
    e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    e0.record()
    for k in range(steps):
        last = trainer.step(*batches[(k + 1) % 4])
    e1.record()
    torch.cuda.synchronize()
    losses.append(float(last.mean()))
    return {"model": "text convolution, group norm, every parameter private", "B": B, "T": T,
            "parameters": sum(p.numel() for p in trainer.model.params.values()),
            "loss_first": losses[0], "loss_last": losses[-1], "steps": steps,
            "gradient_norm": float(trainer.norm), "ms_per_step": e0.elapsed_time(e1) / steps}


if __name__ == "__main__":
    import json
    import sys

    args = dict(a.split("=", 1) for a in sys.argv[1:])
    print(json.dumps(bench(B=int(args.get("B", 128)), T=int(args.get("T", 256)),
                           steps=int(args.get("steps", 20)),
                           sigma=float(args.get("sigma", 0.5)))), flush=True)
