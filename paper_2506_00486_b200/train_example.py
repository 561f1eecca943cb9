#!/usr/bin/env python
"""A small training run with every piece of the library that a step uses.

    python -m paper_2506_00486_b200.train_example [--bits 8] [--steps 200] [--lam 1e-6]

A residual MLP with layer norm learns a random teacher of the same shape.  Weights are drawn from a GG (gg_sample), the
forward and backward passes use gg_layer_norm and gg_layer_norm_grad (matrix products are torch's), the GG penalty of the
weights is fitted and its gradient added to the loss's (gg_fused), and the step clips by the global norm and updates bf16
weights with 32- or 8-bit states (gg_grad_norm, gg_adamw_step).
"""
import argparse

import torch
from torch.autograd.function import once_differentiable

from paper_2506_00486_b200 import Context, Segments, gg_init_alpha


class LayerNorm(torch.autograd.Function):
    """Layer norm over the last dimension for autograd: y = weight * xhat + bias, each of the two may be None.

    LayerNorm.apply(x, weight, bias, ctx, eps=1e-5).  Its gradient is that of the first order: it cannot be differentiated again.
    Every call allocates its outputs; a loop over fixed buffers is faster with Context.make_layer_norm and make_layer_norm_grad."""

    @staticmethod
    def forward(fctx, x, weight, bias, ctx, eps=1e-5):
        rows = x.reshape(-1, x.shape[-1])
        if rows.stride(1) != 1 or rows.stride(0) < rows.shape[1]:      # strided columns, rows that overlap
            rows = rows.contiguous()
        out = ctx.gg_layer_norm(rows, weight, bias, eps=eps)
        fctx.save_for_backward(rows, weight, out["mean"], out["rstd"])
        fctx.ctx, fctx.bias_dtype = ctx, None if bias is None else bias.dtype
        return out["y"].view(x.shape)

    @staticmethod
    @once_differentiable
    def backward(fctx, dy):
        rows, weight, mean, rstd = fctx.saved_tensors
        want_dx, want_dweight, want_dbias = fctx.needs_input_grad[:3]
        out = fctx.ctx.gg_layer_norm_grad(dy.reshape(rows.shape).contiguous(), rows, mean, rstd, weight, want_dx=want_dx,
                                          want_dweight=want_dweight or want_dbias)
        return (out["dx"].view(dy.shape) if want_dx else None, out["dweight"].to(weight.dtype) if want_dweight else None,
                out["dbias"].to(fctx.bias_dtype) if want_dbias else None, None, None)


class Mlp:
    """`layers` blocks x + W2 relu(W1 norm(x)), all parameters bf16."""

    def __init__(self, ctx, layers, width, hidden, beta, seed):
        dev = ctx.device
        self.ctx, self.layers = ctx, layers
        shapes = [s for _ in range(layers) for s in ((hidden, width), (width, hidden))]
        self.matrices = [torch.empty(s, dtype=torch.bfloat16, device=dev) for s in shapes]
        ctx.gg_sample([m.view(-1) for m in self.matrices], [beta] * len(shapes), [gg_init_alpha(s[1], 2.0, beta) for s in shapes], seed)
        self.vectors = [f(width, dtype=torch.bfloat16, device=dev) for _ in range(layers) for f in (torch.ones, torch.zeros)]

    @property
    def parameters(self):
        return self.matrices + self.vectors

    def __call__(self, x):
        for i in range(self.layers):
            h = LayerNorm.apply(x, self.vectors[2 * i], self.vectors[2 * i + 1], self.ctx)
            x = x + torch.relu(h @ self.matrices[2 * i].t()) @ self.matrices[2 * i + 1].t()
        return x


def train(ctx, bits=8, steps=200, lam=1e-6, lr=2e-3, layers=2, width=256, hidden=512, batch=512, seed=1):
    """Returns the loss of every step, the clip factors and the fitted shape of each matrix at the end, as tensors."""
    teacher, model = (Mlp(ctx, layers, width, hidden, beta, s) for beta, s in ((2.0, seed + 100), (1.0, seed)))
    params = model.parameters
    for p in params:
        p.requires_grad_(True)
        p.grad = torch.zeros_like(p)
    flat, grads = Segments([p.detach().view(-1) for p in params]), Segments([p.grad.view(-1) for p in params])
    k = len(model.matrices)
    # the penalty of the matrices: fitted in each step, its gradient added to what the backward pass left
    penalty = ctx.make_fused(Segments(flat.tensors[:k]), grad=Segments(grads.tensors[:k]), lam=lam, accumulate_grad=True, want_hist=False)
    decay = torch.tensor([0.01] * k + [0.0] * (len(params) - k), dtype=torch.float32, device=ctx.device)
    step = ctx.make_adamw_step(flat, grads, **ctx.adamw_state(flat, bits), weight_decay=decay, max_norm=1.0, seed=seed)
    gen = torch.Generator(device=ctx.device).manual_seed(seed)
    losses, scales = [], []
    for t in range(1, steps + 1):
        x = torch.randn((batch, width), generator=gen, device=ctx.device).bfloat16()
        loss = (model(x) - teacher(x).detach()).float().square().mean()
        for p in params:
            p.grad.zero_()
        loss.backward()
        penalty()
        scales.append(step(t, lr)["scale"].clone())
        losses.append(loss.detach())
    return torch.stack(losses), torch.cat(scales), penalty.outputs["beta"].clone()


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--bits", type=int, choices=(32, 8), default=8)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--lam", type=float, default=1e-6)
    a = ap.parse_args()
    losses, scales, beta = train(Context(0), a.bits, a.steps, a.lam)
    for t in range(0, a.steps, max(1, a.steps // 10)):
        print(f"step {t + 1:5d}  loss {losses[t].item():.4f}  clip {scales[t].item():.3f}")
    print(f"step {a.steps:5d}  loss {losses[-1].item():.4f}  fitted shapes {[round(b, 2) for b in beta.tolist()]}")


if __name__ == "__main__":
    main()
