#!/usr/bin/env python
"""A small training run with every piece of the library that a step uses.

    python -m paper_2506_00486_b200.train_example [--task features|tokens] [--bits 8] [--steps 200] [--lam 1e-6]

Features: a residual MLP with layer norm learns a random teacher of the same shape.  Tokens: a decoder of gated blocks with dropout
(no attention: a token's successor depends on it alone) learns the successors of a random Markov chain by the cross entropy over its
vocabulary (gg_gated_linear, gg_dropout, gg_cross_entropy and their gradients).  Weights are drawn from a GG (gg_sample), the
forward and backward passes use gg_layer_norm and gg_layer_norm_grad (matrix products are torch's), the GG penalty of the
weights is fitted and its gradient added to the loss's (gg_fused), and the step clips by the global norm and updates bf16
weights with 32- or 8-bit states (gg_grad_norm, gg_adamw_step).

A backward pass through the autograd forms below may be captured into a graph like any other of torch: with leaves whose eager graphs
are gone, since torch ties their gradients to the stream that first made them.  Context's make_* calls have no such tie.  Dropout in such
a step takes its counter from the device.
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


def _matrix(t):
    """The rows of t as a matrix that the library reads: contiguous rows that do not overlap."""
    rows = t.reshape(-1, t.shape[-1])
    return rows if rows.stride(1) == 1 and rows.stride(0) >= rows.shape[1] else rows.contiguous()


class GatedLinear(torch.autograd.Function):
    """act(x @ w_gate.t()) * (x @ w_up.t()) over the last dimension for autograd, all bfloat16.

    GatedLinear.apply(x, w_gate, w_up, ctx, act="silu").  Its gradient cannot be differentiated again."""

    @staticmethod
    def forward(fctx, x, w_gate, w_up, ctx, act="silu"):
        rows, w_gate, w_up = _matrix(x), _matrix(w_gate), _matrix(w_up)
        out = ctx.gg_gated_linear(rows, w_gate, w_up, act=act, keep=any(fctx.needs_input_grad[:3]))
        fctx.save_for_backward(rows, w_gate, w_up, out["gate"], out["up"])
        fctx.ctx, fctx.act, fctx.shape = ctx, act, x.shape
        return out["h"].view(*x.shape[:-1], w_gate.shape[0])

    @staticmethod
    @once_differentiable
    def backward(fctx, dh):
        rows, w_gate, w_up, gate, up = fctx.saved_tensors
        want_dx, *want = fctx.needs_input_grad[:3]
        out = fctx.ctx.gg_gated_linear_grad(_matrix(dh), rows, w_gate, w_up, gate, up, act=fctx.act, want_dx=want_dx, want_dweight=any(want))
        return (out["dx"].view(fctx.shape) if want_dx else None, *(out[n] if w else None for n, w in zip(("dw_gate", "dw_up"), want)), None, None)


class CrossEntropy(torch.autograd.Function):
    """The cross entropy of the logits h @ w.t(), which are never stored, for autograd: float32 losses of h's leading shape.

    CrossEntropy.apply(h, w, target, ctx): h and w bfloat16, target int64 of h's leading shape, negative where there is none (its loss
    is 0: divide the sum by the number of the others for a mean).  Its gradient cannot be differentiated again."""

    @staticmethod
    def forward(fctx, h, w, target, ctx):
        rows, w, flat = _matrix(h), _matrix(w), target.reshape(-1).contiguous()
        out = ctx.gg_cross_entropy(rows, w, flat)
        fctx.save_for_backward(rows, w, flat, out["lse"])
        fctx.ctx, fctx.shape = ctx, h.shape
        return out["loss"].view(target.shape)

    @staticmethod
    @once_differentiable
    def backward(fctx, dloss):
        rows, w, target, lse = fctx.saved_tensors
        want_dh, want_dw = fctx.needs_input_grad[:2]
        out = fctx.ctx.gg_cross_entropy_grad(dloss.reshape(-1).contiguous(), rows, w, target, lse, want_dh=want_dh, want_dw=want_dw)
        return out["dh"].view(fctx.shape) if want_dh else None, out["dw"], None, None


class Dropout(torch.autograd.Function):
    """residual + dropout of x (residual may be None) over the last dimension for autograd; the mask is drawn again for the gradient.

    Dropout.apply(x, residual, p, ctx, seed, t, tensor_id): seed, step t and tensor_id as in Context.make_dropout.  A graph keeps a t that is a
    number, and every replay draws one mask: a step that is captured takes an int64 device tensor of one value for t and advances it
    after its backward pass.  Its gradient cannot be differentiated again."""

    @staticmethod
    def forward(fctx, x, residual, p, ctx, seed, t, tensor_id):
        t_dev = t if isinstance(t, torch.Tensor) else None

        def draw(v, r=None):
            return ctx.gg_dropout(_matrix(v), p, t if t_dev is None else 0, residual=None if r is None else _matrix(r), seed=seed, tensor_id=tensor_id,
                                  t_dev=t_dev)["y"].view(v.shape)

        fctx.draw = draw
        fctx.save_for_backward(t_dev)
        return draw(x, residual)

    @staticmethod
    @once_differentiable
    def backward(fctx, dy):
        fctx.saved_tensors       # (raises if the step has been advanced since: this would be another mask)
        return fctx.draw(dy) if fctx.needs_input_grad[0] else None, dy if fctx.needs_input_grad[1] else None, None, None, None, None, None


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


def draws(seed):
    """The seeds of a decoder's initial weights, dropout masks and rounding: one generator serves all three, counted by tensor and
    step, and with one seed it would round an update by the bits that dropped an element of the same number."""
    return dict(weights=seed + (1 << 32), dropout=seed, rounding=seed + (2 << 32))


class Decoder:
    """Token embedding, `layers` blocks x + dropout(W_down (silu(W_gate norm(x)) * W_up norm(x))), norm, output matrix; all bf16."""

    def __init__(self, ctx, layers, width, hidden, vocab, beta, p, seed):
        dev = ctx.device
        self.ctx, self.layers, self.p, self.seed = ctx, layers, p, draws(seed)["dropout"]
        shapes = [s for _ in range(layers) for s in ((hidden, width), (hidden, width), (width, hidden))] + [(vocab, width)] * 2
        self.matrices = [torch.empty(s, dtype=torch.bfloat16, device=dev) for s in shapes]
        ctx.gg_sample([m.view(-1) for m in self.matrices], [beta] * len(shapes), [gg_init_alpha(s[1], 2.0, beta) for s in shapes], draws(seed)["weights"])
        self.vectors = [f(width, dtype=torch.bfloat16, device=dev) for _ in range(layers + 1) for f in (torch.ones, torch.zeros)]

    @property
    def parameters(self):
        return self.matrices + self.vectors

    def __call__(self, tokens, target, t):
        """The loss of every position in step t."""
        *blocks, embedding, output = self.matrices
        x = embedding[tokens]
        for i in range(self.layers):
            w_gate, w_up, w_down = blocks[3 * i:3 * i + 3]
            h = GatedLinear.apply(LayerNorm.apply(x, self.vectors[2 * i], self.vectors[2 * i + 1], self.ctx), w_gate, w_up, self.ctx)
            x = Dropout.apply(h @ w_down.t(), x, self.p, self.ctx, self.seed, t, i)
        return CrossEntropy.apply(LayerNorm.apply(x, *self.vectors[-2:], self.ctx), output, target, self.ctx)


def stepper(ctx, model, bits, lam, seed):
    """The flat gradients' views and what ends a step: the GG penalty of the matrices, and the clipped AdamW step."""
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
    return params, penalty, step


def train_tokens(ctx, bits=8, steps=200, lam=1e-6, lr=2e-3, layers=2, width=256, hidden=512, vocab=1000, batch=512, p=0.1, seed=1):
    """As train, for the decoder: every token has four successors, and a tenth of the positions has no target."""
    model = Decoder(ctx, layers, width, hidden, vocab, 1.0, p, seed)
    params, penalty, step = stepper(ctx, model, bits, lam, draws(seed)["rounding"])
    gen = torch.Generator(device=ctx.device).manual_seed(seed)
    successors = torch.randint(0, vocab, (vocab, 4), generator=gen, device=ctx.device)
    losses, scales = [], []
    for t in range(1, steps + 1):
        tokens = torch.randint(0, vocab, (batch,), generator=gen, device=ctx.device)
        target = successors[tokens, torch.randint(0, 4, (batch,), generator=gen, device=ctx.device)]
        target = torch.where(torch.rand(batch, generator=gen, device=ctx.device) < 0.1, -100, target)
        loss = model(tokens, target, t).sum() / (target >= 0).sum().clamp_min(1)
        for q in params:
            q.grad.zero_()
        loss.backward()
        penalty()
        scales.append(step(t, lr)["scale"].clone())
        losses.append(loss.detach())
    torch.cuda.synchronize(ctx.device)
    ctx.gg_product_status()
    return torch.stack(losses), torch.cat(scales), penalty.outputs["beta"].clone()


def train(ctx, bits=8, steps=200, lam=1e-6, lr=2e-3, layers=2, width=256, hidden=512, batch=512, seed=1):
    """Returns the loss of every step, the clip factors and the fitted shape of each matrix at the end, as tensors."""
    teacher, model = (Mlp(ctx, layers, width, hidden, beta, s) for beta, s in ((2.0, seed + 100), (1.0, seed)))
    params, penalty, step = stepper(ctx, model, bits, lam, seed)
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
    ap.add_argument("--task", choices=("features", "tokens"), default="features")
    ap.add_argument("--bits", type=int, choices=(32, 8), default=8)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--lam", type=float, default=1e-6)
    a = ap.parse_args()
    losses, scales, beta = (train if a.task == "features" else train_tokens)(Context(0), a.bits, a.steps, a.lam)
    for t in range(0, a.steps, max(1, a.steps // 10)):
        print(f"step {t + 1:5d}  loss {losses[t].item():.4f}  clip {scales[t].item():.3f}")
    print(f"step {a.steps:5d}  loss {losses[-1].item():.4f}  fitted shapes {[round(b, 2) for b in beta.tolist()]}")


if __name__ == "__main__":
    main()
