"""Gradients against what does not use their formulas: exact differences of the gated block, term by term, and the whole decoder in 64
bits with the roundings added as the independent errors that they are.

The block's inputs are small integers: gate and up are below 16 in magnitude, so h = relu(gate) up and the differences of two of them are exact in bf16, and
where no gate reaches 0 a central difference of the (then bilinear) h is its derivative.  What is left is the rounding of the gradient
itself, 2^-8 of it, and the tests assert that half of a term, let alone a whole one, is more than that."""
import math

import pytest
import torch

from oracle import product_oracle as o

pytestmark = pytest.mark.gpu
BF16 = 2.0 ** -8


@pytest.fixture(scope="module")
def ctx():
    import __graft_entry__ as entry
    entry.build()
    from paper_2506_00486_b200 import Context
    c = Context(0, guard=True)
    yield c
    c.check_guards()
    c.close()


class Integers:
    """A block of integers and a dh that is 0 where a step of at most 2 in gate or up could reach a kink or 16."""

    def __init__(self, ctx, seed, rows, width, hidden):
        gen = torch.Generator(device="cuda").manual_seed(seed)

        def ints(least, most, *shape):
            return torch.randint(least, most + 1, shape, generator=gen, device="cuda").double()

        self.ctx, self.x = ctx, ints(-2, 2, rows, width)
        self.wg, self.wu = (ints(-1, 1, hidden, width) * (torch.rand((hidden, width), generator=gen, device="cuda") < 12 / width) for _ in range(2))
        gate, up = self.x @ self.wg.t(), self.x @ self.wu.t()
        self.dh = torch.where((gate.abs() >= 3) & (gate.abs() <= 13) & (up.abs() <= 13), ints(-2, 2, rows, hidden), 0.0)
        self.gate, self.up = gate, up

    def h(self, **changed):
        x, wg, wu = (changed.get(n, getattr(self, n)).bfloat16() for n in ("x", "wg", "wu"))
        return self.ctx.gg_gated_linear(x, wg, wu, act="relu")["h"].double()

    def gradient(self):
        f = self.ctx.gg_gated_linear(self.x.bfloat16(), self.wg.bfloat16(), self.wu.bfloat16(), act="relu", keep=True)
        grad = self.ctx.gg_gated_linear_grad(self.dh.bfloat16(), self.x.bfloat16(), self.wg.bfloat16(), self.wu.bfloat16(), f["gate"], f["up"], act="relu")
        return {k: t.double() for k, t in grad.items()}

    def difference(self, name, column, by_row):
        """The derivative of sum(dh h) by column `column` of x (for each row) or of a weight (for each of its rows)."""
        step = torch.zeros_like(getattr(self, name))
        step[:, column] = 1.0
        up, down = (self.h(**{name: getattr(self, name) + s * step}) for s in (1, -1))
        return ((up - down) / 2 * self.dh).sum(1 if by_row else 0)


@pytest.mark.parametrize("rows,width,hidden", [(30, 24, 90), (200, 40, 130), (300, 33, 260)])
def test_the_gated_block_against_exact_differences(ctx, rows, width, hidden):
    b = Integers(ctx, rows, rows, width, hidden)
    assert (b.dh != 0).double().mean() > 0.2
    got = b.gradient()
    for name, of, by_row in (("dx", "x", True), ("dw_gate", "wg", False), ("dw_up", "wu", False)):
        want = torch.stack([b.difference(of, j, by_row) for j in range(width)], 1)
        assert ((got[name] - want).abs() <= BF16 * want.abs()).all(), name
    # the bound tells the terms apart: in most rows of dx half of either is more than it allows
    value, slope = b.gate.clamp_min(0.0), (b.gate > 0).double()
    terms = (b.dh * b.up * slope) @ b.wg, (b.dh * value) @ b.wu
    want = terms[0] + terms[1]
    assert ((got["dx"] - want).abs() <= BF16 * want.abs()).all()
    for wrong in (terms[0], terms[1], want - terms[0] / 2, want - terms[1] / 2, 1.5 * want, 0.5 * want):
        assert ((wrong - want).abs() > BF16 * want.abs()).any(1).double().mean() > 0.9


def norm64(x, w, b, eps=1e-5):
    xc = x - x.mean(-1, keepdim=True)
    return w * xc / (xc.square().mean(-1, keepdim=True) + eps).sqrt() + b


@pytest.mark.parametrize("width,hidden,vocab,rows", [(64, 96, 300, 130), (72, 200, 1001, 300), (128, 400, 2000, 1000)])
def test_the_decoder_with_independent_roundings(ctx, width, hidden, vocab, rows):
    # Between the parameters and a gradient lie 28 roundings to bf16 at most: forward norm, gate, up, h, the projection and the sum with the residual for each
    # of two blocks, the last norm; back d, dh, the norm's dx, dgate, dup, dx, dh of the projection, dropout (twice), the gradient itself.  One is off by
    # up to 2^-8 of its number, evenly spread (over sqrt(3) in the 2-norm), and thousands of them are independent, so that the errors add in
    # squares; the norms, gates and the softmax here enlarge none of them by more than 2.
    from paper_2506_00486_b200.train_example import Decoder
    bound = 2.0 * math.sqrt(28.0 / 3.0) * BF16
    model = Decoder(ctx, 2, width, hidden, vocab, 2.0, 0.2, 5)
    for p in model.parameters:
        p.requires_grad_(True)
    gen = torch.Generator(device="cuda").manual_seed(width)
    tokens = torch.randint(0, vocab, (rows,), generator=gen, device="cuda")
    target = torch.where(torch.rand(rows, generator=gen, device="cuda") < 0.2, -100, torch.randint(0, vocab, (rows,), generator=gen, device="cuda"))
    n = (target >= 0).sum()
    got = torch.autograd.grad(model(tokens, target, 3).sum() / n, model.parameters)

    def gradients(change=None):
        params = [p.detach().double().requires_grad_(True) for p in model.parameters]
        k = len(model.matrices)
        mats, vecs = params[:k], params[k:]
        x = mats[-2][tokens]
        for i in range(2):
            wg, wu, wd = mats[3 * i:3 * i + 3]
            y = norm64(x, *vecs[2 * i:2 * i + 2])
            a, u = y @ wg.t(), y @ wu.t()
            if change == "a gate without its slope":
                a = a.detach()
            if change == "an up that is constant":
                u = u.detach()
            kept = torch.from_numpy(o.dropout_bits(rows, width, 3, i, 5) >= 13107).cuda()       # 0.2 * 65536, rounded
            scale = 1.0 if change == "dropout unscaled" else 1.0 / (1.0 - 13107 / 65536)
            x = x + (a * torch.sigmoid(a) * u) @ wd.t() * kept * scale
        logits = norm64(x, *vecs[-2:]) @ mats[-1].t()
        loss = torch.nn.functional.cross_entropy(logits, target, reduction="sum") / n
        return torch.autograd.grad(loss, params, allow_unused=True)

    def worst(want):
        return max(((g.double() - w).norm() / w.norm()).item() if w is not None else 1.0 for g, w in zip(got, want))

    assert worst(gradients()) <= bound
    for change in ("a gate without its slope", "an up that is constant", "dropout unscaled"):
        assert worst(gradients(change)) > bound, change       # (each of these mistakes is more than the bound allows)
