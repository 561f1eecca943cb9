"""The gradient of the vocabulary loss has no error that all positions share, wherever in the batch the first position with a target is.

d = weight (p - 1) at a position's target is nearly the weight itself, and mostly one number.  Rounded to bf16 it would be off by up to 2^-8
everywhere alike; relative to the weight it is p - 1 that is rounded."""
import pytest
import torch

from product_util import matrix

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    import __graft_entry__ as entry
    entry.build()
    from paper_2506_00486_b200 import Context
    c = Context(0)
    yield c
    c.close()


@pytest.mark.parametrize("first", [0, 255, 256, 257, 4095, 4096, 8447, 8448, 9000, 70000])
def test_no_shared_error(ctx, first):
    rows, width, vocab = first + 800, 64, 2000
    gen = torch.Generator(device="cuda").manual_seed(first)
    h, w = matrix(gen, rows, width), matrix(gen, vocab, width, scale=0.05)
    target = torch.randint(0, vocab, (rows,), generator=gen, device="cuda")
    target[:first] = -100
    # 1 + 0.55 / 128 lies 0.45 of a bf16 step, 0.35 %, below its neighbour
    dloss = torch.full((rows,), (1.0 + 0.55 / 128) / (1.0 - 1.0 / vocab), device="cuda")
    out = ctx.gg_cross_entropy(h, w, target)
    got = ctx.gg_cross_entropy_grad(dloss, h, w, target, out["lse"])
    there = torch.nonzero(target >= 0)[:, 0]
    p = torch.exp(h.double() @ w.double().t() - out["lse"].double()[:, None])[there]
    # p - 1 at the target is off by half a step of the numbers below 1 at most, 2^-9, and where p is below 2^-9 (most rows here) by p itself
    at = p[torch.arange(there.numel(), device="cuda"), target[there]]
    shared = torch.where(at <= 2.0 ** -9, at, 2.0 ** -9).mean().item()
    d = p.clone()
    d[torch.arange(there.numel(), device="cuda"), target[there]] -= 1.0
    d *= dloss[there].double()[:, None]
    for name, want, have in (("dh", d @ w.double(), got["dh"][there].double()), ("dw", d.t() @ h[there].double(), got["dw"].double())):
        off = (have * want).sum().item() / (want * want).sum().item() - 1.0
        # and the result's own rounding, 2^-9 for each of its numbers in either direction: 6 of the mean's standard deviations
        assert abs(off) <= 2 * shared + 6 * 2.0 ** -9 / want.numel() ** 0.5, (name, off)
