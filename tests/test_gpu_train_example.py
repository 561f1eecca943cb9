"""The pieces of a training step together: the example's run learns, with 32-bit and with 8-bit states alike."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    import __graft_entry__ as entry
    entry.build()
    from paper_2506_00486_b200 import Context
    c = Context(0)
    yield c
    c.close()


def test_the_example_learns_and_8_bits_follow_32(ctx):
    from paper_2506_00486_b200.train_example import train
    last = {}
    for bits in (32, 8):
        losses, scales, beta = train(ctx, bits=bits, steps=150)
        assert torch.isfinite(losses).all() and torch.isfinite(scales).all()
        assert ((scales > 0) & (scales <= 1)).all() and ((beta > 0.05) & (beta < 20)).all()
        last[bits] = losses[-20:].mean().item()
        assert last[bits] < 0.5 * losses[:5].mean().item()
    assert last[8] < 1.25 * last[32]


def test_the_run_repeats_itself(ctx):
    from paper_2506_00486_b200.train_example import train
    a, b = (train(ctx, bits=8, steps=3)[0] for _ in range(2))
    assert torch.equal(a, b)


def test_layer_norm_for_autograd_matches_torch(ctx):
    from paper_2506_00486_b200.train_example import LayerNorm
    gen = torch.Generator(device="cuda").manual_seed(0)
    x, w, b, dy = (torch.randn(s, generator=gen, device="cuda") for s in ((4, 33, 384), (384,), (384,), (4, 33, 384)))
    for t in (x, w, b):
        t.requires_grad_(True)
    LayerNorm.apply(x, w, b, ctx).backward(dy)
    got = [t.grad.clone() for t in (x, w, b)]
    x64, w64, b64 = (t.detach().double().requires_grad_(True) for t in (x, w, b))
    xc = x64 - x64.mean(-1, keepdim=True)
    (w64 * xc / (xc.square().mean(-1, keepdim=True) + 1e-5).sqrt() + b64).backward(dy.double())
    for g, t in zip(got, (x64, w64, b64)):
        assert torch.allclose(g.double(), t.grad, rtol=1e-4, atol=1e-4)
