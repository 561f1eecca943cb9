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


def norm64(x, w, b, eps=1e-5):
    xc = x - x.mean(-1, keepdim=True)
    y = xc / (xc.square().mean(-1, keepdim=True) + eps).sqrt()
    y = y if w is None else y * w
    return y if b is None else y + b


def test_the_gradient_of_layer_norm_is_not_differentiable_again(ctx):
    # it is computed outside autograd: a second derivative through it would take it for a constant
    from paper_2506_00486_b200.train_example import LayerNorm
    x = torch.randn(4, 96, device="cuda", requires_grad=True)
    w, b = torch.ones(96, device="cuda"), torch.zeros(96, device="cuda")
    first, = torch.autograd.grad(LayerNorm.apply(x, w, b, ctx).square().sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        (first * torch.randn_like(first)).sum().backward()


@pytest.mark.parametrize("layout", ["columns", "rows", "overlapping", "one dimension"])
def test_layer_norm_of_strided_inputs(ctx, layout):
    from paper_2506_00486_b200.train_example import LayerNorm
    gen = torch.Generator(device="cuda").manual_seed(1)
    base = torch.randn((60, 2, 48), generator=gen, device="cuda")
    x = {"columns": base[:, 0].t(), "rows": base[:, 1], "overlapping": base[:1, 0].expand(5, 48), "one dimension": base[0, 0]}[layout].detach().requires_grad_(True)
    w = torch.randn(x.shape[-1], generator=gen, device="cuda", requires_grad=True)
    b = torch.randn(x.shape[-1], generator=gen, device="cuda", requires_grad=True)
    dy = torch.randn(x.shape, generator=gen, device="cuda")
    y = LayerNorm.apply(x, w, b, ctx)
    x64, w64, b64 = (t.detach().double().requires_grad_(True) for t in (x, w, b))
    y64 = norm64(x64, w64, b64)
    assert y.shape == x.shape and torch.allclose(y.double(), y64, rtol=1e-5, atol=1e-5)
    for g, want in zip(torch.autograd.grad(y, (x, w, b), dy), torch.autograd.grad(y64, (x64, w64, b64), dy.double())):
        assert torch.allclose(g.double(), want, rtol=1e-4, atol=1e-4)


@pytest.mark.parametrize("given", ["neither", "weight", "bias"])
@pytest.mark.parametrize("eps", [1e-5, 0.5])
def test_layer_norm_with_eps_and_without_weight_or_bias(ctx, given, eps):
    from paper_2506_00486_b200.train_example import LayerNorm
    gen = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn((7, 100), generator=gen, device="cuda", requires_grad=True)
    v = torch.randn(100, generator=gen, device="cuda", requires_grad=True)
    w, b = v if given == "weight" else None, v if given == "bias" else None
    dy = torch.randn(x.shape, generator=gen, device="cuda")
    y = LayerNorm.apply(x, w, b, ctx, eps)
    x64, v64 = x.detach().double().requires_grad_(True), v.detach().double().requires_grad_(True)
    y64 = norm64(x64, v64 if w is not None else None, v64 if b is not None else None, eps)
    assert torch.allclose(y.double(), y64, rtol=1e-5, atol=1e-5)
    of, of64 = ((x,), (x64,)) if given == "neither" else ((x, v), (x64, v64))
    for g, want in zip(torch.autograd.grad(y, of, dy), torch.autograd.grad(y64, of64, dy.double())):
        assert torch.allclose(g.double(), want, rtol=1e-4, atol=1e-4)


def test_layer_norm_computes_only_the_gradients_that_are_asked_for(ctx):
    from paper_2506_00486_b200.train_example import LayerNorm
    x, w, b = torch.randn(4, 64, device="cuda"), torch.ones(64, device="cuda"), torch.zeros(64, device="cuda")
    for which in range(3):
        t = [v.clone().requires_grad_(i == which) for i, v in enumerate((x, w, b))]
        LayerNorm.apply(*t, ctx).sum().backward()
        assert [v.grad is not None for v in t] == [i == which for i in range(3)]
