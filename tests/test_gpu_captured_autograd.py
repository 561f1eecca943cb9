"""A decoder block's forward and backward pass through the autograd forms in one graph: each replay is the eager pass of its step."""
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


def tensors(seed=1):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x, wg, wu, wd, wo = ((torch.randn(s, generator=gen, device="cuda") * k).bfloat16() for s, k in (((100, 64), 1.0), ((96, 64), 0.2), ((96, 64), 0.2), ((64, 96), 0.2), ((300, 64), 0.2)))
    weight, bias = torch.ones(64, device="cuda").bfloat16(), torch.zeros(64, device="cuda").bfloat16()
    target = torch.randint(-30, 300, (100,), generator=gen, device="cuda")
    return [x, weight, bias, wg, wu, wd, wo], target


def step(ctx, leaves, target, t):
    """(losses, gradients) of a block in step t; the leaves are made here, so that no other graph of them lives."""
    from paper_2506_00486_b200.train_example import CrossEntropy, Dropout, GatedLinear, LayerNorm
    x, weight, bias, wg, wu, wd, wo = leaves = [v.detach().requires_grad_(True) for v in leaves]
    h = GatedLinear.apply(LayerNorm.apply(x, weight, bias, ctx), wg, wu, ctx)
    loss = CrossEntropy.apply(Dropout.apply(h @ wd.t(), x, 0.4, ctx, 7, t, 2), wo, target, ctx)
    return loss.detach(), torch.autograd.grad(loss.sum(), leaves)


def test_replays_draw_the_masks_of_their_steps(ctx):
    leaves, target = tensors()
    t_dev = torch.full((1,), 5, dtype=torch.int64, device="cuda")
    want = [step(ctx, leaves, target, 5 + i) for i in range(3)]
    eager = step(ctx, leaves, target, t_dev)
    assert torch.equal(eager[0], want[0][0]) and all(torch.equal(a, b) for a, b in zip(eager[1], want[0][1]))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss, grads = step(ctx, leaves, target, t_dev)
        t_dev.add_(1)
    for w_loss, w_grads in want:
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(loss, w_loss) and all(torch.equal(a, b) for a, b in zip(grads, w_grads))
    assert t_dev.item() == 8 and not torch.equal(want[0][0], want[1][0])
    del graph


def test_a_step_that_is_advanced_before_the_backward_pass_is_refused(ctx):
    from paper_2506_00486_b200.train_example import Dropout
    x = torch.randn(10, 32, device="cuda").bfloat16().requires_grad_(True)
    t_dev = torch.ones(1, dtype=torch.int64, device="cuda")
    y = Dropout.apply(x, None, 0.5, ctx, 1, t_dev, 0)
    t_dev.add_(1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()


def test_a_step_counter_that_is_none_is_refused(ctx):
    from paper_2506_00486_b200.train_example import Dropout
    x = torch.randn(10, 32, device="cuda").bfloat16()
    for bad in (torch.ones(2, dtype=torch.int64, device="cuda"), torch.ones(1, device="cuda"), torch.ones(1, dtype=torch.int64)):
        with pytest.raises(ValueError, match="t_dev"):
            Dropout.apply(x, None, 0.5, ctx, 1, bad, 0)
