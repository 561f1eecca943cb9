"""The operators of a decoder's training step together: the example runs, repeats itself, and its gradients are those of the same
model in 64 bits; the autograd forms on strided inputs, for single gradients and in a captured step."""
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
    c = Context(0)
    yield c
    c.close()


@pytest.mark.parametrize("bits", [32, 8])
def test_the_example_runs_and_repeats_itself(ctx, bits):
    from paper_2506_00486_b200.train_example import train_tokens
    (a, scales, beta), (b, _, _) = (train_tokens(ctx, bits=bits, steps=4) for _ in range(2))
    assert torch.isfinite(a).all() and torch.isfinite(scales).all() and torch.isfinite(beta).all()
    assert torch.equal(a, b)


def norm64(x, w, b, eps=1e-5):
    xc = x - x.mean(-1, keepdim=True)
    return w * xc / (xc.square().mean(-1, keepdim=True) + eps).sqrt() + b


@pytest.mark.parametrize("width,hidden,vocab,rows", [(64, 96, 300, 130), (72, 200, 1001, 300)])
def test_gradients_of_the_whole_model(ctx, width, hidden, vocab, rows):
    # Roundings to bf16 between the parameters and a gradient, each half a unit (2^-8) of the tensor at most: forward norm, gate, up, h, the
    # projection, the sum with the residual (twice for two blocks), the last norm; back d, dh, the norm's dx, dgate, dup, dx, dh of the projection, dropout
    # (twice), the gradient itself: 28.  They are independent, so that their sum in the 2-norm is about sqrt(28) / sqrt(3) half units; all of
    # them at their largest and passed on undiminished are 28 half units, and the norms here enlarge none of them by more than 2.
    from paper_2506_00486_b200.train_example import Decoder
    model = Decoder(ctx, 2, width, hidden, vocab, 2.0, 0.2, 5)
    for p in model.parameters:
        p.requires_grad_(True)
    gen = torch.Generator(device="cuda").manual_seed(width)
    tokens = torch.randint(0, vocab, (rows,), generator=gen, device="cuda")
    target = torch.where(torch.rand(rows, generator=gen, device="cuda") < 0.2, -100, torch.randint(0, vocab, (rows,), generator=gen, device="cuda"))
    n = (target >= 0).sum()
    loss = model(tokens, target, 3)
    got = torch.autograd.grad(loss.sum() / n, model.parameters)
    params = [p.detach().double().requires_grad_(True) for p in model.parameters]
    k = len(model.matrices)
    mats, vecs = params[:k], params[k:]
    x = mats[-2][tokens]
    for i in range(2):
        wg, wu, wd = mats[3 * i:3 * i + 3]
        y = norm64(x, *vecs[2 * i:2 * i + 2])
        a = y @ wg.t()
        kept = torch.from_numpy(o.dropout_bits(rows, width, 3, i, 5) >= 13107).cuda()       # 0.2 * 65536, rounded
        x = x + (a * torch.sigmoid(a) * (y @ wu.t())) @ wd.t() * kept / (1.0 - 13107 / 65536)
    logits = norm64(x, *vecs[-2:]) @ mats[-1].t()
    want_loss = torch.nn.functional.cross_entropy(logits, target, reduction="none")
    want = torch.autograd.grad(want_loss.sum() / n, params)
    assert ((loss == 0) == (target < 0)).all() or (loss[target < 0] == 0).all()
    assert (loss.double() - want_loss).norm() <= 56 * BF16 * want_loss.norm()
    for g, w, p in zip(got, want, model.parameters):
        assert g.shape == p.shape and (g.double() - w).norm() <= 56 * BF16 * w.norm()


def test_autograd_forms_on_strided_and_batched_inputs(ctx):
    from paper_2506_00486_b200.train_example import CrossEntropy, Dropout, GatedLinear
    gen = torch.Generator(device="cuda").manual_seed(7)

    def rand(*shape, scale=1.0):
        return (torch.randn(shape, generator=gen, device="cuda") * scale).bfloat16()

    base, both, out = rand(4, 40, 2, 48), rand(2, 96, 48, scale=0.2), rand(48, 500, scale=0.2)
    x, w_gate, w_up, w_out = base[:, :, 1], both[0], both[1], out.t()
    leaves = [t.detach().requires_grad_(True) for t in (x, w_gate, w_up, w_out)]
    target = torch.randint(0, 500, (40, 4), generator=gen, device="cuda").t()
    h = GatedLinear.apply(leaves[0], leaves[1], leaves[2], ctx, "gelu")
    assert h.shape == (4, 40, 96)
    y = Dropout.apply(h[..., ::2], leaves[0], 0.3, ctx, 1, 2, 3)
    loss = CrossEntropy.apply(y, leaves[3], target, ctx)
    assert loss.shape == (4, 40) and loss.dtype == torch.float32
    weight = torch.rand((40, 4), generator=gen, device="cuda").t()
    got = torch.autograd.grad(loss, leaves, weight)
    d = [t.detach().double().requires_grad_(True) for t in leaves]
    h = torch.nn.functional.gelu(d[0] @ d[1].t()) * (d[0] @ d[2].t())
    kept = torch.from_numpy(o.dropout_bits(160, 48, 2, 3, 1) >= 19661).cuda().view(4, 40, 48)
    y = h[..., ::2] * kept / (1.0 - 19661 / 65536) + d[0]
    want = torch.autograd.grad((torch.nn.functional.cross_entropy((y @ d[3].t()).view(-1, 500), target.reshape(-1), reduction="none").view(4, 40) * weight).sum(), d)
    # (nine roundings on the longest way, as above)
    for g, w in zip(got, want):
        assert (g.double() - w).norm() <= 18 * BF16 * w.norm()


def test_only_the_gradients_that_are_asked_for(ctx):
    from paper_2506_00486_b200.train_example import CrossEntropy, Dropout, GatedLinear
    x, w, v = (torch.randn(s, device="cuda").bfloat16() for s in ((8, 16), (24, 16), (24, 16)))
    for which in range(3):
        t = [u.clone().requires_grad_(i == which) for i, u in enumerate((x, w, v))]
        GatedLinear.apply(*t, ctx).sum().backward()
        assert [u.grad is not None for u in t] == [i == which for i in range(3)]
    target = torch.zeros(8, dtype=torch.int64, device="cuda")
    for which in range(2):
        t = [u.clone().requires_grad_(i == which) for i, u in enumerate((x, w))]
        CrossEntropy.apply(*t, target, ctx).sum().backward()
        assert [u.grad is not None for u in t] == [i == which for i in range(2)]
        t = [u.clone().requires_grad_(i == which) for i, u in enumerate((x, x))]
        Dropout.apply(*t, 0.5, ctx, 0, 1, 0).sum().backward()
        assert [u.grad is not None for u in t] == [i == which for i in range(2)]
    y = Dropout.apply(x, None, 0.5, ctx, 0, 1, 0)
    assert not y.requires_grad
    with torch.no_grad():
        q = w.clone().requires_grad_(True)
        assert not GatedLinear.apply(x, q, v, ctx).requires_grad and not CrossEntropy.apply(x, q, target, ctx).requires_grad


def test_a_second_derivative_is_refused(ctx):
    from paper_2506_00486_b200.train_example import GatedLinear
    x = torch.randn(4, 96, device="cuda").bfloat16().requires_grad_(True)
    w = torch.randn(8, 96, device="cuda").bfloat16()
    first, = torch.autograd.grad(GatedLinear.apply(x, w, w, ctx).float().square().sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        first.sum().backward()


def test_a_captured_step_draws_new_masks(ctx):
    # forward, backward and update of one block in a graph, the step counter on the device
    gen = torch.Generator(device="cuda").manual_seed(8)
    x, wg, wu, wo = ((torch.randn(s, generator=gen, device="cuda") * 0.2).bfloat16() for s in ((100, 64), (128, 64), (128, 64), (300, 128)))
    target = torch.randint(0, 300, (100,), generator=gen, device="cuda")
    t_dev = torch.zeros(1, dtype=torch.int64, device="cuda")
    dloss = torch.full((100,), 0.01, device="cuda")
    gated = ctx.make_gated_linear(x, wg, wu, keep=True)
    h = gated.outputs["h"]
    drop = ctx.make_dropout(h, 0.5, seed=9, tensor_id=1, t_dev=t_dev)
    loss = ctx.make_cross_entropy(drop.outputs["y"], wo, target)
    dloss_h = ctx.make_cross_entropy_grad(dloss, drop.outputs["y"], wo, target, loss.outputs["lse"])
    back = ctx.make_dropout(dloss_h.outputs["dh"], 0.5, seed=9, tensor_id=1, t_dev=t_dev)
    grad = ctx.make_gated_linear_grad(back.outputs["y"], x, wg, wu, gated.outputs["gate"], gated.outputs["up"])

    def step():
        gated()
        drop(5)
        loss()
        dloss_h()
        back(5)
        return grad()

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
        t_dev.add_(1)
    seen = []
    for i in range(3):
        graph.replay()
        torch.cuda.synchronize()
        seen.append({k: t.clone() for k, t in grad.outputs.items()})
        bits = torch.from_numpy(o.dropout_bits(100, 128, 5 + i, 1, 9)).cuda()
        assert torch.equal(drop.outputs["y"] == 0, (bits < 32768) | (h == 0))
    assert not torch.equal(seen[0]["dx"], seen[1]["dx"])
    t_dev.zero_()
    eager = step()
    assert all(torch.equal(eager[k], seen[0][k]) for k in eager)
