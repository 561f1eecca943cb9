"""The vocabulary loss and its gradient against the 64-bit form: every size around the tiles, strides, positions without a
target, targets twice and beyond the vocabulary, logits that are large, infinite or nan, graphs and streams, refusals.

Bounds: product_util's for sums; a logit l is off by dl = SUM(width) sum|h w|.  exp(l - x) in fp32: l - x is rounded once, scaled by log2 e
rounded twice, and exp2 is off by 2 units: relative 4 U (|l - x| + 1) + 4 U, and dl and the error of x add to it.  The sums of exponentials
are added 32 to a chain per tile and joined over tiles: 64 + tiles U covers both."""
import numpy as np
import pytest
import torch

from oracle import product_oracle as o
from product_util import BF16, SUM, U, around, host, matrix, near

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    import __graft_entry__ as entry
    entry.build()
    from paper_2506_00486_b200 import Context
    c = Context(0, guard=True)
    yield c
    c.check_guards()
    c.close()


def targets(gen, rows, vocab, ignored):
    t = torch.randint(0, vocab, (rows,), generator=gen, device="cuda")
    return torch.where(torch.rand(rows, generator=gen, device="cuda") < ignored, -100, t)


def problem(seed, rows, width, vocab, ignored=0.2, pad=0, shift=0, scale=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    h, w = matrix(gen, rows, width, pad, shift), matrix(gen, vocab, width, pad, shift, scale * 2.0 / width ** 0.5)
    dloss = torch.rand(rows, generator=gen, device="cuda") + 0.5
    return h, w, targets(gen, rows, vocab, ignored), dloss


def logit_error(h, w):
    return SUM(h.shape[1]) * (np.abs(host(h)) @ np.abs(host(w)).T)


def check_loss(h, w, target, out):
    loss, lse, logits = o.cross_entropy(host(h), host(w), target.tolist())
    dl, tiles = logit_error(h, w), w.shape[0] / 256 + 1
    span = np.abs(logits - lse[:, None])
    p = np.exp(logits - lse[:, None])
    rel = (p * (dl + 4 * U * (span + 2))).sum(axis=1) + (64 + tiles) * U          # of the sum of exponentials
    tol = rel + 4 * U * (np.abs(lse) + 1) + 4 * U * np.log(w.shape[0] + 1)
    near(out["lse"], lse, tol, "lse")
    at = np.array([logits[r, t] if 0 <= t < w.shape[0] else 0.0 for r, t in enumerate(target.tolist())])
    dat = np.array([dl[r, t] if 0 <= t < w.shape[0] else 0.0 for r, t in enumerate(target.tolist())])
    good = ~np.isnan(loss)
    assert np.array_equal(np.isnan(host(out["loss"])), ~good)
    near(host(out["loss"])[good], loss[good], (tol + dat + U * (np.abs(at) + np.abs(lse)) + U * np.abs(loss))[good], "loss")


def check_grad(dloss, h, w, target, lse, out, base=None):
    hd, wd, g = host(h), host(w), host(dloss)
    dh, dw, d = o.cross_entropy_grad(g, hd, wd, target.tolist(), host(lse))
    logits = hd @ wd.T
    p = np.where((target.cpu().numpy() >= 0)[:, None], np.abs(g)[:, None] * np.exp(logits - host(lse)[:, None]), 0.0)
    derr = p * (logit_error(h, w) + 4 * U * (np.abs(logits - host(lse)[:, None]) + 2)) + 4 * U * (p + np.abs(d))
    derr = derr + BF16 * (np.abs(d) + derr)
    if out["dh"] is not None:
        tol = derr @ np.abs(wd) + (SUM(w.shape[0]) + 64 * U) * (np.abs(d) @ np.abs(wd))
        near(out["dh"], dh, tol + BF16 * (np.abs(dh) + tol) + 1e-37, "dh")
    if out["dw"] is not None:
        tol = derr.T @ np.abs(hd) + SUM(h.shape[0]) * (np.abs(d).T @ np.abs(hd))
        want = dw if base is None else dw + base
        near(out["dw"], want, tol + 2 * U * np.abs(want) + BF16 * (np.abs(want) + tol) + 1e-37, "dw")


SHAPES = [(1, 1, 1), (1, 8, 7), (2, 3, 2), (3, 64, 256), (2, 100, 257), (1, 896, 5000), (33, 200, 1000), (128, 64, 256), (129, 65, 513), (256, 128, 512),
          (257, 72, 31), (5, 4096, 100), (700, 33, 2049), (64, 1000, 300), (1, 16, 70001), (2000, 24, 9)]


@pytest.mark.parametrize("rows,width,vocab", SHAPES)
def test_loss_and_gradient(ctx, rows, width, vocab):
    h, w, target, dloss = problem(rows * 31 + width, rows, width, vocab)
    out = ctx.gg_cross_entropy(h, w, target)
    check_loss(h, w, target, out)
    check_grad(dloss, h, w, target, out["lse"], ctx.gg_cross_entropy_grad(dloss, h, w, target, out["lse"]))


@pytest.mark.parametrize("pad,shift", [(8, 0), (16, 8), (1, 0), (0, 1), (3, 5), (0, 4)])
@pytest.mark.parametrize("rows,width,vocab", [(13, 96, 300), (130, 77, 520)])
def test_strides_and_alignment(ctx, rows, width, vocab, pad, shift):
    h, w, target, dloss = problem(pad + 7 * shift + rows, rows, width, vocab, pad=pad, shift=shift)
    gen = torch.Generator(device="cuda").manual_seed(9)
    dh, dw = matrix(gen, rows, width, pad, shift), matrix(gen, vocab, width, pad, shift)
    before = [around(t, shift) for t in (dh, dw)]
    out = ctx.gg_cross_entropy(h, w, target)
    check_loss(h, w, target, out)
    check_grad(dloss, h, w, target, out["lse"], ctx.gg_cross_entropy_grad(dloss, h, w, target, out["lse"], dh=dh, dw=dw))
    for t, b in zip((dh, dw), before):
        assert torch.equal(around(t, shift), b)


@pytest.mark.parametrize("ignored", [0.0, 1.0])
def test_all_and_no_positions_have_a_target(ctx, ignored):
    h, w, target, dloss = problem(5, 200, 48, 300, ignored=ignored)
    out = ctx.gg_cross_entropy(h, w, target)
    check_loss(h, w, target, out)
    grad = ctx.gg_cross_entropy_grad(dloss, h, w, target, out["lse"])
    check_grad(dloss, h, w, target, out["lse"], grad)
    if ignored == 1.0:
        assert not out["loss"].any() and not grad["dh"].any() and not grad["dw"].any()


def test_the_same_target_many_times(ctx):
    h, w, _, dloss = problem(6, 300, 64, 700)
    target = torch.full((300,), 699, device="cuda")
    out = ctx.gg_cross_entropy(h, w, target)
    check_loss(h, w, target, out)
    check_grad(dloss, h, w, target, out["lse"], ctx.gg_cross_entropy_grad(dloss, h, w, target, out["lse"]))


@pytest.mark.parametrize("beyond", [300, 511, 512, 2 ** 40])
def test_a_target_beyond_the_vocabulary_is_nan_in_its_row(ctx, beyond):
    h, w, target, dloss = problem(7, 40, 32, 300, ignored=0.0)
    target[11] = beyond
    out = ctx.gg_cross_entropy(h, w, target)
    check_loss(h, w, target, out)
    grad = ctx.gg_cross_entropy_grad(dloss, h, w, target, out["lse"])
    nan = torch.isnan(grad["dh"]).all(1)
    assert nan[11] and nan.sum() == 1 and torch.isnan(grad["dw"]).all()
    keep = torch.arange(40, device="cuda") != 11
    again = ctx.gg_cross_entropy_grad(dloss[keep], h[keep], w, target[keep], out["lse"][keep], want_dw=False)
    assert torch.equal(again["dh"], grad["dh"][keep])


@pytest.mark.parametrize("scale", [30.0, 300.0])
def test_large_logits(ctx, scale):
    # the largest probability of a row is 1 to all bits; differences of hundreds underflow
    h, w, target, dloss = problem(8, 65, 64, 500, scale=scale)
    out = ctx.gg_cross_entropy(h, w, target)
    check_loss(h, w, target, out)
    check_grad(dloss, h, w, target, out["lse"], ctx.gg_cross_entropy_grad(dloss, h, w, target, out["lse"]))


@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_what_is_not_finite_stays_in_its_row(ctx, bad):
    h, w, target, dloss = problem(9, 70, 40, 400, ignored=0.3)
    clean = ctx.gg_cross_entropy(h, w, target)
    rows = torch.zeros(70, dtype=torch.bool, device="cuda")
    rows[[3, 68]] = True
    target[3], target[68] = 5, -100
    h[rows, 7] = bad
    out = ctx.gg_cross_entropy(h, w, target)
    assert not torch.isfinite(out["lse"][rows]).any() and not torch.isfinite(out["loss"][3]) and out["loss"][68] == 0.0
    assert torch.equal(out["lse"][~rows], clean["lse"][~rows]) and torch.equal(out["loss"][~rows], clean["loss"][~rows])
    dh = ctx.gg_cross_entropy_grad(dloss, h, w, target, out["lse"], want_dw=False)["dh"]
    assert torch.isnan(dh[3]).all() and not dh[68].any()              # (a position without a target has no gradient, whatever it holds)
    h[rows] = 0.0
    want = ctx.gg_cross_entropy_grad(dloss, h, w, target, out["lse"], want_dw=False)["dh"]
    assert torch.equal(dh[~rows], want[~rows])


def test_logits_of_minus_infinity(ctx):
    # tokens that a mask rules out: -inf times a positive feature
    h, w, target, dloss = problem(10, 20, 16, 600, ignored=0.0)
    h[:, 0] = 1.0
    w[100:400, 0] = -float("inf")
    target[:] = torch.randint(0, 100, (20,), device="cuda")
    out = ctx.gg_cross_entropy(h, w, target)
    left = torch.cat((w[:100], w[400:]))
    ref = ctx.gg_cross_entropy(h, left, target)
    assert torch.allclose(out["lse"], ref["lse"], rtol=1e-5) and torch.allclose(out["loss"], ref["loss"], rtol=1e-5, atol=1e-5)
    dw = ctx.gg_cross_entropy_grad(dloss, h, w, target, out["lse"], want_dh=False)["dw"]
    assert not dw[100:400].any() and torch.isfinite(dw).all()


def test_weights_of_the_loss(ctx):
    h, w, target, dloss = problem(11, 50, 24, 300, ignored=0.0)
    dloss[::3] = 0.0
    dloss[1::3] *= -1e-6
    dloss[2::3] *= 1e6
    lse = ctx.gg_cross_entropy(h, w, target)["lse"]
    check_grad(dloss, h, w, target, lse, ctx.gg_cross_entropy_grad(dloss, h, w, target, lse))


@pytest.mark.parametrize("first", [1, 40, 255, 300, 4097, 5000])
def test_a_batch_that_begins_without_targets(ctx, first):
    # whichever weight the gradient is kept relative to, or none
    h, w, target, dloss = problem(18, 5300, 24, 100, ignored=0.0)
    target[:first] = -100
    dloss[first:first + 20] = 0.0
    dloss[first + 20:first + 25] = torch.tensor([1e-35, float(torch.finfo(torch.float32).tiny), 1e-20, 3e4, -7.0], device="cuda")
    lse = ctx.gg_cross_entropy(h, w, target)["lse"]
    check_grad(dloss, h, w, target, lse, ctx.gg_cross_entropy_grad(dloss, h, w, target, lse))


def test_one_gradient_at_a_time_accumulation_and_repeatability(ctx):
    h, w, target, dloss = problem(12, 333, 120, 1111)
    lse = ctx.gg_cross_entropy(h, w, target)["lse"]
    both = ctx.gg_cross_entropy_grad(dloss, h, w, target, lse)
    dh = ctx.gg_cross_entropy_grad(dloss, h, w, target, lse, want_dw=False)
    dw = ctx.gg_cross_entropy_grad(dloss, h, w, target, lse, want_dh=False)
    assert dh["dw"] is None and dw["dh"] is None and torch.equal(dh["dh"], both["dh"]) and torch.equal(dw["dw"], both["dw"])
    base = matrix(torch.Generator(device="cuda").manual_seed(1), 1111, 120, scale=0.1)
    sums = base.clone()
    out = ctx.gg_cross_entropy_grad(dloss, h, w, target, lse, dw=sums, accumulate=True)
    check_grad(dloss, h, w, target, lse, out, base=host(base))
    assert torch.equal(out["dh"], both["dh"])
    assert ctx.gg_cross_entropy_grad(dloss, h, w, target, lse, want_dh=False, want_dw=False) == dict(dh=None, dw=None)


def test_no_positions(ctx):
    h, w, target, dloss = problem(13, 0, 16, 20)
    out = ctx.gg_cross_entropy(h, w, target)
    assert out["loss"].numel() == 0
    base = torch.ones(20, 16, dtype=torch.bfloat16, device="cuda")
    ctx.gg_cross_entropy_grad(dloss, h, w, target, out["lse"], dw=base, accumulate=True)
    assert (base == 1).all()
    assert not ctx.gg_cross_entropy_grad(dloss, h, w, target, out["lse"])["dw"].any()


def test_gradient_against_differences_of_the_forward_pass(ctx):
    # along a direction in h that is exact in bf16: h +- e s with all three on one grid
    h, w, target, dloss = problem(14, 24, 32, 200, ignored=0.1)
    gen = torch.Generator(device="cuda").manual_seed(2)
    h.copy_((h.float().clamp(-2, 2) * 16).round() / 16)
    sign = torch.where(torch.rand(h.shape, generator=gen, device="cuda") < 0.5, -1.0, 1.0)
    e = 1 / 16
    lse = ctx.gg_cross_entropy(h, w, target)["lse"]
    dh = ctx.gg_cross_entropy_grad(dloss, h, w, target, lse, want_dw=False)["dh"]
    losses = [(ctx.gg_cross_entropy((h.float() + f * e * sign).bfloat16(), w, target)["loss"].double() * dloss).sum().item() for f in (1, -1, 2, -2)]
    # fourth-order difference: the error is e^4 f'''''/ 30; with directions of length |W s| ~ 11 and derivatives of the log-sum-exp bounded by
    # that length to the fifth power times 24, e |W s| ~ 0.7 leaves a few percent of a row's slope
    diff = (8 * (losses[0] - losses[1]) - (losses[2] - losses[3])) / (12 * e)
    want = (dh.double() * sign).sum().item()
    assert abs(diff - want) <= 0.05 * (dh.double() * sign).sum(1).abs().sum().item()


def test_on_another_stream_and_in_a_graph(ctx):
    from paper_2506_00486_b200 import Context
    mine = Context(0)                 # (its scratch is first needed inside the capture)
    h, w, target, dloss = problem(15, 200, 136, 900)
    want = ctx.gg_cross_entropy(h, w, target)
    wantg = ctx.gg_cross_entropy_grad(dloss, h, w, target, want["lse"])
    loss = mine.make_cross_entropy(h, w, target)
    grad = mine.make_cross_entropy_grad(dloss, h, w, target, loss.outputs["lse"])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss()
        grad()
    for t in (*loss.outputs.values(), *grad.outputs.values()):
        t.zero_()
    # a larger call outgrows the scratch that the graph holds
    big = problem(16, 1500, 136, 3000)
    mine.gg_cross_entropy_grad(big[3], big[0], big[1], big[2], mine.gg_cross_entropy(*big[:3])["lse"])
    other = [torch.full((1 << 20,), 3.0, device="cuda") for _ in range(16)]
    graph.replay()
    torch.cuda.synchronize()
    assert all((t == 3.0).all() for t in other)
    assert torch.equal(loss.outputs["loss"], want["loss"]) and torch.equal(grad.outputs["dh"], wantg["dh"]) and torch.equal(grad.outputs["dw"], wantg["dw"])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = mine.gg_cross_entropy(h, w, target)
    side.synchronize()
    assert torch.equal(again["lse"], want["lse"])
    del graph
    mine.close()


def test_refusals(ctx):
    from paper_2506_00486_b200 import GGError
    h, w, target, dloss = problem(17, 8, 16, 20)
    lse = torch.zeros(8, device="cuda")
    before = ctx.launch_count
    for bad in ((h.float(), w, target), (h, w.float(), target), (h.half(), w, target)):
        with pytest.raises(TypeError):
            ctx.gg_cross_entropy(*bad)
    for bad in ((h[:, :8], w, target), (h, w, target[:5]), (h, w, target.int()), (h.t(), w, target), (h, w.cpu(), target), (h[0], w, target)):
        with pytest.raises(ValueError):
            ctx.gg_cross_entropy(*bad)
    for kw in (dict(dh=h[:4]), dict(dw=w.float()), dict(accumulate=True)):
        with pytest.raises(ValueError):
            ctx.gg_cross_entropy_grad(dloss, h, w, target, lse, **kw)
    for bad in (dloss[:3], dloss.double()):
        with pytest.raises(ValueError):
            ctx.gg_cross_entropy_grad(bad, h, w, target, lse)
    for kw in (dict(dh=h), dict(dw=w)):           # the logits are computed again from both
        with pytest.raises(GGError) as e:
            ctx.gg_cross_entropy_grad(dloss, h, w, target, lse, **kw)
        assert e.value.status == 1
    with pytest.raises(GGError) as e:
        ctx.gg_cross_entropy(h, w[:0], target)
    assert e.value.status == 1
    run = ctx.make_cross_entropy(h, w, target)
    for field, value, status in (("dtype", 0, 2), ("h_ld", 3, 1), ("target", None, 1), ("w", None, 1), ("rows", -1, 1), ("rows", 1 << 31, 1), ("width", 0, 1),
                                 ("h", h.data_ptr() + 1, 3), ("target", target.data_ptr() + 4, 3), ("loss", lse.data_ptr() + 2, 3)):
        keep = getattr(run.args, field)
        setattr(run.args, field, value)
        with pytest.raises(GGError) as e:
            run()
        assert e.value.status == status, field
        setattr(run.args, field, keep)
    assert ctx.launch_count == before


@pytest.mark.parametrize("width", [1, 64, 512, 513, 520, 1025])
@pytest.mark.parametrize("shape", ["up", "down", "peak", "holes"])
def test_logits_that_grow_along_the_vocabulary(ctx, width, shape):
    # The largest logit moves through a tile's columns, and whole runs of columns are -infinity.  A sum is rescaled up to eight times on its
    # way through a tile: each is an exponential, relative 4 U (step + 2), and the steps together are no more than the span.
    vocab, rows = 700, 150
    gen = torch.Generator(device="cuda").manual_seed(width)
    l = torch.arange(vocab, device="cuda") / 16
    l = {"up": l, "down": l.flip(0), "peak": (l - l[300]).abs().neg(), "holes": l.clone()}[shape].bfloat16()
    if shape == "holes":
        l[:96] = l[160:230] = l[512:] = -float("inf")
    h, w = torch.zeros(rows, width, device="cuda").bfloat16(), torch.randn(vocab, width, generator=gen, device="cuda").bfloat16()
    h[:, width // 2], w[:, width // 2] = 1.0, l
    target = torch.randint(96, 160, (rows,), generator=gen, device="cuda")
    target[::7] = -1
    out = ctx.gg_cross_entropy(h, w, target)
    x = host(l)
    top = x.max()
    lse = top + np.log(np.exp(x - top).sum())
    p = np.exp(x - lse)
    span = np.where(np.isinf(x), 0.0, np.abs(np.where(np.isinf(x), lse, x) - lse))
    rel = (p * (8 * U * (span + 2) + 64 * U)).sum() + (64 + vocab / 256 + 1) * U
    tol = rel + 4 * U * (abs(lse) + 1) + 4 * U * np.log(vocab + 1)
    near(out["lse"], np.full(rows, lse), tol, "lse")
    t = target.tolist()
    want = np.array([0.0 if i < 0 else lse - x[i] for i in t])
    near(out["loss"], want, tol + U * (abs(lse) + 2 * np.abs(x[np.maximum(t, 0)])), "loss")
