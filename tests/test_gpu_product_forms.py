"""The vocabulary loss, the gated block and their gradients in every form that the product kernel has, against 64 bits on the device.

Which form a call takes follows from its sizes (product_tiling), so each shape says which form it is there for and the test asks the
rule whether it still is: CTAs of a tile, its halves, the warps that end it, whether the long axis is split, and for the loss in how many pieces the
vocabulary is taken (a later piece adds to the fp32 sums of those before it).

Bounds as in test_gpu_products_large; positions are taken in blocks, so that no matrix of 64 bits is as large as the logits."""
import pytest
import torch

from product_forms import gated_forms, loss_forms
from product_util import BF16, SUM, U
from test_gpu_products_large import check_gated, gated_problem, loss_problem, near

pytestmark = pytest.mark.gpu
ONE, PAIR, HALVES = 1, 2, 3


def form(kind, end_warps=8, split=False):
    return (2 if kind > ONE else 1, 2 if kind == HALVES else 1, end_warps, split)


LOSS = [
    (3, 9, 2, dict(lse=form(ONE), d=form(ONE), dw=form(ONE), dh=form(ONE))),
    (1, 609, 2, dict(lse=form(ONE))),
    (1, 9, 1017, dict(dh=form(ONE, split=True))),
    (1, 1976, 518, dict(dw=form(ONE, 16))),
    (133, 3756, 2295, dict(dh=form(PAIR, split=True))),
    (146, 17, 4896, dict(d=form(ONE, 16))),
    (162, 2182, 2, dict(lse=form(PAIR), d=form(PAIR))),
    (167, 409, 25079, dict(lse=form(PAIR))),
    (184, 2537, 1328, dict(dh=form(PAIR))),
    (295, 1548, 5439, dict(dw=form(PAIR, 16))),
    (386, 3330, 1284, dict(dw=form(HALVES))),
    (710, 1570, 2, dict(dh=form(ONE, 16))),
    (962, 9, 2, dict(dw=form(ONE, split=True))),
    (1458, 955, 410, dict(dw=form(PAIR))),
    (1665, 10, 9547, dict(dw=form(HALVES, split=True))),
    (3853, 1534, 176, dict(dw=form(PAIR, split=True))),
    (9721, 16, 1479, dict(dh=form(HALVES, split=True))),
    (9809, 291, 401, dict(dh=form(HALVES))),
    (9934, 9, 65, dict(lse=form(ONE, 16))),
    (20314, 511, 144, dict(d=form(PAIR, 16))),
    (20644, 486, 210, dict(lse=form(PAIR, 16))),
    (21566, 291, 266, dict(dh=form(PAIR, 16))),
    # two pieces: stored, then added to what is rounded
    (18920, 21, 14155, dict(dh=form(PAIR), pieces=2)),
    (21499, 9, 13047, dict(dh=form(HALVES), pieces=2)),
    (3590, 1052, 127151, dict(dh=form(ONE), pieces=2)),
    (2089, 10, 133458, dict(dh=form(PAIR, split=True), pieces=2)),
    (6201, 129, 49238, dict(dh=form(ONE, split=True), pieces=2)),
    (7310, 9, 36622, dict(dh=form(HALVES, split=True), pieces=2)),
    # three and more: added in memory in between
    (7473, 1139, 84244, dict(dh=form(ONE), pieces=3)),
    (18035, 29, 31706, dict(dh=form(PAIR), pieces=3)),
    (28620, 9, 18980, dict(dh=form(HALVES), pieces=3)),
    (8096, 84, 71656, dict(dh=form(PAIR, split=True), pieces=3)),
    (7125, 14, 76086, dict(dh=form(HALVES, split=True), pieces=3)),
    (16384, 64, 50257, dict(pieces=4)),
    # a micro-batch of the small decoder
    (4096, 896, 151936, dict(lse=form(PAIR), d=form(PAIR), dw=form(PAIR), dh=form(HALVES, split=True), pieces=3)),
]
GATED = [
    (3, 9, 2, dict(h=form(ONE), dx=form(ONE), dw=form(ONE))),
    (1, 12, 456, dict(dx=form(ONE, split=True))),
    (1, 2512, 145, dict(dw=form(ONE, 16))),
    (137, 3120, 1190, dict(dx=form(PAIR, split=True))),
    (139, 2794, 617, dict(dx=form(PAIR))),
    (163, 3422, 2, dict(h=form(PAIR))),
    (283, 1107, 3795, dict(dw=form(PAIR, 16))),
    (396, 593, 3375, dict(dw=form(HALVES))),
    (412, 2723, 2, dict(dx=form(ONE, 16))),
    (994, 14, 2, dict(dw=form(ONE, split=True))),
    (1023, 1000, 2731, dict(dx=form(PAIR, split=True))),
    (1227, 1266, 143, dict(dw=form(PAIR))),
    (2298, 1641, 131, dict(dw=form(PAIR, split=True))),
    (2518, 9, 3148, dict(dw=form(HALVES, split=True))),
    (2984, 1922, 130, dict(dx=form(HALVES))),
    (4273, 3034, 66, dict(dx=form(PAIR, 16))),
    (9495, 11, 752, dict(dx=form(HALVES, split=True))),
]


@pytest.fixture(scope="module")
def ctx():
    import __graft_entry__ as entry
    entry.build()
    from paper_2506_00486_b200 import Context
    c = Context(0, guard=True)
    yield c
    c.check_guards()
    c.close()


def added(got, fresh, base):
    """got = base + the sum that fresh is the bf16 of: that rounding, and the result's."""
    want = fresh.double() + base.double()
    near(got, want, BF16 * (fresh.double().abs() + want.abs() * (1 + BF16)) + 1e-37)


@pytest.mark.parametrize("rows,width,vocab,forms", LOSS)
def test_loss_and_gradient(ctx, rows, width, vocab, forms):
    assert forms.items() <= loss_forms(rows, width, vocab).items()
    h, w, target, dloss = loss_problem(rows + vocab, rows, width, vocab)
    out = ctx.gg_cross_entropy(h, w, target)
    grad = ctx.gg_cross_entropy_grad(dloss, h, w, target, out["lse"])
    base = torch.randn_like(w)
    sums = ctx.gg_cross_entropy_grad(dloss, h, w, target, out["lse"], want_dh=False, dw=base.clone(), accumulate=True)["dw"]
    added(sums, grad["dw"], base)
    w64 = w.double()
    wabs = w64.abs()
    dw, dw_tol, dw_abs = (torch.zeros_like(w64) for _ in range(3))
    block = max(1, (1 << 26) // vocab)
    for first in range(0, rows, block):
        s = slice(first, first + block)
        h64, t = h[s].double(), target[s]
        row, there = torch.arange(t.numel(), device="cuda"), t >= 0
        logits = h64 @ w64.t()
        lse = torch.logsumexp(logits, 1)
        dl = SUM(width) * (h64.abs() @ wabs.t())
        far = logits - lse[:, None]
        p = torch.exp(far)
        err = dl + 4 * U * (far.abs() + 2)
        tol = (p * err).sum(1) + (64 + vocab / 256) * U + 4 * U * (lse.abs() + 12)
        near(out["lse"][s], lse, tol)
        at = torch.where(there, logits[row, t.clamp_min(0)], lse)
        near(out["loss"][s], lse - at, torch.where(there, tol + dl[row, t.clamp_min(0)] + 2 * U * (at.abs() + lse.abs()), 0.0))
        d = torch.exp(logits - out["lse"][s].double()[:, None])
        err = d * err
        d[row[there], t[there]] -= 1.0
        weight = torch.where(there, dloss[s].double(), 0.0)[:, None]
        d, err = d * weight, err * weight
        err = err + 8 * U * d.abs() + BF16 * (d.abs() + err)
        want, tol = d @ w64, err @ wabs + (SUM(vocab) + 256 * U) * (d.abs() @ wabs)
        near(grad["dh"][s], want, tol + BF16 * (want.abs() + tol) + 1e-37)
        dw += d.t() @ h64
        dw_tol += err.t() @ h64.abs()
        dw_abs += d.abs().t() @ h64.abs()
    tol = dw_tol + (SUM(rows) + 256 * U) * dw_abs
    near(grad["dw"], dw, tol + BF16 * (dw.abs() + tol) + 1e-37)


@pytest.mark.parametrize("rows,width,hidden,forms", GATED)
def test_gated_block_and_gradient(ctx, rows, width, hidden, forms):
    assert forms.items() <= gated_forms(rows, width, hidden).items()
    x, wg, wu, dh = gated_problem(rows + hidden, rows, width, hidden)
    check_gated(ctx, x, wg, wu, dh, "silu")
    f = ctx.gg_gated_linear(x, wg, wu, keep=True)
    args = (dh, x, wg, wu, f["gate"], f["up"])
    fresh = ctx.gg_gated_linear_grad(*args, want_dx=False)
    base = [torch.randn_like(wg), torch.randn_like(wg)]
    out = ctx.gg_gated_linear_grad(*args, want_dx=False, dw_gate=base[0].clone(), dw_up=base[1].clone(), accumulate=True)
    for name, b in zip(("dw_gate", "dw_up"), base):
        added(out[name], fresh[name], b)


def test_no_form_is_left_out():
    """Every form that a call of a wide range of shapes takes is one of those above."""
    import math
    import random
    rng = random.Random(3)
    size = lambda least, most: int(round(math.exp(rng.uniform(math.log(least), math.log(most)))))
    have = {"loss": {}, "gated": {}}
    for kind, of, cases in (("loss", loss_forms, LOSS), ("gated", gated_forms, GATED)):
        for *shape, _ in cases:
            for key, value in key_of(kind, shape, of(*shape)):
                have[kind].setdefault(key, set()).add(value)
    for _ in range(20000):
        for kind, of, shape in (("loss", loss_forms, (size(1, 40000), size(1, 8192), size(2, 160000))), ("gated", gated_forms, (size(1, 40000), size(1, 8192), size(1, 16384)))):
            for key, value in key_of(kind, shape, of(*shape)):
                assert value in have[kind][key], (kind, key, value, shape)


def key_of(kind, shape, forms):
    """(operator's part, form); for dh also whether there are one, two or more pieces, for the loss whether its sums are runs."""
    for key, value in forms.items():
        if key == "dh":
            yield key, (value, min(forms["pieces"], 3))
        elif key == "lse":
            yield key, (value, shape[1] > 512)
        elif key != "pieces":
            yield key, value
