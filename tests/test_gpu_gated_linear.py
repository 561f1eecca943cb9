"""The gated block and its gradient against the 64-bit form: every size around the tiles, strides, all activations, extreme
values, halves of one matrix, graphs and streams, refusals.

Bounds: product_util's for sums.  The activation and its derivative are Lipschitz with 1.13 and 0.8 and are evaluated to 16 U (relative, and
of max(1, |a|) where they are sums of two terms); the exponentials take a rounded argument, relative 4 U (|a| + 1)."""
import numpy as np
import pytest
import torch

from oracle import product_oracle as o
from product_util import BF16, SUM, U, around, host, matrix, near

pytestmark = pytest.mark.gpu
ACTS = ["silu", "gelu", "gelu_tanh", "relu"]


@pytest.fixture(scope="module")
def ctx():
    import __graft_entry__ as entry
    entry.build()
    from paper_2506_00486_b200 import Context
    c = Context(0, guard=True)
    yield c
    c.check_guards()
    c.close()


def problem(seed, rows, width, hidden, pad=0, shift=0, scale=1.5):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = matrix(gen, rows, width, pad, shift)
    wg, wu = (matrix(gen, hidden, width, pad, shift, scale / width ** 0.5) for _ in range(2))
    return x, wg, wu, matrix(gen, rows, hidden, pad, shift, 0.1)


def check_forward(x, wg, wu, act, out):
    xd, gd, ud = host(x), host(wg), host(wu)
    h, gate, up = o.gated_linear(xd, gd, ud, act)
    ge, ue = (SUM(x.shape[1]) * (np.abs(xd) @ np.abs(t).T) for t in (gd, ud))
    value, _ = o.activation(gate, act)
    ve = 1.13 * ge + 16 * U * (np.abs(gate) + 1) * np.maximum(np.abs(value), np.abs(gate) * 2.0 ** -20)
    tol = ve * (np.abs(up) + ue) + np.abs(value) * ue + 4 * U * np.abs(h)
    near(out["h"], h, tol + BF16 * (np.abs(h) + tol) + 1e-37, "h")
    if out["gate"] is not None:
        near(out["gate"], gate, ge + BF16 * (np.abs(gate) + ge) + 1e-37, "gate")
        near(out["up"], up, ue + BF16 * (np.abs(up) + ue) + 1e-37, "up")


def check_grad(dh, x, wg, wu, gate, up, act, out, base=None):
    xd, gd, ud, hd, ad, bd = (host(t) for t in (x, wg, wu, dh, gate, up))
    dx, dwg, dwu, dg, du = o.gated_linear_grad(hd, xd, gd, ud, ad, bd, act)
    value, slope = o.activation(ad, act)
    one = 16 * U * (np.abs(ad) + 1)
    dge = np.abs(hd * bd) * (one * np.maximum(np.abs(slope), 0.25)) + BF16 * 1.01 * np.abs(dg)
    due = np.abs(hd) * one * np.maximum(np.abs(value), np.abs(ad) * 2.0 ** -20) + BF16 * 1.01 * np.abs(du)
    if out["dx"] is not None:
        terms = np.abs(dg) @ np.abs(gd) + np.abs(du) @ np.abs(ud)
        tol = dge @ np.abs(gd) + due @ np.abs(ud) + (SUM(2 * wg.shape[0]) + 64 * U) * terms
        near(out["dx"], dx, tol + BF16 * (np.abs(dx) + tol) + 1e-37, "dx")
    for name, want, d, e in (("dw_gate", dwg, dg, dge), ("dw_up", dwu, du, due)):
        if out[name] is not None:
            tol = e.T @ np.abs(xd) + SUM(x.shape[0]) * (np.abs(d).T @ np.abs(xd))
            want = want if base is None else want + base[name]
            near(out[name], want, tol + 2 * U * np.abs(want) + BF16 * (np.abs(want) + tol) + 1e-37, name)


SHAPES = [(1, 1, 1), (1, 64, 128), (2, 7, 5), (3, 896, 200), (64, 128, 129), (127, 65, 300), (128, 64, 128), (129, 130, 127), (256, 256, 384), (257, 33, 513),
          (5, 2048, 64), (700, 40, 70), (33, 1000, 31)]


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("rows,width,hidden", SHAPES)
def test_forward_and_gradient(ctx, rows, width, hidden, act):
    x, wg, wu, dh = problem(rows * 7 + width, rows, width, hidden)
    out = ctx.gg_gated_linear(x, wg, wu, act=act, keep=True)
    check_forward(x, wg, wu, act, out)
    only = ctx.gg_gated_linear(x, wg, wu, act=act)
    assert only["gate"] is None and torch.equal(only["h"], out["h"])
    check_grad(dh, x, wg, wu, out["gate"], out["up"], act, ctx.gg_gated_linear_grad(dh, x, wg, wu, out["gate"], out["up"], act=act))


@pytest.mark.parametrize("pad,shift", [(8, 0), (16, 8), (1, 0), (0, 1), (3, 5), (0, 4)])
@pytest.mark.parametrize("rows,width,hidden", [(13, 96, 300), (130, 77, 131)])
def test_strides_and_alignment(ctx, rows, width, hidden, pad, shift):
    x, wg, wu, dh = problem(pad + 7 * shift + rows, rows, width, hidden, pad=pad, shift=shift)
    gen = torch.Generator(device="cuda").manual_seed(3)
    h, dx = matrix(gen, rows, hidden, pad, shift), matrix(gen, rows, width, pad, shift)
    dwg, dwu = matrix(gen, hidden, width, pad, shift), matrix(gen, hidden, width, pad, shift)
    gate, up = matrix(gen, rows, hidden, pad, shift), matrix(gen, rows, hidden, pad, shift)
    before = [around(t, shift) for t in (h, dx, dwg, dwu)]
    out = ctx.gg_gated_linear(x, wg, wu, out=h, keep=True)
    check_forward(x, wg, wu, "silu", out)
    gate.copy_(out["gate"])
    up.copy_(out["up"])
    check_grad(dh, x, wg, wu, gate, up, "silu", ctx.gg_gated_linear_grad(dh, x, wg, wu, gate, up, dx=dx, dw_gate=dwg, dw_up=dwu))
    for t, b in zip((h, dx, dwg, dwu), before):
        assert torch.equal(around(t, shift), b)


@pytest.mark.parametrize("order", ["stacked", "interleaved"])
def test_both_weights_in_one_matrix(ctx, order):
    gen = torch.Generator(device="cuda").manual_seed(4)
    both = matrix(gen, 2 * 150, 64, scale=0.2)
    wg, wu = (both[:150], both[150:]) if order == "stacked" else (both[::2], both[1::2])
    x, dh = matrix(gen, 70, 64), matrix(gen, 70, 150)
    out = ctx.gg_gated_linear(x, wg, wu, keep=True)
    check_forward(x, wg, wu, "silu", out)
    grads = torch.full_like(both, 5.0)
    dwg, dwu = (grads[:150], grads[150:]) if order == "stacked" else (grads[::2], grads[1::2])
    check_grad(dh, x, wg, wu, out["gate"], out["up"], "silu", ctx.gg_gated_linear_grad(dh, x, wg, wu, out["gate"], out["up"], dw_gate=dwg, dw_up=dwu))


@pytest.mark.parametrize("act", ACTS)
def test_the_whole_range_of_the_activation(ctx, act):
    # one feature: gate runs over a grid, up and dh are 1
    a = torch.cat((torch.linspace(-40, 40, 2001), torch.tensor([0.0, -0.0, 1e-30, -1e-30, 1e4, -1e4, 1e30, -1e30, 200.0, -200.0]))).bfloat16().cuda()
    x = torch.zeros((a.numel(), 2), dtype=torch.bfloat16, device="cuda")
    x[:, 0], x[:, 1] = a, 1.0
    wg, wu = torch.tensor([[1.0, 0.0]], dtype=torch.bfloat16, device="cuda"), torch.tensor([[0.0, 1.0]], dtype=torch.bfloat16, device="cuda")
    out = ctx.gg_gated_linear(x, wg, wu, act=act, keep=True)
    with np.errstate(over="ignore", invalid="ignore"):
        value, slope = o.activation(host(a), act)
    near(out["h"][:, 0], value, (BF16 + 16 * U * (np.abs(host(a)) + 1)) * np.abs(value) + 2.0 ** -120, "value")
    dh = torch.ones((a.numel(), 1), dtype=torch.bfloat16, device="cuda")
    dx = ctx.gg_gated_linear_grad(dh, x, wg, wu, out["gate"], out["up"], act=act, want_dweight=False)["dx"]
    sane = np.abs(host(a)) < 1e5        # (beyond, the 64-bit derivative of the tanh form is inf * 0)
    tol = 2 * BF16 * np.abs(slope) + 16 * U * (np.abs(host(a)) + 1) * np.maximum(np.abs(slope), 0.25) + 2.0 ** -120
    near(host(dx)[sane, 0], slope[sane], tol[sane], "slope")
    assert np.allclose(host(dx)[~sane, 0], np.where(host(a)[~sane] > 0, 1.0, 0.0))


def test_what_is_not_finite_stays_in_its_row(ctx):
    x, wg, wu, dh = problem(5, 140, 64, 200)
    clean = ctx.gg_gated_linear(x, wg, wu, keep=True)
    x2 = x.clone()
    x2[17, 3], x2[139, 0] = float("nan"), float("inf")
    out = ctx.gg_gated_linear(x2, wg, wu, keep=True)
    bad = torch.zeros(140, dtype=torch.bool, device="cuda")
    bad[[17, 139]] = True
    assert torch.isnan(out["h"][17]).all() and not torch.isfinite(out["gate"][139]).any()
    for k in ("h", "gate", "up"):
        assert torch.equal(out[k][~bad], clean[k][~bad])
    for act in ACTS:
        out = ctx.gg_gated_linear(x2, wg, wu, act=act, keep=True)
        assert torch.isnan(out["h"][17]).all()
        dx = ctx.gg_gated_linear_grad(dh, x2, wg, wu, out["gate"], out["up"], act=act, want_dweight=False)["dx"]
        assert torch.isnan(dx[17]).all() and torch.isfinite(dx[~bad]).all()


def test_one_gradient_at_a_time_accumulation_and_repeatability(ctx):
    x, wg, wu, dh = problem(6, 333, 120, 411)
    f = ctx.gg_gated_linear(x, wg, wu, keep=True)
    args = (dh, x, wg, wu, f["gate"], f["up"])
    both = ctx.gg_gated_linear_grad(*args)
    dx, dw = ctx.gg_gated_linear_grad(*args, want_dweight=False), ctx.gg_gated_linear_grad(*args, want_dx=False)
    assert dx["dw_gate"] is None and dw["dx"] is None and torch.equal(dx["dx"], both["dx"])
    assert torch.equal(dw["dw_gate"], both["dw_gate"]) and torch.equal(dw["dw_up"], both["dw_up"])
    gen = torch.Generator(device="cuda").manual_seed(1)
    base = {k: matrix(gen, 411, 120, scale=0.1) for k in ("dw_gate", "dw_up")}
    out = ctx.gg_gated_linear_grad(*args, accumulate=True, **{k: t.clone() for k, t in base.items()})
    check_grad(dh, x, wg, wu, f["gate"], f["up"], "silu", out, base={k: host(t) for k, t in base.items()})


@pytest.mark.parametrize("rows,hidden", [(0, 5), (5, 0)])
def test_nothing_to_do(ctx, rows, hidden):
    x, wg, wu, dh = problem(7, rows, 16, hidden)
    out = ctx.gg_gated_linear(x, wg, wu, keep=True)
    grad = ctx.gg_gated_linear_grad(dh, x, wg, wu, out["gate"], out["up"])
    assert not grad["dx"].any() and not grad["dw_gate"].any() and not grad["dw_up"].any()
    ones = [torch.ones_like(wg) for _ in range(2)]
    ctx.gg_gated_linear_grad(dh, x, wg, wu, out["gate"], out["up"], dw_gate=ones[0], dw_up=ones[1], accumulate=True)
    assert all((t == 1).all() for t in ones)


def test_gradient_against_differences(ctx):
    # relu, so that the forward pass is quadratic between kinks and a central difference exact; steps on one grid with x
    x, wg, wu, dh = problem(8, 30, 24, 90)
    x.copy_((x.float().clamp(-2, 2) * 32).round() / 32)
    f = ctx.gg_gated_linear(x, wg, wu, act="relu", keep=True)
    dx = ctx.gg_gated_linear_grad(dh, x, wg, wu, f["gate"], f["up"], act="relu", want_dweight=False)["dx"]
    sign = torch.where(torch.rand(x.shape, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda") < 0.5, -1.0, 1.0)
    e = 1 / 32
    hs = [ctx.gg_gated_linear((x.float() + s * e * sign).bfloat16(), wg, wu, act="relu")["h"].double() for s in (1, -1)]
    got, want = ((hs[0] - hs[1]) / (2 * e) * dh.double()).sum(1), (dx.double() * sign).sum(1)
    # a rounded h is off by 2^-9 |h| on average over both, and a kink within e |W s| of a gate moves its term by as much
    slack = ((BF16 * (hs[0].abs() + hs[1].abs()) / (2 * e)) * dh.double().abs()).sum(1)
    kinks = (f["gate"].double().abs() <= e * (wg.double() @ sign.t().double()).abs().t() + 0.02).double()
    reach = ((wg.double() @ sign.t().double()).abs().t() * (f["up"].double().abs() + 1.0) * kinks * dh.double().abs()).sum(1)
    assert (got - want).abs().sum() <= (slack + reach + 2 * BF16 * dx.double().abs().sum(1)).sum()


def test_on_another_stream_and_in_a_graph(ctx):
    from paper_2506_00486_b200 import Context
    mine = Context(0)
    x, wg, wu, dh = problem(9, 200, 136, 300, pad=1)          # (operands that are laid out again in scratch)
    want = ctx.gg_gated_linear(x, wg, wu, keep=True)
    wantg = ctx.gg_gated_linear_grad(dh, x, wg, wu, want["gate"], want["up"])
    run = mine.make_gated_linear(x, wg, wu, keep=True)
    grad = mine.make_gated_linear_grad(dh, x, wg, wu, run.outputs["gate"], run.outputs["up"])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
        grad()
    for t in (*run.outputs.values(), *grad.outputs.values()):
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(run.outputs["h"], want["h"]) and all(torch.equal(grad.outputs[k], wantg[k]) for k in wantg)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = mine.gg_gated_linear(x, wg, wu)
    side.synchronize()
    assert torch.equal(again["h"], want["h"])
    del graph
    mine.close()


def test_refusals(ctx):
    from paper_2506_00486_b200 import GGError
    x, wg, wu, dh = problem(10, 8, 16, 20)
    f = ctx.gg_gated_linear(x, wg, wu, keep=True)
    before = ctx.launch_count
    for bad in ((x.float(), wg, wu), (x, wg.half(), wu), (x, wg, wu.float())):
        with pytest.raises(TypeError):
            ctx.gg_gated_linear(*bad)
    for bad, kw in (((x[:, :8], wg, wu), {}), ((x, wg, wu[:5]), {}), ((x, wg, wu), dict(act="swish")), ((x, wg, wu), dict(out=dh[:4])), ((x, wg.t(), wu), {}),
                    ((x.cpu(), wg, wu), {})):
        with pytest.raises(ValueError):
            ctx.gg_gated_linear(*bad, **kw)
    args = (dh, x, wg, wu, f["gate"], f["up"])
    for kw in (dict(dx=x[:4]), dict(dw_gate=wg.float()), dict(accumulate=True), dict(accumulate=True, dw_gate=wg.clone()), dict(act=0)):
        with pytest.raises(ValueError):
            ctx.gg_gated_linear_grad(*args, **kw)
    for kw in (dict(dx=x), dict(dw_gate=wg), dict(dw_up=wg)):
        with pytest.raises(GGError) as e:
            ctx.gg_gated_linear_grad(*args, **kw)
        assert e.value.status == 1
    run = ctx.make_gated_linear(x, wg, wu)
    for field, value, status in (("dtype", 0, 2), ("act", 4, 1), ("act", -1, 1), ("x_ld", 3, 1), ("x", None, 1), ("h", None, 1), ("rows", -1, 1), ("width", 0, 1),
                                 ("hidden", 1 << 31, 1), ("x", x.data_ptr() + 1, 3), ("gate", dh.data_ptr() + 1, 3)):
        keep = getattr(run.args, field)
        setattr(run.args, field, value)
        if field == "gate":
            run.args.gate_ld = 20
        with pytest.raises(GGError) as e:
            run()
        assert e.value.status == status, field
        setattr(run.args, field, keep)
    assert ctx.launch_count == before


@pytest.mark.parametrize("rows", [70, 300, 700])
def test_a_wait_that_runs_out_is_reported_and_leaves_the_context_usable(rows):
    # the barriers of the copies expect more bytes than come: every wait of the kernel runs out, none faults
    from paper_2506_00486_b200 import Context, GGError
    from paper_2506_00486_b200.binding import HOOK_EXTRA_ARRIVALS, HOOK_WAIT_CAP
    mine = Context(0)
    x, wg, wu, dh = problem(11, rows, 200, 300)
    want = mine.gg_gated_linear(x, wg, wu, keep=True)
    wantg = mine.gg_gated_linear_grad(dh, x, wg, wu, want["gate"], want["up"])
    mine.gg_test_hook(HOOK_EXTRA_ARRIVALS, 1)
    mine.gg_test_hook(HOOK_WAIT_CAP, 256)
    mine.gg_gated_linear(x, wg, wu)
    torch.cuda.synchronize()
    with pytest.raises(GGError, match="ran out"):
        mine.gg_gated_linear(x, wg, wu)
    mine.gg_gated_linear_grad(dh, x, wg, wu, want["gate"], want["up"])
    torch.cuda.synchronize()
    mine.gg_test_hook(HOOK_EXTRA_ARRIVALS, 0)
    mine.gg_test_hook(HOOK_WAIT_CAP, 1 << 18)
    with pytest.raises(GGError, match="ran out"):
        mine.gg_gated_linear(x, wg, wu)
    again = mine.gg_gated_linear(x, wg, wu, keep=True)
    grad = mine.gg_gated_linear_grad(dh, x, wg, wu, want["gate"], want["up"])
    assert all(torch.equal(again[k], want[k]) for k in want) and all(torch.equal(grad[k], wantg[k]) for k in wantg)
    mine.close()


def test_outputs_that_are_one_another_are_refused(ctx):
    # (the calls return before anything is launched)
    from paper_2506_00486_b200 import GGError
    x, wg, wu, _ = problem(11, 8, 16, 16)
    run = ctx.make_gated_linear(x, wg, wu, keep=True)
    before = ctx.launch_count
    h, gate, up = (run.outputs[k].data_ptr() for k in ("h", "gate", "up"))
    for change in (dict(gate=h), dict(up=h), dict(gate=up), dict(gate=x.data_ptr()), dict(up=x.data_ptr()), dict(h=x.data_ptr())):
        now = dict(h=h, gate=gate, up=up) | change
        for field, value in now.items():
            setattr(run.args, field, value)
        with pytest.raises(GGError) as e:
            run()
        assert e.value.status == 1
    assert ctx.launch_count == before
