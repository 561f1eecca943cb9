"""The vocabulary loss, the gated block and their gradients at sizes that reach their other forms: tiles of two halves, sums cut into
splits, pieces of the vocabulary, blocks of positions, long sums, elements past 32 bits, and random shapes.  The 64-bit
values come from torch on the device.

Bounds as in the tests of each operator, from product_util's: a sum of n products SUM(n) sum|terms|, half a unit for each bf16 rounding."""
import pytest
import torch

from product_util import BF16, SUM, U, matrix

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


def near(got, want, tol):
    off = (got.double() - want).abs() - tol
    assert bool((off <= 0).all()), float(off.max())


def loss_problem(seed, rows, width, vocab, ignored=0.2, pad=0, shift=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    h, w = matrix(gen, rows, width, pad, shift), matrix(gen, vocab, width, pad, shift, 2.0 / width ** 0.5)
    t = torch.randint(0, vocab, (rows,), generator=gen, device="cuda")
    t = torch.where(torch.rand(rows, generator=gen, device="cuda") < ignored, -100, t)
    return h, w, t, torch.rand(rows, generator=gen, device="cuda") + 0.5


def check_loss(ctx, h, w, target, dloss):
    h64, w64 = h.double(), w.double()
    logits = h64 @ w64.t()
    lse = torch.logsumexp(logits, 1)
    out = ctx.gg_cross_entropy(h, w, target)
    dl = SUM(h.shape[1]) * (h64.abs() @ w64.abs().t())
    p = torch.exp(logits - lse[:, None])
    tol = (p * (dl + 4 * U * ((logits - lse[:, None]).abs() + 2))).sum(1) + (64 + w.shape[0] / 256) * U + 4 * U * (lse.abs() + 12)
    near(out["lse"], lse, tol)
    there, row = target >= 0, torch.arange(h.shape[0], device="cuda")
    at = torch.where(there, logits[row, target.clamp_min(0)], lse)
    near(out["loss"], lse - at, torch.where(there, tol + dl[row, target.clamp_min(0)] + 2 * U * (at.abs() + lse.abs()), 0.0))
    grad = ctx.gg_cross_entropy_grad(dloss, h, w, target, out["lse"])
    d = torch.exp(logits - out["lse"].double()[:, None])
    err = d * (dl + 4 * U * ((logits - lse[:, None]).abs() + 2))
    d[row[there], target[there]] -= 1.0
    weight = torch.where(there, dloss.double(), 0.0)[:, None]
    d, err = d * weight, err * weight
    err = err + 8 * U * d.abs() + BF16 * (d.abs() + err)
    for name, a, b, n in (("dh", d, w64, w.shape[0]), ("dw", d.t(), h64, h.shape[0])):
        want, tol = a @ b, (err if name == "dh" else err.t()) @ b.abs() + (SUM(n) + 256 * U) * (a.abs() @ b.abs())
        near(grad[name], want, tol + BF16 * (want.abs() + tol) + 1e-37)


def act_and_slope(a, act):
    a = a.double().requires_grad_(True)
    f = {"silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu, "relu": torch.nn.functional.relu,
         "gelu_tanh": lambda v: torch.nn.functional.gelu(v, approximate="tanh")}[act](a)
    return f.detach(), torch.autograd.grad(f.sum(), a)[0]


def check_gated(ctx, x, wg, wu, dh, act):
    x64, g64, u64 = x.double(), wg.double(), wu.double()
    gate, up = x64 @ g64.t(), x64 @ u64.t()
    ge, ue = (SUM(x.shape[1]) * (x64.abs() @ t.abs().t()) for t in (g64, u64))
    value, _ = act_and_slope(gate, act)
    out = ctx.gg_gated_linear(x, wg, wu, act=act, keep=True)
    ve = 1.13 * ge + 16 * U * (gate.abs() + 1) * torch.maximum(value.abs(), gate.abs() * 2.0 ** -20)
    tol = ve * (up.abs() + ue) + value.abs() * ue + 4 * U * (value * up).abs()
    near(out["h"], value * up, tol + BF16 * ((value * up).abs() + tol) + 1e-37)
    near(out["gate"], gate, ge + BF16 * (gate.abs() + ge))
    grad = ctx.gg_gated_linear_grad(dh, x, wg, wu, out["gate"], out["up"], act=act)
    value, slope = act_and_slope(out["gate"], act)
    d64, a, b = dh.double(), out["gate"].double(), out["up"].double()
    dg, du = d64 * b * slope, d64 * value
    one = 16 * U * (a.abs() + 1)
    dge = (d64 * b).abs() * (one * slope.abs().clamp_min(0.25)) + BF16 * 1.01 * dg.abs()
    due = d64.abs() * one * torch.maximum(value.abs(), a.abs() * 2.0 ** -20) + BF16 * 1.01 * du.abs()
    want = dg @ g64 + du @ u64
    tol = dge @ g64.abs() + due @ u64.abs() + (SUM(2 * wg.shape[0]) + 64 * U) * (dg.abs() @ g64.abs() + du.abs() @ u64.abs())
    near(grad["dx"], want, tol + BF16 * (want.abs() + tol) + 1e-37)
    for name, d, e in (("dw_gate", dg, dge), ("dw_up", du, due)):
        want, tol = d.t() @ x64, e.t() @ x64.abs() + SUM(x.shape[0]) * (d.abs().t() @ x64.abs())
        near(grad[name], want, tol + BF16 * (want.abs() + tol) + 1e-37)


def gated_problem(seed, rows, width, hidden, pad=0, shift=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (matrix(gen, rows, width, pad, shift), *(matrix(gen, hidden, width, pad, shift, 1.5 / width ** 0.5) for _ in range(2)),
            matrix(gen, rows, hidden, pad, shift, 0.1))


# positions beyond one block; pieces of the vocabulary (more than 512 MB of logits' gradient); a long sum over few and over many rows
@pytest.mark.parametrize("rows,width,vocab", [(33001, 16, 300), (33000, 40, 9000), (20, 64, 40000), (5000, 520, 700), (1030, 4104, 1100), (300, 2048, 3000), (9000, 72, 500)])
def test_loss_forms(ctx, rows, width, vocab):
    check_loss(ctx, *loss_problem(rows, rows, width, vocab))


@pytest.mark.parametrize("rows,width,hidden", [(20000, 520, 300), (3000, 1100, 2056), (600, 4104, 520), (40, 300, 9000), (1, 5000, 70), (1, 30000, 6), (9000, 65, 300)])
def test_gated_forms(ctx, rows, width, hidden):
    check_gated(ctx, *gated_problem(rows, rows, width, hidden), "silu")


@pytest.mark.parametrize("seed", range(30))
def test_random_shapes(ctx, seed):
    rng = torch.Generator().manual_seed(seed)

    def size(most):
        return int(round(float(most) ** float(torch.rand(1, generator=rng))))

    pad, shift = (int(torch.randint(0, 10, (1,), generator=rng)) for _ in range(2))
    check_loss(ctx, *loss_problem(seed, size(3000), size(1500), size(6000), pad=pad, shift=shift))
    act = ("silu", "gelu", "gelu_tanh", "relu")[seed % 4]
    check_gated(ctx, *gated_problem(seed, size(3000), size(1500), size(2500), pad=shift, shift=pad), act)


@pytest.mark.parametrize("width", [72, 65])
def test_gradients_of_weights_that_are_split_and_added(ctx, width):
    # few columns, many rows: the sums are cut into splits, joined, and added to what is there
    x, wg, wu, dh = gated_problem(3, 9000, width, 300)
    f = ctx.gg_gated_linear(x, wg, wu, keep=True)
    args = (dh, x, wg, wu, f["gate"], f["up"])
    fresh = ctx.gg_gated_linear_grad(*args)
    base = [torch.randn_like(wg), torch.randn_like(wg)]
    out = ctx.gg_gated_linear_grad(*args, dw_gate=base[0].clone(), dw_up=base[1].clone(), accumulate=True)
    for name, b in zip(("dw_gate", "dw_up"), base):
        want = fresh[name].double() + b.double()       # (fresh is rounded once, the sum once)
        near(out[name], want, BF16 * (fresh[name].double().abs() + want.abs() * (1 + BF16)) + 1e-37)
    h, w, target, dloss = loss_problem(4, 9000, width, 500)
    lse = ctx.gg_cross_entropy(h, w, target)["lse"]
    fresh = ctx.gg_cross_entropy_grad(dloss, h, w, target, lse)["dw"]
    base = torch.randn_like(w)
    out = ctx.gg_cross_entropy_grad(dloss, h, w, target, lse, dw=base.clone(), accumulate=True)["dw"]
    want = fresh.double() + base.double()
    near(out, want, BF16 * (fresh.double().abs() + want.abs() * (1 + BF16)) + 1e-37)


def test_elements_past_32_bits(ctx):
    # 40000 rows, 60000 elements apart: the last begin beyond 2^31
    rows, ld = 40000, 60000
    wide = torch.zeros(rows * ld, dtype=torch.bfloat16, device="cuda").view(rows, ld)
    h, w, target, dloss = loss_problem(1, 200, 64, rows)
    wide[:, 1000:1064] = w
    far = wide[:, 1000:1064]
    near_out, far_out = ctx.gg_cross_entropy(h, w, target), ctx.gg_cross_entropy(h, far, target)
    assert torch.equal(near_out["lse"], far_out["lse"])
    want = ctx.gg_cross_entropy_grad(dloss, h, w, target, near_out["lse"])
    got = ctx.gg_cross_entropy_grad(dloss, h, far, target, near_out["lse"], dw=wide[:, 2000:2064])
    assert torch.equal(got["dw"], want["dw"]) and torch.equal(got["dh"], want["dh"])
    assert not wide[:, :1000].any() and not wide[:, 1064:2000].any() and not wide[:, 2064:].any()
    # the same far places as rows and results of the gated block
    _, wg, wu, _ = gated_problem(2, 1, 64, 40)
    a = ctx.gg_gated_linear(w, wg, wu, keep=True)
    b = ctx.gg_gated_linear(far, wg, wu, out=wide[:, 3000:3040], keep=True)
    assert all(torch.equal(a[k], b[k]) for k in a)
    ga = ctx.gg_gated_linear_grad(a["h"], w, wg, wu, a["gate"], a["up"])
    gb = ctx.gg_gated_linear_grad(b["h"], far, wg, wu, a["gate"], a["up"], dx=wide[:, 4000:4064])
    assert all(torch.equal(ga[k], gb[k]) for k in ga)
