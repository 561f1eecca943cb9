"""Layer norm and its gradient against the 64-bit form: types, widths that no vector divides, strides, in place, one
row and none, rows with infinities.

Tolerances.  u = 2^-24.  A sum of n terms in fp32 whose longest chain has D additions is off by at most
D u sum|terms|; D is taken as 48 + n / 64 (a chain per thread and a tree over threads).  The bounds below follow from
that and from one rounding for each further operation, and bf16 storage adds 2^-8 of a value (half a unit is 2^-9, and
a value within the fp32 error of a tie may go the other way)."""
import numpy as np
import pytest
import torch

from oracle import train_oracle as o

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def ctx():
    import __graft_entry__ as entry
    entry.build()
    from paper_2506_00486_b200 import Context
    c = Context(0, guard=True)
    yield c
    c.check_guards()
    c.close()


def host(t):
    return None if t is None else t.double().cpu().numpy()


def matrix(gen, rows, cols, dtype, pad=0, shift=0, scale=1.0, mean=0.0):
    """A [rows, cols] view with row stride cols + pad that starts `shift` elements into its buffer."""
    flat = torch.full((rows * (cols + pad) + shift + 8,), 7.0, dtype=dtype, device="cuda")
    t = flat[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    t.copy_(torch.randn((rows, cols), generator=gen, device="cuda") * scale + mean)
    return t


def affine(gen, cols, dtype):
    return ((1.0 + 0.3 * torch.randn(cols, generator=gen, device="cuda")).to(dtype),
            (0.5 * torch.randn(cols, generator=gen, device="cuda")).to(dtype))


def store(dtype):
    return 2.0 ** -8 if dtype == torch.bfloat16 else U


def check_forward(x, w, b, eps, out):
    xd, wd, bd = host(x), host(w), host(b)
    y, mean, rstd = o.layer_norm(xd, wd, bd, eps)
    n = xd.shape[1]
    D = 48 + n / 64
    mean_err = (D + 2) * U * np.abs(xd).mean(axis=1)
    # the variance moves by the square of the error of the mean, and by the roundings of its own sum
    rstd_rel = ((D + 6) * U + (mean_err * rstd) ** 2 + 2 * U * (np.abs(xd).max(axis=1) * rstd)) / 2 + 3 * U
    wa = np.abs(wd) if wd is not None else 1.0
    xhat = np.abs(xd - mean[:, None]) * rstd[:, None]
    tol = wa * ((mean_err * rstd)[:, None] + U * np.abs(xd) * rstd[:, None] + xhat * (rstd_rel[:, None] + 4 * U)) + 2 * U * np.abs(y)
    tol = tol + store(x.dtype) * (np.abs(y) + tol) + 1e-37
    assert np.all(np.abs(host(out["y"]) - y) <= tol)
    assert np.all(np.abs(host(out["mean"]) - mean) <= mean_err + 1e-37)
    assert np.all(np.abs(host(out["rstd"]) - rstd) <= rstd_rel * rstd)


def check_grad(dy, x, mean, rstd, w, out, base=(0.0, 0.0)):
    dyd, xd, md, rd, wd = host(dy), host(x), host(mean), host(rstd), host(w)
    dx, dw, db = o.layer_norm_grad(dyd, xd, md, rd, wd)
    rows, n = xd.shape
    D, DR = 48 + n / 64, 48 + rows / 64
    # xhat carries the rounding of x - mean, which a large mean makes large against xhat
    xerr = (U * (np.abs(xd) + np.abs(md[:, None])) * rd[:, None]) + 2 * U * np.abs((xd - md[:, None]) * rd[:, None])
    xhat = np.abs((xd - md[:, None]) * rd[:, None])
    d = np.abs(dyd * (1.0 if wd is None else wd))
    c1, c2 = d.mean(axis=1, keepdims=True), (d * xhat).mean(axis=1, keepdims=True)
    c2err = (D + 6) * U * c2 + (d * xerr).mean(axis=1, keepdims=True)
    tol = rd[:, None] * (6 * U * d + (D + 6) * U * c1 + xhat * c2err + xerr * c2 + 6 * U * xhat * c2)
    tol = tol + store(x.dtype) * (np.abs(dx) + tol) + 1e-37
    if out["dx"] is not None:
        assert np.all(np.abs(host(out["dx"]) - dx) <= tol)
    if out["dweight"] is not None:
        t = (DR + 6) * U * (np.abs(dyd) * xhat).sum(axis=0) + (np.abs(dyd) * xerr).sum(axis=0) + 2 * U * np.abs(base[0] + dw) + 1e-37
        assert np.all(np.abs(host(out["dweight"]) - (base[0] + dw)) <= t)
    if out["dbias"] is not None:
        t = (DR + 4) * U * np.abs(dyd).sum(axis=0) + 2 * U * np.abs(base[1] + db) + 1e-37
        assert np.all(np.abs(host(out["dbias"]) - (base[1] + db)) <= t)


SHAPES = [(1, 1), (1, 896), (3, 2), (7, 8), (5, 31), (2, 255), (33, 256), (9, 1000), (4, 1023), (300, 1024), (5, 2048), (3, 4096), (2, 4104),
          (3, 8192), (2, 11008), (2, 16384), (1, 20000), (2, 40000), (700, 64), (5000, 24), (1300, 520)]


@pytest.mark.parametrize("dtype,w_dtype", [("float32", "float32"), ("bfloat16", "bfloat16"), ("bfloat16", "float32"), ("float32", "bfloat16")])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_forward_and_gradient(ctx, rows, cols, dtype, w_dtype):
    dtype, w_dtype = getattr(torch, dtype), getattr(torch, w_dtype)
    gen = torch.Generator(device="cuda").manual_seed(rows * 7919 + cols)
    x, dy = matrix(gen, rows, cols, dtype, mean=0.2), matrix(gen, rows, cols, dtype, scale=0.01)
    w, b = affine(gen, cols, w_dtype)
    out = ctx.gg_layer_norm(x, w, b)
    check_forward(x, w, b, 1e-5, out)
    grad = ctx.gg_layer_norm_grad(dy, x, out["mean"], out["rstd"], w)
    check_grad(dy, x, out["mean"], out["rstd"], w, grad)


@pytest.mark.parametrize("cols", [96, 1000, 1024, 4096, 9000])
@pytest.mark.parametrize("pad,shift", [(8, 0), (16, 8), (1, 0), (0, 1), (3, 5)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_strides_and_alignment(ctx, cols, pad, shift, dtype):
    dtype = getattr(torch, dtype)
    gen = torch.Generator(device="cuda").manual_seed(cols + 31 * pad + shift)
    rows = 13
    x, dy = matrix(gen, rows, cols, dtype, pad, shift), matrix(gen, rows, cols, dtype, pad, shift)
    w, b = affine(gen, cols, dtype)
    y, dx = matrix(gen, rows, cols, dtype, pad, shift), matrix(gen, rows, cols, dtype, pad, shift)
    before = [t.clone() for t in (y.as_strided((rows * (cols + pad),), (1,)), dx.as_strided((rows * (cols + pad),), (1,)))]
    out = ctx.gg_layer_norm(x, w, b, out=y)
    check_forward(x, w, b, 1e-5, out)
    check_grad(dy, x, out["mean"], out["rstd"], w, ctx.gg_layer_norm_grad(dy, x, out["mean"], out["rstd"], w, dx=dx))
    if pad:      # what lies between the rows is untouched
        for t, old in zip((y, dx), before):
            gap = t.as_strided((rows, cols + pad), (cols + pad, 1))[:, cols:]
            assert torch.equal(gap, old.view(rows, cols + pad)[:, cols:])


@pytest.mark.parametrize("misaligned", ["weight", "bias", "y", "dy", "dx"])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_one_operand_off_the_vector_boundary(ctx, misaligned, dtype):
    dtype, rows, cols = getattr(torch, dtype), 6, 2048
    gen = torch.Generator(device="cuda").manual_seed(5)

    def at(name):
        return 1 if name == misaligned else 0

    x = matrix(gen, rows, cols, dtype)
    dy, y, dx = (matrix(gen, rows, cols, dtype, shift=at(n)) for n in ("dy", "y", "dx"))
    w = torch.cat([torch.ones(at("weight"), device="cuda"), torch.randn(cols, generator=gen, device="cuda")]).to(dtype)[at("weight"):]
    b = torch.cat([torch.ones(at("bias"), device="cuda"), torch.randn(cols, generator=gen, device="cuda")]).to(dtype)[at("bias"):]
    out = ctx.gg_layer_norm(x, w, b, out=y)
    check_forward(x, w, b, 1e-5, out)
    check_grad(dy, x, out["mean"], out["rstd"], w, ctx.gg_layer_norm_grad(dy, x, out["mean"], out["rstd"], w, dx=dx))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("cols", [130, 1024, 4096, 40000])
def test_without_weight_and_bias_and_with_one_of_them(ctx, dtype, cols):
    dtype = getattr(torch, dtype)
    gen = torch.Generator(device="cuda").manual_seed(cols)
    x, dy = matrix(gen, 9, cols, dtype), matrix(gen, 9, cols, dtype)
    w, b = affine(gen, cols, torch.float32)
    for ww, bb in ((None, None), (w, None), (None, b)):
        out = ctx.gg_layer_norm(x, ww, bb)
        check_forward(x, ww, bb, 1e-5, out)
        grad = ctx.gg_layer_norm_grad(dy, x, out["mean"], out["rstd"], ww)
        assert (grad["dweight"] is None) == (ww is None)
        check_grad(dy, x, out["mean"], out["rstd"], ww, grad)
    grad = ctx.gg_layer_norm_grad(dy, x, out["mean"], out["rstd"], None, want_dx=False, want_dweight=True)
    assert grad["dx"] is None
    check_grad(dy, x, out["mean"], out["rstd"], None, grad)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("cols", [33, 1024, 4096, 30000])
def test_in_place(ctx, dtype, cols):
    dtype = getattr(torch, dtype)
    gen = torch.Generator(device="cuda").manual_seed(cols)
    x, dy = matrix(gen, 40, cols, dtype), matrix(gen, 40, cols, dtype)
    w, b = affine(gen, cols, dtype)
    out = ctx.gg_layer_norm(x, w, b)
    y = x.clone()
    ctx.gg_layer_norm(y, w, b, out=y)
    assert torch.equal(y, out["y"])
    want = ctx.gg_layer_norm_grad(dy, x, out["mean"], out["rstd"], w)
    for over in ("dy", "x"):
        d, xx = dy.clone(), x.clone()
        got = ctx.gg_layer_norm_grad(d, xx, out["mean"], out["rstd"], w, dx=d if over == "dy" else xx)
        for k in ("dx", "dweight", "dbias"):
            assert torch.equal(got[k], want[k]), (over, k)


@pytest.mark.parametrize("cols", [100, 1024, 4096])
def test_a_large_mean_and_a_constant_row(ctx, cols):
    gen = torch.Generator(device="cuda").manual_seed(cols)
    x = matrix(gen, 6, cols, torch.float32, mean=3000.0)
    x[2] = 5.0
    x[3] = 0.0
    w, b = affine(gen, cols, torch.float32)
    out = ctx.gg_layer_norm(x, w, b)
    check_forward(x, w, b, 1e-5, out)
    assert torch.equal(out["y"][2], b) and torch.equal(out["y"][3], b)
    # no row is without spread here, so eps may be 0
    x = matrix(gen, 6, cols, torch.float32)
    check_forward(x, w, b, 0.0, ctx.gg_layer_norm(x, w, b, eps=0.0))


@pytest.mark.parametrize("cols", [100, 1024, 4096, 30000])
def test_infinities_and_nan_stay_in_their_row(ctx, cols):
    gen = torch.Generator(device="cuda").manual_seed(cols)
    x, dy = matrix(gen, 8, cols, torch.float32), matrix(gen, 8, cols, torch.float32)
    w, b = affine(gen, cols, torch.float32)
    clean = ctx.gg_layer_norm(x, w, b)
    x2 = x.clone()
    x2[1, 3], x2[4, cols - 1], x2[6, 0] = float("inf"), float("nan"), -float("inf")
    out = ctx.gg_layer_norm(x2, w, b)
    bad = torch.tensor([1, 4, 6], device="cuda")
    good = torch.tensor([0, 2, 3, 5, 7], device="cuda")
    assert torch.isnan(out["y"][bad]).all() and torch.equal(out["y"][good], clean["y"][good])
    grad, want = (ctx.gg_layer_norm_grad(dy, x2, s["mean"], s["rstd"], w) for s in (out, clean))
    ref = ctx.gg_layer_norm_grad(dy, x, clean["mean"], clean["rstd"], w)
    assert torch.isnan(grad["dx"][bad]).all() and torch.equal(grad["dx"][good], ref["dx"][good])
    assert torch.isnan(grad["dweight"]).all() and torch.equal(grad["dbias"], ref["dbias"])
    assert want["dx"].shape == x.shape


@pytest.mark.parametrize("rows,cols", [(0, 64), (5, 0), (0, 0)])
def test_nothing_to_do(ctx, rows, cols):
    x = torch.empty((rows, cols), device="cuda")
    out = ctx.gg_layer_norm(x)
    assert out["y"].shape == x.shape
    one = torch.ones(cols, device="cuda")
    zeros = torch.zeros(rows, device="cuda")
    grad = ctx.gg_layer_norm_grad(x, x, zeros, zeros, one)
    assert not grad["dweight"].any() and not grad["dbias"].any()


@pytest.mark.parametrize("rows,cols", [(1, 17), (200, 1024), (999, 4096)])
def test_accumulation_and_repeatability(ctx, rows, cols):
    gen = torch.Generator(device="cuda").manual_seed(rows)
    x, dy = matrix(gen, rows, cols, torch.bfloat16), matrix(gen, rows, cols, torch.bfloat16)
    w, b = affine(gen, cols, torch.bfloat16)
    out = ctx.gg_layer_norm(x, w, b)
    first = ctx.gg_layer_norm_grad(dy, x, out["mean"], out["rstd"], w)
    again = ctx.gg_layer_norm_grad(dy, x, out["mean"], out["rstd"], w)
    for k in first:
        assert torch.equal(first[k], again[k])
    dw, db = (torch.randn(cols, generator=gen, device="cuda") for _ in range(2))
    base = host(dw), host(db)
    got = ctx.gg_layer_norm_grad(dy, x, out["mean"], out["rstd"], w, dweight=dw, dbias=db, accumulate=True)
    assert got["dweight"] is dw and got["dbias"] is db
    check_grad(dy, x, out["mean"], out["rstd"], w, got, base)


def test_gradient_against_differences_of_the_forward_pass(ctx):
    # L = sum(dy * y); along a direction e of x the difference quotient of two fp32 forward passes, summed in fp64, has
    # the rounding error of y (4u |y|, independent over n elements) over 2h, and h^2 of the third derivative
    gen = torch.Generator(device="cuda").manual_seed(11)
    rows, cols, h = 64, 768, 1e-2
    x, dy, e = (matrix(gen, rows, cols, torch.float32) for _ in range(3))
    w, b = affine(gen, cols, torch.float32)
    out = ctx.gg_layer_norm(x, w, b)
    grad = ctx.gg_layer_norm_grad(dy, x, out["mean"], out["rstd"], w)
    up, down = (ctx.gg_layer_norm(x + s * h * e, w, b)["y"] for s in (1, -1))
    quotient = ((up.double() - down.double()) * dy.double()).sum().item() / (2 * h)
    want = (grad["dx"].double() * e.double()).sum().item()
    n = rows * cols
    assert abs(quotient - want) <= 40 * (U / h) * n ** 0.5 + 40 * h * h * n ** 0.5


def test_on_another_stream_and_in_a_graph(ctx):
    gen = torch.Generator(device="cuda").manual_seed(2)
    x, dy = matrix(gen, 257, 1024, torch.bfloat16), matrix(gen, 257, 1024, torch.bfloat16)
    w, b = affine(gen, 1024, torch.bfloat16)
    fwd = ctx.make_layer_norm(x, w, b)
    ref = {k: v.clone() for k, v in fwd().items()}
    bwd = ctx.make_layer_norm_grad(dy, x, fwd.outputs["mean"], fwd.outputs["rstd"], w)
    refg = {k: v.clone() for k, v in bwd().items()}
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for t in (*fwd.outputs.values(), *bwd.outputs.values()):
        t.zero_()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        fwd()
        bwd()
    side.synchronize()
    assert all(torch.equal(fwd.outputs[k], ref[k]) for k in ref) and all(torch.equal(bwd.outputs[k], refg[k]) for k in refg)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fwd()
        bwd()
    for t in (*fwd.outputs.values(), *bwd.outputs.values()):
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(fwd.outputs[k], ref[k]) for k in ref) and all(torch.equal(bwd.outputs[k], refg[k]) for k in refg)


def test_rows_past_32_bits_of_offset(ctx):
    # 70001 rows 61440 elements apart: the last row starts past element 2^32
    gen = torch.Generator(device="cuda").manual_seed(4)
    rows, cols, ld = 70001, 520, 61440
    flat = torch.empty((rows - 1) * ld + cols, dtype=torch.bfloat16, device="cuda")
    x = flat.as_strided((rows, cols), (ld, 1))
    x.copy_(torch.randn((rows, cols), generator=gen, device="cuda"))
    w, b = affine(gen, cols, torch.bfloat16)
    out = ctx.gg_layer_norm(x, w, b)
    near = ctx.gg_layer_norm(x.contiguous(), w, b)
    assert torch.equal(out["y"], near["y"])
    dy = near["y"]
    a = ctx.gg_layer_norm_grad(dy, x, out["mean"], out["rstd"], w)
    c = ctx.gg_layer_norm_grad(dy, x.contiguous(), out["mean"], out["rstd"], w)
    assert all(torch.equal(a[k], c[k]) for k in a)


def test_refusals(ctx):
    from paper_2506_00486_b200 import GGError, binding
    x = torch.randn(4, 64, device="cuda")
    one, rows = torch.ones(64, device="cuda"), torch.ones(4, device="cuda")
    before = ctx.launch_count
    for call in (lambda: ctx.gg_layer_norm(x.t()), lambda: ctx.gg_layer_norm(x[0]), lambda: ctx.gg_layer_norm(x.cpu()),
                 lambda: ctx.gg_layer_norm(x, one[:63]), lambda: ctx.gg_layer_norm(x, one, one.bfloat16()),
                 lambda: ctx.gg_layer_norm(x, out=x.bfloat16()), lambda: ctx.gg_layer_norm(x[:1].expand(4, 64)),
                 lambda: ctx.gg_layer_norm_grad(x[:3], x, rows, rows), lambda: ctx.gg_layer_norm_grad(x, x, rows[:3], rows),
                 lambda: ctx.gg_layer_norm_grad(x, x, rows.double(), rows),
                 lambda: ctx.gg_layer_norm_grad(x, x, rows, rows, one, accumulate=True),
                 lambda: ctx.gg_layer_norm_grad(x, x, rows, rows, one, dweight=one.bfloat16(), dbias=one)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        ctx.gg_layer_norm(x.double())
    for eps in (-1e-5, float("nan")):
        with pytest.raises(GGError) as e:
            ctx.gg_layer_norm(x, eps=eps)
        assert e.value.status == 1
    # what only the C interface can be given
    run = ctx.make_layer_norm(x, one, one)
    back = ctx.make_layer_norm_grad(x, x, rows, rows, one)
    L = binding.lib()

    def status(entry, args, **change):
        a = type(args).from_buffer_copy(args)
        for k, v in change.items():
            setattr(a, k, v)
        return getattr(L, entry)(ctx._h, binding.ctypes.byref(a), None)

    p = x.data_ptr()
    for entry, args, cases in (
            ("gg_layer_norm", run.args, [(dict(rows=-1), 1), (dict(cols=-1), 1), (dict(x_ld=63), 1), (dict(y_ld=63), 1), (dict(x=None), 1),
                                         (dict(y=None), 1), (dict(dtype=2), 2), (dict(w_dtype=9), 2), (dict(x=p + 2), 3), (dict(y=p + 1), 3),
                                         (dict(weight=p + 2), 3), (dict(mean=p + 1), 3), (dict(rstd=p + 2), 3)]),
            ("gg_layer_norm_grad", back.args, [(dict(rows=-1), 1), (dict(cols=-4), 1), (dict(dy_ld=1), 1), (dict(x_ld=1), 1), (dict(dx_ld=1), 1),
                                               (dict(mean=None), 1), (dict(rstd=None), 1), (dict(dy=None), 1), (dict(x=None), 1),
                                               (dict(dtype=-1), 2), (dict(w_dtype=2), 2), (dict(dy=p + 2), 3), (dict(dx=p + 1), 3),
                                               (dict(weight=p + 1), 3), (dict(dweight=p + 2), 3), (dict(dbias=p + 1), 3)])):
        for change, want in cases:
            assert status(entry, args, **change) == want, (entry, change)
        assert getattr(L, entry)(ctx._h, None, None) == 1 and getattr(L, entry)(None, binding.ctypes.byref(args), None) == 1
    assert ctx.launch_count == before
