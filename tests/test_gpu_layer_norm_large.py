"""Layer norm and its gradient on matrices of many rows, against the 64-bit form computed on the device: every CTA takes
several rows, rows are wide, and the sums over the rows go through slices.

Tolerances: as in test_gpu_layer_norm.py.  u = 2^-24; a sum of n terms in fp32 whose longest chain has D additions is off by at
most D u sum|terms|, D = 48 + n / 64; one rounding for each further operation; bf16 storage adds 2^-8 of a value."""
import pytest
import torch

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TINY = 1e-37


@pytest.fixture(scope="module")
def ctx():
    import __graft_entry__ as entry
    entry.build()
    from paper_2506_00486_b200 import Context
    c = Context(0, guard=True)
    yield c
    c.check_guards()
    c.close()


def matrix(gen, rows, cols, dtype, pad=0, shift=0, scale=1.0, mean=0.0):
    """A [rows, cols] view with row stride cols + pad that starts `shift` elements into its buffer and ends with it."""
    flat = torch.full((rows * (cols + pad) - pad + shift,), 7.0, dtype=dtype, device="cuda")
    t = flat[shift:].as_strided((rows, cols), (cols + pad, 1), shift)
    t.copy_(torch.randn((rows, cols), generator=gen, device="cuda") * scale + mean)
    return t


def affine(gen, cols, dtype):
    return ((1.0 + 0.3 * torch.randn(cols, generator=gen, device="cuda")).to(dtype),
            (0.5 * torch.randn(cols, generator=gen, device="cuda")).to(dtype))


def store(dtype):
    return 2.0 ** -8 if dtype == torch.bfloat16 else U


def within(got, want, tol):
    off = (got.double() - want).abs_()
    assert not torch.isnan(off).any() and (off <= tol).all(), (off - tol).max().item()


def check_forward(x, w, b, eps, out):
    xd, wd, bd = (None if t is None else t.double() for t in (x, w, b))
    n = xd.shape[1]
    D = 48 + n / 64
    mean = xd.mean(1, keepdim=True)
    rstd = 1.0 / torch.sqrt((xd - mean).square().mean(1, keepdim=True) + eps)
    xhat = (xd - mean) * rstd
    y = xhat if wd is None else xhat * wd
    y = y if bd is None else y + bd
    mean_err = (D + 2) * U * xd.abs().mean(1, keepdim=True)
    rstd_rel = ((D + 6) * U + (mean_err * rstd).square() + 2 * U * (xd.abs().amax(1, keepdim=True) * rstd)) / 2 + 3 * U
    tol = mean_err * rstd + U * xd.abs() * rstd + xhat.abs() * (rstd_rel + 4 * U)
    tol = (tol if wd is None else tol * wd.abs()) + 2 * U * y.abs()
    within(out["y"], y, tol + store(x.dtype) * (y.abs() + tol) + TINY)
    within(out["mean"], mean[:, 0], mean_err[:, 0] + TINY)
    within(out["rstd"], rstd[:, 0], (rstd_rel * rstd)[:, 0])


def check_grad(dy, x, mean, rstd, w, out, base=(0.0, 0.0)):
    g, xd, wd = (None if t is None else t.double() for t in (dy, x, w))
    m, r = mean.double()[:, None], rstd.double()[:, None]
    rows, n = xd.shape
    D, DR = 48 + n / 64, 48 + rows / 64
    xhat = (xd - m) * r
    d = g if wd is None else g * wd
    xerr = U * (xd.abs() + m.abs()) * r + 2 * U * xhat.abs()
    if out["dx"] is not None:
        dx = r * (d - d.mean(1, keepdim=True) - xhat * (d * xhat).mean(1, keepdim=True))
        da = d.abs()
        c1, c2 = da.mean(1, keepdim=True), (da * xhat.abs()).mean(1, keepdim=True)
        c2err = (D + 6) * U * c2 + (da * xerr).mean(1, keepdim=True)
        tol = r * (6 * U * da + (D + 6) * U * c1 + xhat.abs() * c2err + xerr * c2 + 6 * U * xhat.abs() * c2)
        within(out["dx"], dx, tol + store(x.dtype) * (dx.abs() + tol) + TINY)
    if out["dweight"] is not None:
        dw, db = base[0] + (g * xhat).sum(0), base[1] + g.sum(0)
        ga = g.abs()
        within(out["dweight"], dw, (DR + 6) * U * (ga * xhat.abs()).sum(0) + (ga * xerr).sum(0) + 2 * U * dw.abs() + TINY)
        within(out["dbias"], db, (DR + 4) * U * ga.sum(0) + 2 * U * db.abs() + TINY)


# fp32 above 8192 columns goes by single elements, weight and bias staged in shared memory as far as it reaches: both sides of
# that limit, and bf16 at the widest row this form takes
@pytest.mark.parametrize("with_affine", [True, False])
@pytest.mark.parametrize("dtype,cols,pad", [("float32", 8200, 0), ("float32", 12284, 0), ("float32", 12285, 0), ("float32", 12288, 0), ("float32", 13001, 0),
                                            ("float32", 13824, 0), ("float32", 14332, 0), ("float32", 14333, 0), ("float32", 16384, 0),
                                            ("bfloat16", 16379, 0), ("bfloat16", 16383, 0), ("bfloat16", 16384, 5)])
def test_wide_rows_in_large_numbers(ctx, dtype, cols, pad, with_affine):
    dtype = getattr(torch, dtype)
    gen = torch.Generator(device="cuda").manual_seed(cols)
    rows = 16 * torch.cuda.get_device_properties(0).multi_processor_count + 5
    x = matrix(gen, rows, cols, dtype, pad, mean=0.2)
    w, b = affine(gen, cols, dtype) if with_affine else (None, None)
    check_forward(x, w, b, 1e-5, ctx.gg_layer_norm(x, w, b))


# the same for the gradient, whose rows (two at a time) reach the limit of shared memory earlier: beyond it each row is read twice
@pytest.mark.parametrize("dtype,cols,pad", [("float32", 8192, 0), ("float32", 9825, 0), ("float32", 11000, 3), ("float32", 11460, 0), ("float32", 11480, 0),
                                            ("float32", 12288, 0), ("bfloat16", 16383, 0), ("bfloat16", 16384, 5), ("bfloat16", 16385, 0)])
def test_gradient_of_wide_rows_in_large_numbers(ctx, dtype, cols, pad):
    dtype = getattr(torch, dtype)
    gen = torch.Generator(device="cuda").manual_seed(cols)
    rows = 16 * torch.cuda.get_device_properties(0).multi_processor_count + 5
    x, dy = matrix(gen, rows, cols, dtype, pad, mean=0.2), matrix(gen, rows, cols, dtype, pad, scale=0.01)
    w, _ = affine(gen, cols, dtype)
    xd = x.double()
    mean = xd.mean(1).float()
    rstd = (1.0 / torch.sqrt((xd - mean.double()[:, None]).square().mean(1) + 1e-5)).float()
    del xd
    check_grad(dy, x, mean, rstd, w, ctx.gg_layer_norm_grad(dy, x, mean, rstd, w))


# Several rows for every warp or CTA of every form.  Vectors: rows within a warp (24, 64, 520), CTAs of 1 to 4 vectors a thread.
# Single elements: 8, 16 and 32 a thread within a warp (200, 511, 1023) and over a CTA (1100, 2001, 5001, 9001, 16383), weight and
# bias staged (many rows) or not.
SHAPES = [(20000, 24), (30011, 64), (20000, 520), (6000, 896), (5000, 2048), (16384, 4096), (4001, 8192), (3001, 16384), (2400, 11008),
          (20011, 31), (15000, 200), (9001, 255), (9001, 511), (4099, 1023), (9001, 1023), (5003, 1100), (1500, 2001), (9000, 2001),
          (3000, 5001), (2003, 9001), (2500, 16383)]


@pytest.mark.parametrize("dtype,w_dtype", [("float32", "float32"), ("bfloat16", "bfloat16"), ("bfloat16", "float32"), ("float32", "bfloat16")])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_forward_and_gradient_of_many_rows(ctx, rows, cols, dtype, w_dtype):
    dtype, w_dtype = getattr(torch, dtype), getattr(torch, w_dtype)
    gen = torch.Generator(device="cuda").manual_seed(rows * 7919 + cols)
    x, dy = matrix(gen, rows, cols, dtype, mean=0.2), matrix(gen, rows, cols, dtype, scale=0.01)
    w, b = affine(gen, cols, w_dtype)
    out = ctx.gg_layer_norm(x, w, b)
    check_forward(x, w, b, 1e-5, out)
    check_grad(dy, x, out["mean"], out["rstd"], w, ctx.gg_layer_norm_grad(dy, x, out["mean"], out["rstd"], w))


@pytest.mark.parametrize("cols", [200, 896, 1023, 2049, 4096])
@pytest.mark.parametrize("pad,shift", [(8, 0), (1, 0), (0, 1), (3, 5)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_strides_alignment_and_in_place_with_many_rows(ctx, cols, pad, shift, dtype):
    dtype, rows = getattr(torch, dtype), 5003
    gen = torch.Generator(device="cuda").manual_seed(cols + 31 * pad + shift)
    x, dy, y, dx = (matrix(gen, rows, cols, dtype, pad, shift) for _ in range(4))
    w, b = affine(gen, cols, dtype)
    out = ctx.gg_layer_norm(x, w, b, out=y)
    check_forward(x, w, b, 1e-5, out)
    grad = ctx.gg_layer_norm_grad(dy, x, out["mean"], out["rstd"], w, dx=dx)
    check_grad(dy, x, out["mean"], out["rstd"], w, grad)
    if pad:      # what lies between the rows is untouched
        for t in (y, dx):
            gap = t.as_strided((rows - 1, pad), (cols + pad, 1), t.storage_offset() + cols)
            assert (gap == 7.0).all()
    # over x, over dy
    again = matrix(gen, rows, cols, dtype, pad, shift)
    again.copy_(x)
    assert torch.equal(ctx.gg_layer_norm(again, w, b, out=again)["y"], y)
    for over in ("dy", "x"):
        g, xx = (matrix(gen, rows, cols, dtype, pad, shift) for _ in range(2))
        g.copy_(dy)
        xx.copy_(x)
        got = ctx.gg_layer_norm_grad(g, xx, out["mean"], out["rstd"], w, dx=g if over == "dy" else xx)
        assert all(torch.equal(got[k], grad[k]) for k in grad), over


@pytest.mark.parametrize("rows,cols", [(3000, 1023), (3000, 1024), (2500, 5001)])
def test_sums_alone_accumulation_and_one_vector_with_many_rows(ctx, rows, cols):
    gen = torch.Generator(device="cuda").manual_seed(cols)
    x, dy = matrix(gen, rows, cols, torch.float32), matrix(gen, rows, cols, torch.float32)
    w, b = affine(gen, cols, torch.float32)
    for ww, bb in ((None, None), (w, None), (None, b)):
        out = ctx.gg_layer_norm(x, ww, bb)
        check_forward(x, ww, bb, 1e-5, out)
    mean, rstd = out["mean"], out["rstd"]
    check_grad(dy, x, mean, rstd, None, ctx.gg_layer_norm_grad(dy, x, mean, rstd, None))
    check_grad(dy, x, mean, rstd, w, ctx.gg_layer_norm_grad(dy, x, mean, rstd, w, want_dx=False))
    dw, db = (torch.randn(cols, generator=gen, device="cuda") for _ in range(2))
    base = dw.double(), db.double()
    got = ctx.gg_layer_norm_grad(dy, x, mean, rstd, w, dweight=dw, dbias=db, accumulate=True)
    check_grad(dy, x, mean, rstd, w, got, base)


@pytest.mark.parametrize("cols", [1000, 1023, 5001])
def test_infinities_and_nan_stay_in_their_row_among_many(ctx, cols):
    gen = torch.Generator(device="cuda").manual_seed(cols)
    rows = 4000
    x = matrix(gen, rows, cols, torch.float32)
    w, b = affine(gen, cols, torch.float32)
    clean = {k: t.clone() for k, t in ctx.gg_layer_norm(x, w, b).items()}
    bad = torch.arange(7, rows, 97, device="cuda")
    x[bad, torch.randint(cols, bad.shape, generator=gen, device="cuda")] = float("inf")
    x[bad[::2], 0] = float("nan")
    out = ctx.gg_layer_norm(x, w, b)
    good = torch.ones(rows, dtype=torch.bool, device="cuda")
    good[bad] = False
    assert torch.isnan(out["y"][bad]).all() and all(torch.equal(out[k][good], clean[k][good]) for k in clean)


@pytest.mark.parametrize("cols", [64, 1000, 1023, 4096])
def test_rows_of_very_large_and_very_small_elements(ctx, cols):
    # squares from 1e-30 to 1e34: sums of both are normal fp32 numbers.  A row beyond that range changes nothing but itself
    gen = torch.Generator(device="cuda").manual_seed(cols)
    rows = 3000
    x = matrix(gen, rows, cols, torch.float32)
    x.mul_((10.0 ** (-15.0 + 32.0 * torch.rand((rows, 1), generator=gen, device="cuda", dtype=torch.float64))).float())
    w, b = affine(gen, cols, torch.float32)
    clean = {k: t.clone() for k, t in ctx.gg_layer_norm(x, w, b, eps=0.0).items()}
    check_forward(x, w, b, 0.0, clean)
    x[5::50] = 1e25 * torch.randn((60, cols), generator=gen, device="cuda")
    out = ctx.gg_layer_norm(x, w, b, eps=0.0)
    huge = torch.zeros(rows, dtype=torch.bool, device="cuda")
    huge[5::50] = True
    assert all(torch.equal(out[k][~huge], clean[k][~huge]) for k in clean)
    assert not out["rstd"][huge].any() and torch.equal(out["y"][huge], b.expand(60, cols))
