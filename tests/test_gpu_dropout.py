"""Dropout against the 64-bit form: the mask bit for bit, types, odd widths, strides, in place, the residual, what is dropped
whatever it is, a step that a captured graph advances, positions past 32 bits, refusals.

Bounds: a kept element is scaled by a factor rounded once and the product is rounded once, the residual adds one more rounding:
3 U of each magnitude, and the storage type's half unit."""
import numpy as np
import pytest
import torch

from oracle import product_oracle as o
from product_util import BF16, U, around, host, matrix, near

pytestmark = pytest.mark.gpu
SEED = 0x123456789ABCDEF0


@pytest.fixture(scope="module")
def ctx():
    import __graft_entry__ as entry
    entry.build()
    from paper_2506_00486_b200 import Context
    c = Context(0, guard=True)
    yield c
    c.check_guards()
    c.close()


def check(x, p, y, t, tensor_id=0, residual=None, seed=SEED):
    rows, cols = x.shape
    bits = o.dropout_bits(rows, cols, t, tensor_id, seed)
    want = o.dropout(host(x), p, bits, host(residual))
    big = np.abs(o.dropout(host(x), p, bits)) + (0 if residual is None else np.abs(host(residual)))
    near(y, want, 3 * U * big + (BF16 if y.dtype == torch.bfloat16 else U) * (np.abs(want) + 3 * U * big) + 1e-37)
    if residual is None and p > 0:
        assert np.array_equal(host(y) == 0, (bits < int(np.floor(p * 65536 + 0.5))) | (host(x) == 0))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 7), (3, 8), (2, 9), (7, 1000), (1, 4096), (300, 1023), (5, 16384), (1000, 24), (4099, 1), (64, 896)])
def test_mask_and_values(ctx, rows, cols, dtype):
    gen = torch.Generator(device="cuda").manual_seed(rows + cols)
    x, r = (matrix(gen, rows, cols, dtype=getattr(torch, dtype)) for _ in range(2))
    for t, p, res in ((1, 0.1, None), (2, 0.5, r), (2 ** 40 + 3, 0.9, None)):
        check(x, p, ctx.gg_dropout(x, p, t, residual=res, seed=SEED, tensor_id=rows)["y"], t, rows, res)


@pytest.mark.parametrize("pad,shift", [(8, 0), (1, 0), (0, 1), (3, 5), (4, 4)])
@pytest.mark.parametrize("cols", [64, 96, 1001])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_strides_and_alignment(ctx, cols, pad, shift, dtype):
    gen, dtype = torch.Generator(device="cuda").manual_seed(cols + pad), getattr(torch, dtype)
    x, r, y = (matrix(gen, 13, cols, pad, shift, dtype=dtype) for _ in range(3))
    before = around(y, shift)
    check(x, 0.3, ctx.gg_dropout(x, 0.3, 5, residual=r, out=y, seed=SEED)["y"], 5, residual=r)
    assert torch.equal(around(y, shift), before)
    # the mask does not depend on strides, alignment or type
    dense = ctx.gg_dropout(x.contiguous().float(), 0.3, 5, seed=SEED)["y"]
    assert torch.equal(dense == 0, ctx.gg_dropout(x, 0.3, 5, seed=SEED)["y"] == 0)


@pytest.mark.parametrize("which", [0, 1, 2])
def test_one_operand_off_the_vector_boundary(ctx, which):
    gen = torch.Generator(device="cuda").manual_seed(which)
    x, r, y = (matrix(gen, 9, 256, shift=1 if i == which else 0) for i in range(3))
    check(x, 0.2, ctx.gg_dropout(x, 0.2, 1, residual=r, out=y, seed=SEED)["y"], 1, residual=r)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("cols", [256, 77])
def test_in_place(ctx, cols, dtype):
    gen = torch.Generator(device="cuda").manual_seed(cols)
    x, r = (matrix(gen, 33, cols, dtype=getattr(torch, dtype)) for _ in range(2))
    want = ctx.gg_dropout(x, 0.4, 9, residual=r, seed=SEED)["y"].clone()
    for target in (0, 1):
        a, b = x.clone(), r.clone()
        assert torch.equal(ctx.gg_dropout(a, 0.4, 9, residual=b, out=(a, b)[target], seed=SEED)["y"], want)


def test_the_ends_of_p(ctx):
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = matrix(gen, 40, 333)
    assert torch.equal(ctx.gg_dropout(x, 0.0, 3)["y"], x)
    assert torch.equal(ctx.gg_dropout(x, 2.0 ** -18, 3)["y"], x)                 # rounds to 0
    check(x, 1.0 - 2.0 ** -16, ctx.gg_dropout(x, 1.0 - 2.0 ** -16, 3, seed=SEED)["y"], 3)


def test_what_is_dropped_does_not_matter(ctx):
    gen = torch.Generator(device="cuda").manual_seed(2)
    x, r = matrix(gen, 20, 128, dtype=torch.float32), matrix(gen, 20, 128, dtype=torch.float32)
    clean = ctx.gg_dropout(x, 0.5, 1, residual=r, seed=SEED)["y"].clone()
    dropped = torch.from_numpy(o.dropout_bits(20, 128, 1, 0, SEED) < 32768).cuda()
    for bad in (float("nan"), float("inf"), -float("inf")):
        y = ctx.gg_dropout(torch.where(dropped, bad, x), 0.5, 1, residual=r, seed=SEED)["y"]
        assert torch.equal(y, clean)
    assert torch.isnan(ctx.gg_dropout(torch.where(dropped, x, float("nan")), 0.5, 1, seed=SEED)["y"])[~dropped].all()


def test_the_gradient_is_the_same_call(ctx):
    gen = torch.Generator(device="cuda").manual_seed(3)
    x, dy = matrix(gen, 50, 100, dtype=torch.float32), matrix(gen, 50, 100, dtype=torch.float32)
    y = ctx.gg_dropout(x, 0.25, 6, seed=1, tensor_id=2)["y"]
    dx = ctx.gg_dropout(dy, 0.25, 6, seed=1, tensor_id=2)["y"]
    # y is linear in x: <dy, y(x)> = <dx, x>, term by term
    assert torch.allclose(dy.double() * y.double(), dx.double() * x.double(), rtol=1e-6, atol=1e-12)


def test_steps_tensors_and_seeds_draw_different_masks(ctx):
    x = torch.ones(64, 512, device="cuda")
    masks = [ctx.gg_dropout(x, 0.5, t, seed=s, tensor_id=i)["y"].clone() for t, s, i in ((1, 0, 0), (2, 0, 0), (1, 1, 0), (1, 0, 1), (1, 2 ** 32, 0))]
    for i, a in enumerate(masks):
        for b in masks[:i]:
            share = ((a == 0) == (b == 0)).double().mean().item()
            assert abs(share - 0.5) <= 5 * 0.5 / (64 * 512) ** 0.5


def test_a_graph_that_advances_its_step(ctx):
    gen = torch.Generator(device="cuda").manual_seed(4)
    x = matrix(gen, 30, 200)
    t_dev = torch.zeros(1, dtype=torch.int64, device="cuda")
    drop = ctx.make_dropout(x, 0.3, seed=SEED, tensor_id=4, t_dev=t_dev)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        drop(10)
        t_dev.add_(1)
    for i in range(3):
        graph.replay()
        torch.cuda.synchronize()
        check(x, 0.3, drop.outputs["y"], 10 + i, 4)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y = ctx.gg_dropout(x, 0.3, 77, seed=SEED)["y"]
    side.synchronize()
    check(x, 0.3, y, 77)


@pytest.mark.parametrize("rows,cols", [(1, 2 ** 31 + 4111), (2 ** 16 + 3, 2 ** 15 + 24)])
def test_positions_past_32_bits(ctx, rows, cols):
    x = torch.ones((rows, cols), dtype=torch.bfloat16, device="cuda")
    y = ctx.gg_dropout(x, 0.5, 1, out=x, seed=SEED)["y"]
    if rows == 1:
        tail = 4111 + 8 * 1000
        first = cols - tail - (cols - tail) % 8
        groups = np.arange(first // 8, (cols + 7) // 8, dtype=np.uint64)
        from oracle.train_oracle import philox4x32_10
        same = np.zeros_like(groups)
        w = philox4x32_10((groups & np.uint64(0xFFFFFFFF), groups >> np.uint64(32), same + np.uint64(1), same), (SEED & 0xFFFFFFFF, SEED >> 32))
        bits = np.stack([h for v in w for h in (v & 0xFFFF, v >> 16)], axis=1).reshape(-1)[:cols - first]
        assert np.array_equal(y[0, first:].float().cpu().numpy(), np.where(bits >= 32768, 2.0, 0.0))
    else:
        bits = o.dropout_bits(3, cols, 1, 0, SEED, first=rows - 3)
        assert np.array_equal(y[-3:].float().cpu().numpy(), np.where(bits >= 32768, 2.0, 0.0))


def test_refusals(ctx):
    from paper_2506_00486_b200 import GGError
    x = torch.ones(4, 8, device="cuda")
    before = ctx.launch_count
    for p in (-0.1, 1.0, 1.5, float("nan"), 1.0 - 2.0 ** -18):
        with pytest.raises(GGError) as e:
            ctx.gg_dropout(x, p)
        assert e.value.status == 1
    with pytest.raises(TypeError):
        ctx.gg_dropout(x.half(), 0.1)
    for kw in (dict(residual=x[:2]), dict(residual=x.bfloat16()), dict(out=x[:, :4]), dict(t_dev=torch.zeros(1, device="cuda"))):
        with pytest.raises(ValueError):
            ctx.gg_dropout(x, 0.1, **kw)
    with pytest.raises(ValueError):
        ctx.gg_dropout(x[0], 0.1)
    run = ctx.make_dropout(x, 0.1)
    for field, value, status in (("dtype", 7, 2), ("x_ld", 3, 1), ("x", None, 1), ("y", None, 1), ("rows", -1, 1), ("x", x.data_ptr() + 2, 3), ("t_dev", x.data_ptr() + 4, 3)):
        keep = getattr(run.args, field)
        setattr(run.args, field, value)
        with pytest.raises(GGError) as e:
            run()
        assert e.value.status == status, field
        setattr(run.args, field, keep)
    assert ctx.gg_dropout(x[:0], 0.1)["y"].shape == (0, 8)
    assert ctx.launch_count == before
