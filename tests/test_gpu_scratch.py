"""Scratch of a context whose first use is on another stream or inside a stream capture."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture
def ctx():
    import __graft_entry__ as entry
    entry.build()
    from paper_2506_00486_b200 import Context
    c = Context(0, guard=True)
    yield c
    c.check_guards()
    c.close()


def gradients(lens, seed=1):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.randn(n, generator=gen, device="cuda") for n in lens]


def norm_of(g):
    return float(sum(t.double().square().sum() for t in g).sqrt())


def test_the_first_gradient_norm_on_another_stream_behind_a_busy_default_stream(ctx):
    g = gradients([5, 20000, 70001])
    want = norm_of(g)
    ctx.gg_fit(g)                       # the plan is known: the norm itself uploads nothing that could wait
    out = dict(norm=torch.full((1,), -1.0, dtype=torch.float64, device="cuda"), scale=torch.full((1,), -1.0, device="cuda"))
    busy = torch.randn(4096, 4096, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(30):
        busy = torch.tanh(busy @ busy)
    with torch.cuda.stream(side):
        ctx.gg_grad_norm(g, 1.0, out)
        first = {k: t.clone() for k, t in out.items()}
        ctx.gg_grad_norm(g, 1.0, out)
    side.synchronize()
    torch.cuda.synchronize()
    for got in (first, out):
        assert abs(got["norm"].item() - want) <= 1e-6 * want and abs(got["scale"].item() * want - 1.0) <= 2e-6


def test_the_first_gradient_norm_inside_a_capture(ctx):
    g = gradients([300, 40000])
    ctx.gg_fit(g)
    out = dict(norm=torch.zeros(1, dtype=torch.float64, device="cuda"), scale=torch.zeros(1, device="cuda"))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.gg_grad_norm(g, 1.0, out)
    for factor in (1.0, 3.0):
        for t in g:
            t.mul_(factor)
        graph.replay()
        torch.cuda.synchronize()
        want = norm_of(g)
        assert abs(out["norm"].item() - want) <= 1e-6 * want


def test_the_first_fused_pass_on_another_stream_behind_a_busy_default_stream(ctx):
    # the tables of the plan and the counters of the entropy step are set up by this very call
    from oracle import gg_oracle as o
    g = [t.mul_(0.02) for t in gradients([70001, 20000, 5])]
    step = torch.full((3,), 2.0 ** -10, device="cuda")
    grad = [torch.empty_like(t) for t in g]
    busy = torch.randn(4096, 4096, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(30):
        busy = torch.tanh(busy @ busy)
    with torch.cuda.stream(side):
        out = ctx.gg_fused(g, grad=grad, lam=1e-4, step=step)
    side.synchronize()
    torch.cuda.synchronize()
    for s, t in enumerate(g):
        x = t.cpu().numpy()
        beta, alpha, *_ = o.fit(x)
        assert abs(out["beta"][s].item() - beta) <= 1e-5 * beta and abs(out["alpha"][s].item() - alpha) <= 1e-5 * alpha
        hist, _ = o.quantise_hist(x, 2.0 ** -10)
        assert abs(o.entropy_bits(hist) - out["entropy_bits"][s].item()) <= 1e-9


def norm_gradient(ctx, rows, cols, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x, dy = (torch.randn((rows, cols), generator=gen, device="cuda") for _ in range(2))
    w = 1.0 + 0.1 * torch.randn(cols, generator=gen, device="cuda")
    out = ctx.gg_layer_norm(x, w)
    return ctx.make_layer_norm_grad(dy, x, out["mean"], out["rstd"], w)


def test_a_captured_gradient_outlives_a_larger_one(ctx):
    # the larger call needs more scratch for its sums; the graph still holds the smaller scratch
    small = norm_gradient(ctx, 2000, 64, 1)
    want = {k: t.clone() for k, t in small().items()}
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        small()
    large = [norm_gradient(ctx, 3000, cols, 2) for cols in (520, 1024, 4096)]
    for run in large:
        run()
    # whatever the driver hands out now must not be what the graph writes to
    other = [torch.full((1 << 18,), 3.0, device="cuda") for _ in range(64)]
    before = [{k: t.clone() for k, t in run().items()} for run in large]
    for t in small.outputs.values():
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(small.outputs[k], want[k]) for k in want)
    assert all((t == 3.0).all() for t in other)
    for run, old in zip(large, before):
        assert all(torch.equal(run()[k], old[k]) for k in old)


def test_sums_over_few_rows_need_no_scratch(ctx):
    # so the first call of a context may be a captured one
    run = norm_gradient(ctx, 20, 896, 3)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    graph.replay()
    torch.cuda.synchronize()
    got = {k: t.clone() for k, t in run.outputs.items()}
    run()
    assert all(torch.equal(run.outputs[k], got[k]) and got[k].any() for k in got)


def test_a_captured_call_keeps_its_plan(ctx):
    # afterwards come enough layouts to fill the context, and one layout at more addresses than it has plans for
    g = gradients([3000, 70001])
    w = [torch.ones_like(t) for t in g]
    st = ctx.adamw_state(w)
    step = ctx.make_adamw_step(w, g, **st, max_norm=1.0, weight_decay=0.0)
    step(1, 1e-3)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(2, 1e-3)
    others = [gradients([100 + i, 50], seed=i) for i in range(80)] + [gradients([3000, 70001], seed=100 + i) for i in range(20)]
    norms = [ctx.gg_grad_norm(t) for t in others]
    for t, out in zip(others, norms):
        assert abs(out["norm"].item() - norm_of(t)) <= 1e-6 * norm_of(t)
    for factor in (1.0, 5.0):
        for t in g:
            t.mul_(factor)
        graph.replay()
        torch.cuda.synchronize()
        want = norm_of(g)
        assert abs(step.outputs["norm"].item() - want) <= 1e-6 * want
        assert abs(step.outputs["scale"].item() * want - 1.0) <= 2e-6
    # the plans that no graph holds are still limited and recycled
    built, repointed = ctx.plan_stats
    for t in others[80:]:
        ctx.gg_grad_norm(t)
    again = ctx.plan_stats
    assert again[0] == built and again[1] > repointed


def test_captured_passes_outlive_larger_scratch(ctx):
    # the entropy step's and the channel-wise pass's scratch, outgrown by later calls
    gen = torch.Generator(device="cuda").manual_seed(7)
    segs = [t.mul_(0.02) for t in gradients([70001, 5000])]
    few = torch.zeros(2, dtype=torch.int32)
    fused = ctx.make_fused(segs, grad=[torch.empty_like(t) for t in segs], lam=1e-4, step=torch.full((2,), 2.0 ** -10, device="cuda"), hist_id=few, n_hist=1)
    matrix = 0.02 * torch.randn((300, 64), generator=gen, device="cuda")
    channels = ctx.make_fused_channels(matrix, grad=torch.empty_like(matrix), step=2.0 ** -10)
    # (the step among the results is the one that was passed in)
    want = [{k: t.clone() for k, t in run().items() if torch.is_tensor(t) and k != "step"} for run in (fused, channels)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fused()
        channels()
    many = [t.mul_(0.02) for t in gradients([3000] * 40, seed=3)]
    ctx.gg_fused(many, grad=[torch.empty_like(t) for t in many], lam=1e-4, step=torch.full((40,), 2.0 ** -10, device="cuda"))
    for cols in (700, 5000):
        wide = 0.02 * torch.randn((2000, cols), generator=gen, device="cuda")
        ctx.gg_fused_channels(wide, grad=torch.empty_like(wide), step=2.0 ** -10)
    other = [torch.full((1 << 16,), 3.0, device="cuda") for _ in range(64)]
    for run, old in zip((fused, channels), want):
        for k in old:
            run.outputs[k].zero_()
    graph.replay()
    torch.cuda.synchronize()
    for run, old in zip((fused, channels), want):
        for k in old:
            assert torch.equal(run.outputs[k], old[k]), k
    assert all((t == 3.0).all() for t in other)
