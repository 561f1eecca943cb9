"""What a product kernel does when one of its waits runs out: the call ends, the next one reports it, and the context computes as
before.  Every form of the kernel, because the CTAs of a pair, the halves of a tile and the ends wait for different things.

The copies' barriers are made to expect bytes that never come, so that every wait of the kernel runs out; nothing faults, and the kernel
waits for what it has started before it ends."""
import pytest
import torch

from product_forms import gated_forms, loss_forms
from product_util import matrix

pytestmark = pytest.mark.gpu

# (form of the loss, of its logits' gradient, of dw, of dh) of each shape; together with the gated block's below, every kernel that there is
LOSS = [(70, 200, 600, dict(lse=(1, 1, 8, False))),
        (174, 2327, 2857, dict(lse=(2, 1, 8, False), d=(2, 1, 8, False), dh=(2, 1, 8, True))),
        (9530, 2, 70, dict(lse=(1, 1, 16, False), dw=(1, 1, 8, True))),
        (145, 1, 4948, dict(d=(1, 1, 16, False))),
        (130, 249, 51949, dict(lse=(2, 1, 16, False))),
        (193, 453, 20289, dict(d=(2, 1, 16, False), dw=(2, 1, 16, False))),
        (2319, 2479, 325, dict(dh=(2, 2, 8, False))),
        (317, 3219, 2, dict(dh=(1, 1, 16, False))),
        (33000, 40, 9000, dict(lse=(1, 1, 16, False), dh=(2, 2, 8, False), pieces=2))]
GATED = [(70, 200, 300, dict(h=(1, 1, 8, False))),
         (189, 2272, 1236, dict(h=(2, 1, 8, False), dx=(2, 1, 8, True))),
         (1, 2481, 139, dict(dw=(1, 1, 16, False))),
         (400, 2503, 977, dict(dw=(2, 2, 8, False))),
         (4005, 3142, 71, dict(dx=(2, 1, 16, False)))]


def stuck(ctx, on):
    from paper_2506_00486_b200.binding import HOOK_EXTRA_ARRIVALS, HOOK_WAIT_CAP
    ctx.gg_test_hook(HOOK_EXTRA_ARRIVALS, int(on))
    ctx.gg_test_hook(HOOK_WAIT_CAP, 256 if on else 1 << 18)


def same(a, b):
    return all(torch.equal(a[k], b[k]) for k in b if b[k] is not None)


def check(runs):
    """runs: (entry, arguments, keywords) of calls that are stuck one by one, and compared before and after."""
    from paper_2506_00486_b200 import Context, GGError
    mine = Context(0)
    want = [getattr(mine, name)(*args, **kw) for name, args, kw in runs]
    for name, args, kw in runs:
        stuck(mine, True)
        getattr(mine, name)(*args, **kw)
        torch.cuda.synchronize()
        stuck(mine, False)
        with pytest.raises(GGError, match="ran out"):
            getattr(mine, name)(*args, **kw)
        for (again, more, kws), w in zip(runs, want):
            assert same(getattr(mine, again)(*more, **kws), w)
        torch.cuda.synchronize()
    mine.close()


@pytest.mark.parametrize("rows,width,vocab,forms", LOSS)
def test_loss_and_gradient(rows, width, vocab, forms):
    from paper_2506_00486_b200 import Context
    assert forms.items() <= loss_forms(rows, width, vocab).items()
    gen = torch.Generator(device="cuda").manual_seed(rows)
    h, w = matrix(gen, rows, width), matrix(gen, vocab, width, scale=2.0 / width ** 0.5)
    target = torch.randint(0, vocab, (rows,), generator=gen, device="cuda")
    dloss = torch.full((rows,), 1.0 / rows, device="cuda")
    first = Context(0)
    lse = first.gg_cross_entropy(h, w, target)["lse"]
    torch.cuda.synchronize()
    first.close()
    check([("gg_cross_entropy", (h, w, target), {}), ("gg_cross_entropy_grad", (dloss, h, w, target, lse), {}),
           ("gg_cross_entropy_grad", (dloss, h, w, target, lse), dict(want_dw=False)), ("gg_cross_entropy_grad", (dloss, h, w, target, lse), dict(want_dh=False))])


@pytest.mark.parametrize("rows,width,hidden,forms", GATED)
def test_gated_block_and_gradient(rows, width, hidden, forms):
    assert forms.items() <= gated_forms(rows, width, hidden).items()
    gen = torch.Generator(device="cuda").manual_seed(rows)
    x, dh = matrix(gen, rows, width), matrix(gen, rows, hidden, scale=0.1)
    wg, wu = (matrix(gen, hidden, width, scale=1.5 / width ** 0.5) for _ in range(2))
    gate, up = matrix(gen, rows, hidden), matrix(gen, rows, hidden)
    args = (dh, x, wg, wu, gate, up)
    runs = [("gg_gated_linear_grad", args, {}), ("gg_gated_linear_grad", args, dict(want_dx=False)), ("gg_gated_linear_grad", args, dict(want_dweight=False))]
    check(([("gg_gated_linear", (x, wg, wu), dict(keep=True))] if rows > 1 else []) + runs)


def small_problem():
    gen = torch.Generator(device="cuda").manual_seed(1)
    return matrix(gen, 200, 136), *(matrix(gen, 300, 136, scale=0.1) for _ in range(2))


def test_it_can_be_asked_for():
    from paper_2506_00486_b200 import Context, GGError
    mine, args = Context(0), small_problem()
    want = mine.gg_gated_linear(*args, keep=True)
    torch.cuda.synchronize()
    mine.gg_product_status()
    stuck(mine, True)
    mine.gg_gated_linear(*args, keep=True)
    torch.cuda.synchronize()
    stuck(mine, False)
    with pytest.raises(GGError, match="ran out") as e:
        mine.gg_product_status()
    assert e.value.status == 6
    mine.gg_product_status()                # (told once)
    assert same(mine.gg_gated_linear(*args, keep=True), want)
    mine.close()


def test_replays_of_a_graph_can_be_asked_about():
    from paper_2506_00486_b200 import Context, GGError
    mine, args = Context(0), small_problem()
    run = mine.make_gated_linear(*args)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    stuck(mine, True)
    with torch.cuda.graph(graph):
        run()
    stuck(mine, False)
    mine.gg_product_status()                # (captured, not run)
    for _ in range(2):
        graph.replay()
        torch.cuda.synchronize()
        with pytest.raises(GGError, match="ran out"):
            mine.gg_product_status()
    mine.gg_product_status()
    del graph
    mine.close()
