"""The AdamW step over many tensors, with states in 32 and in 8 bits, and the gradient norm, against the 64-bit forms.

Tolerances.  u = 2^-24.  m and v are two products and a sum of fp32 factors that are rounded themselves: off by at
most 4 u of the sum of their magnitudes.  The update divides them with a root and a division: 12 u of its own magnitude
on top.  bf16 weights are one of the two neighbours of the exact value; the 8-bit codes are the 64-bit ones, except
where the value plus its noise lies within 5e-5 of a code's width of the next code (8 u relative to a position of at
most 127 codes), where either is right."""
import numpy as np
import pytest
import torch

from oracle import train_oracle as o

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
SEED = 0x1234567890


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
    return t.double().cpu().numpy()


def tensors(gen, lens, dtype, scale, shift=0):
    out = []
    for n in lens:
        t = (torch.randn(n, generator=gen, device="cuda") * scale).to(dtype)
        out.append(torch.cat([t[:shift].clone() if n >= shift else torch.zeros(shift, dtype=dtype, device="cuda"), t])[shift:])
    return out


def check_weight(w_new, w_old, w64, step64, dtype):
    """w64: the exact new weight; step64: the magnitude of the update without decay."""
    tol = 4 * U * np.abs(w_old) + 16 * U * step64 + 1e-37
    if dtype == torch.float32:
        assert np.all(np.abs(w_new - w64) <= tol)
    else:
        spacing = 2.0 ** (np.floor(np.log2(np.maximum(np.abs(w64) + tol, 2.0 ** -126))) - 7)
        assert np.all(np.abs(w_new - w64) <= spacing + tol)


LENS = [[1], [7, 8, 9], [255, 256, 257, 0, 1], [4095, 4096, 4097], [896] * 20, [100003, 5, 70000], [3] * 600]


@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("g_dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("w_dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("lens", LENS, ids=lambda v: f"{len(v)}x{max(v)}")
def test_step_with_states_in_32_bits(ctx, lens, w_dtype, g_dtype, shift):
    w_dtype, g_dtype = getattr(torch, w_dtype), getattr(torch, g_dtype)
    gen = torch.Generator(device="cuda").manual_seed(sum(lens))
    w, g = tensors(gen, lens, w_dtype, 0.02, shift), tensors(gen, lens, g_dtype, 1e-3, shift)
    m, v = tensors(gen, lens, torch.float32, 3e-4, shift), [t.square() for t in tensors(gen, lens, torch.float32, 1e-3)]
    copy = [torch.full((n,), 9.0, dtype=torch.bfloat16, device="cuda") for n in lens]
    decay = torch.rand(len(lens), generator=gen, device="cuda") * 0.2
    old = [[host(t) for t in ts] for ts in (w, g, m, v)]
    ctx.gg_adamw_step(w, g, m, v, t=17, lr=1e-3, w_copy=copy, weight_decay=decay, seed=SEED)
    for i, n in enumerate(lens):
        w0, g0, m0, v0 = (ts[i] for ts in old)
        w1, m1, v1 = o.adamw(w0, g0, m0, v0, 17, 1e-3, decay=float(decay[i]))
        m_mag, v_mag = 0.9 * np.abs(m0) + 0.1 * np.abs(g0), v1
        assert np.all(np.abs(host(m[i]) - m1) <= 4 * U * m_mag)
        assert np.all(np.abs(host(v[i]) - v1) <= 4 * U * v_mag)
        step = 1e-3 / (1 - 0.9 ** 17) * m_mag / (np.sqrt(v1 / (1 - 0.999 ** 17)) + 1e-8)
        check_weight(host(w[i]), w0, w1, step, w_dtype)
        assert np.all(np.abs(host(copy[i]) - w1) <= 2.0 ** -8 * np.abs(w1) + 16 * U * step + 1e-37)


def check_state8(codes, scales, x64, mag, noise, keep):
    """codes and scales against the 64-bit state x64, whose fp32 form may be 4 u of `mag` off."""
    want, scale, pos = o.quantise(x64, noise, keep)
    assert np.all(np.abs(scales - scale) <= 12 * U * scale + 1e-37)
    got = codes.astype(np.int64)
    # moving x64 by its tolerance moves its position by at most this many codes (a binade has 8 of them; at 0, 512 a unit)
    safe = np.maximum(np.abs(x64), 1e-300)
    near = 5e-5 + 16.0 * (16 * U * mag / safe)
    off = np.abs((got & 127) - (want.astype(np.int64) & 127))
    edge = np.abs(pos - np.round(pos)) <= near
    assert np.all((off == 0) | ((off == 1) & edge)), (off.max(), np.flatnonzero((off > 0) & ~edge)[:5])
    # signs, where there is one to see
    clear = (np.abs(x64) > 16 * U * mag)
    assert np.array_equal((got >> 7)[clear], np.signbit(x64).astype(np.int64)[clear])


@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("g_dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("w_dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("lens", LENS, ids=lambda v: f"{len(v)}x{max(v)}")
def test_step_with_states_in_8_bits(ctx, lens, w_dtype, g_dtype, shift):
    w_dtype, g_dtype = getattr(torch, w_dtype), getattr(torch, g_dtype)
    gen = torch.Generator(device="cuda").manual_seed(sum(lens))
    w, g = tensors(gen, lens, w_dtype, 0.02, shift), tensors(gen, lens, g_dtype, 1e-3, shift)
    for t in g:      # a wide range within a block, zeros among it
        t.mul_(torch.exp2(-20.0 * torch.rand(t.numel(), generator=gen, device="cuda")).to(g_dtype))
        t[::13] = 0.0
    st = ctx.adamw_state(w, bits=8)
    if shift:
        st["m"], st["v"] = ([torch.cat([t[:1], t])[1:] if t.numel() else t for t in ts] for ts in (st["m"], st["v"]))
    state = [(np.zeros(n), np.zeros(n)) for n in lens]
    copy = [torch.zeros(n, dtype=torch.bfloat16, device="cuda") for n in lens]
    step = ctx.make_adamw_step(w, g, **st, w_copy=copy, weight_decay=0.1, seed=SEED)
    first = np.cumsum([0] + [-(-n // 256) for n in lens])
    for t in (1, 2, 3):
        w_old = [host(x) for x in w]
        step(t, 1e-3)
        scales = [s.double().cpu().numpy() for s in st["scales"]]
        for i, n in enumerate(lens):
            g0, (m0, r0) = host(g[i]), state[i]
            w1, m1, v1 = o.adamw(w_old[i], g0, m0, r0 * r0, t, 1e-3, decay=0.1)
            m_mag, r1 = 0.9 * np.abs(m0) + 0.1 * np.abs(g0), np.sqrt(v1)
            upd = 1e-3 / (1 - 0.9 ** t) * m_mag / (np.sqrt(v1 / (1 - 0.999 ** t)) + 1e-8)
            check_weight(host(w[i]), w_old[i], w1, 2 * upd, w_dtype)
            assert np.all(np.abs(host(copy[i]) - w1) <= 2.0 ** -8 * np.abs(w1) + 32 * U * upd + 1e-37)
            sl = slice(first[i], first[i + 1])
            mc, vc = (x[i].view(torch.uint8).cpu().numpy() for x in (st["m"], st["v"]))
            check_state8(mc, scales[0][sl], m1, m_mag, o.noise_for(n, t, i, SEED, 0), False)
            check_state8(vc, scales[1][sl], r1, r1, o.noise_for(n, t, i, SEED, 4), True)
            # the next step starts from what is stored
            state[i] = tuple(o.e4m3_value(c) * np.repeat(s[sl], 256)[:n] for c, s in ((mc, scales[0]), (vc, scales[1])))


def test_every_product_and_sum_of_the_states_is_rounded_by_itself(ctx):
    # the scales (and with them the codes) are those of the formula evaluated one fp32 operation at a time: no product is
    # fused with a sum, and the root rounds to nearest (but for about one value in a million: 1 of 512 blocks' largest may differ)
    n = 512 * 256
    gen = torch.Generator(device="cuda").manual_seed(12)
    g = tensors(gen, [n], torch.float32, 1e-3)
    w = [torch.zeros(n, device="cuda")]
    st = ctx.adamw_state(w, 8)
    step = ctx.make_adamw_step(w, g, **st, weight_decay=0.0, seed=1)
    step(1, 1e-3)
    m0, r0 = (c[0].float().view(-1, 256) * s[:, None] for c, s in zip((st["m"], st["v"]), st["scales"]))
    step(2, 1e-3)
    gb = g[0].view(-1, 256)
    m = (m0 * 0.9) + (gb * (1.0 - 0.9))
    r = torch.sqrt(((r0 * r0) * 0.999) + ((gb * gb) * (1.0 - 0.999)))
    for scale, value, off in zip(st["scales"], (m, r), (0, 1)):
        assert (scale != value.abs().amax(1) * (1.0 / 448.0)).sum().item() <= off


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("n", [256, 1000, 70001])
def test_alignment_changes_no_bit(ctx, bits, n):
    gen = torch.Generator(device="cuda").manual_seed(n)
    g = tensors(gen, [n], torch.float32, 1e-3)[0]
    w0 = tensors(gen, [n], torch.float32, 0.02)[0]
    results = []
    for shift in (0, 1):
        def place(t):
            return [torch.cat([t[:1], t])[1:] if shift else t.clone()]

        w = place(w0.clone())
        st = ctx.adamw_state(w, bits)
        st["m"], st["v"] = place(st["m"][0]), place(st["v"][0])
        step = ctx.make_adamw_step(w, place(g), **st, seed=2)
        for t in (1, 2, 3):
            step(t, 1e-3)
        results.append([w[0], st["m"][0], st["v"][0], *st.get("scales", ())])
    for a, b in zip(*results):
        assert torch.equal(a.contiguous().view(torch.uint8), b.clone().view(torch.uint8))


def test_bf16_weights_are_rounded_by_the_stated_noise(ctx):
    n = 5000
    gen = torch.Generator(device="cuda").manual_seed(1)
    w, g = tensors(gen, [n], torch.bfloat16, 0.02), tensors(gen, [n], torch.float32, 1.0)
    st = ctx.adamw_state(w)
    w0, g0 = host(w[0]), host(g[0])
    ctx.gg_adamw_step(w, g, **st, t=1, lr=1e-5, weight_decay=0.0, seed=SEED)
    w1, _, _ = o.adamw(w0, g0, np.zeros(n), np.zeros(n), 1, 1e-5)
    spacing = 2.0 ** (np.floor(np.log2(np.abs(w1))) - 7)
    pos = np.abs(w1) / spacing + o.noise_for(n, 1, 0, SEED, 2) / 65536.0
    want = np.copysign(np.floor(pos) * spacing, w1)
    # an update of 1e-5 in fp32 next to a weight of 0.02: the position is right to 256 codes times a few u
    edge = np.abs(pos - np.round(pos)) < 256 * 8 * U
    assert np.all((host(w[0]) == want) | edge) and edge.mean() < 1e-2
    # (the updates are a fifth of the spacing at most: to nearest, hardly a weight would have moved)
    assert (host(w[0]) != w0).mean() > 0.05


def test_states_in_8_bits_follow_a_decay_of_less_than_a_code(ctx):
    # gradients of zero: r falls by sqrt(0.999) a step, 1/125 of a code; rounding to nearest would keep it for ever.  A step's rounding
    # has a relative deviation of at most sqrt(p (1 - p)) / 8 with p = 0.008, so after 500 steps the mean of 65,280 values is good to
    # 0.0112 sqrt(500) / sqrt(65280) = 0.001 (one deviation)
    n = 65536
    w = [torch.ones(n, device="cuda")]
    g = [torch.zeros(n, device="cuda")]
    st = ctx.adamw_state(w, bits=8)
    st["v"][0].copy_((torch.rand(n, device="cuda") * 250 + 130).to(torch.float8_e4m3fn))
    st["v"][0][::256] = torch.full((n // 256,), 448.0, device="cuda").to(torch.float8_e4m3fn)
    st["scales"][1].fill_(1e-3)
    start = st["v"][0].float().double().cpu().numpy() * 1e-3
    step = ctx.make_adamw_step(w, g, **st, weight_decay=0.0, seed=3)
    for t in range(1, 501):
        step(t, 0.0)
    end = st["v"][0].float().double().cpu().numpy() * np.repeat(st["scales"][1].double().cpu().numpy(), 256)
    inner = np.arange(n) % 256 != 0
    assert abs(end[inner].mean() / start[inner].mean() / 0.999 ** 250 - 1) < 5e-3
    assert np.allclose(end[~inner], start[~inner] * 0.999 ** 250, rtol=1e-4)


def test_noise_differs_by_seed_and_tensor(ctx):
    n = 4096
    g = [torch.full((n,), 1.0, device="cuda")] * 2

    def codes(t, seed):
        w = [torch.full((n,), 0.37, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        st = ctx.adamw_state(w)
        ctx.gg_adamw_step(w, g, **st, t=t, lr=1e-4, weight_decay=0.0, seed=seed)
        return torch.stack(w)

    a = codes(1, 5)
    assert torch.equal(a, codes(1, 5))
    assert not torch.equal(a[0], a[1]) and not torch.equal(a, codes(1, 6)) and not torch.equal(a, codes(1, 5 + (1 << 32)))


@pytest.mark.parametrize("bits", [32, 8])
def test_zero_and_tiny_gradients(ctx, bits):
    n = 700
    w = [torch.ones(n, device="cuda")]
    g = [torch.zeros(n, device="cuda")]
    g[0][256:512] = 1e-38      # m and sqrt(v) of this block stay below 2^-110
    st = ctx.adamw_state(w, bits)
    ctx.gg_adamw_step(w, g, **st, t=1, lr=1e-3, weight_decay=0.0)
    assert torch.equal(w[0], torch.ones(n, device="cuda"))
    if bits == 8:
        for t in (st["m"][0], st["v"][0], *st["scales"]):
            assert not t.float().any()


@pytest.mark.parametrize("bits", [32, 8])
def test_infinities_and_nan_reach_their_own_element_only(ctx, bits):
    n = 1000
    gen = torch.Generator(device="cuda").manual_seed(8)
    g = tensors(gen, [n], torch.float32, 1e-3)
    bad = torch.tensor([3, 300, 301, 999], device="cuda")
    values = torch.tensor([float("inf"), float("nan"), -float("inf"), 3e30], device="cuda")      # (the square of the last overflows)

    def after(grad):
        w = [torch.ones(n, device="cuda")]
        st = ctx.adamw_state(w, bits)
        ctx.gg_adamw_step(w, grad, **st, t=1, lr=1e-3)
        return w[0], st["m"][0].float(), st["v"][0].float()

    g0 = g[0].clone()
    g0[bad] = 0.0
    clean = after([g0])
    g1 = g[0].clone()
    g1[bad] = values
    got = after([g1])
    keep = torch.ones(n, dtype=torch.bool, device="cuda")
    keep[bad] = False
    if bits == 8:      # 3e29 is a finite m, and takes the scale of its block: compare the other blocks' m
        keep_m = keep.clone()
        keep_m[768:] = False
    else:
        keep_m = keep
    assert torch.equal(got[0][keep], clean[0][keep]) and torch.equal(got[1][keep_m], clean[1][keep_m]) and torch.equal(got[2][keep], clean[2][keep])
    assert not torch.isfinite(got[1][bad[:3]]).any() and not torch.isfinite(got[2][bad]).any()
    assert torch.isnan(got[0][bad[:3]]).all()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_a_scale_that_is_not_finite_skips_the_step(ctx, bits, value):
    w = [torch.randn(3000, device="cuda").bfloat16(), torch.randn(5, device="cuda").bfloat16()]
    g = [torch.randn_like(t) for t in w]
    copy = [torch.full_like(t, 4.0) for t in w]
    st = ctx.adamw_state(w, bits)
    flat = [*w, *copy, *st["m"], *st["v"], *st.get("scales", ())]
    old = [t.clone() for t in flat]
    ctx.gg_adamw_step(w, g, **st, t=1, lr=1e-2, w_copy=copy, grad_scale=torch.tensor([value], device="cuda"))
    for a, b in zip(flat, old):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("lens", [[1], [0], [5, 0, 16384, 16385], [100000] * 7, [3] * 2000])
def test_gradient_norm(ctx, lens, dtype):
    dtype = getattr(torch, dtype)
    gen = torch.Generator(device="cuda").manual_seed(len(lens))
    g = tensors(gen, lens, dtype, 0.3)
    want = o.grad_norm([host(t) for t in g])
    out = ctx.gg_grad_norm(g, max_norm=0.5)
    # squares and short sums in fp32, the rest in fp64: the bound of the library's moments, 1e-6 of the sum
    assert abs(out["norm"].item() - want) <= 1e-6 * want
    scale = min(1.0, 0.5 / want) if want else 1.0
    assert abs(out["scale"].item() - scale) <= 1e-6 * scale + U
    free = ctx.gg_grad_norm(g)
    assert free["scale"].item() == 1.0 and free["norm"].item() == out["norm"].item()


def test_gradient_norm_of_extremes(ctx):
    big = [torch.full((1000,), 1e30, device="cuda"), torch.full((70000,), 1e-30, device="cuda")]
    assert ctx.gg_grad_norm(big)["norm"].item() == pytest.approx(1e30 * 1000 ** 0.5, rel=1e-6)
    assert ctx.gg_grad_norm(big[1:])["norm"].item() == pytest.approx(1e-30 * 70000 ** 0.5, rel=1e-6)
    assert ctx.gg_grad_norm([])["norm"].item() == 0.0
    for v in (float("inf"), float("nan")):
        big[1][69999] = v
        out = ctx.gg_grad_norm(big, 1.0)
        assert torch.isnan(out["norm"]).all() and torch.isnan(out["scale"]).all()


@pytest.mark.parametrize("bits", [32, 8])
def test_clipped_step_is_the_step_of_the_scaled_gradient(ctx, bits):
    gen = torch.Generator(device="cuda").manual_seed(6)
    lens = [1000, 77, 40000]
    g = tensors(gen, lens, torch.float32, 1.0)
    results = []
    scale = ctx.gg_grad_norm(g, 0.25)["scale"]
    for kw in (dict(max_norm=0.25), dict(grad_scale=scale)):
        w = [torch.ones(n, device="cuda") for n in lens]
        st = ctx.adamw_state(w, bits)
        ctx.gg_adamw_step(w, g, **st, t=1, lr=1e-2, **kw)
        results.append([*w, *st["m"], *st["v"]])
    for a, b in zip(*results):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    want = o.grad_norm([host(t) for t in g])
    if bits == 32:
        assert np.allclose(host(results[0][3]), 0.1 * host(g[0]) * 0.25 / want, rtol=1e-5)


def test_graph_and_other_stream(ctx):
    gen = torch.Generator(device="cuda").manual_seed(3)
    lens = [5000, 896, 33]
    g = tensors(gen, lens, torch.bfloat16, 1e-2)

    def fresh():
        w = [torch.full((n,), 0.5, dtype=torch.bfloat16, device="cuda") for n in lens]
        st = ctx.adamw_state(w, 8)
        return w, st, ctx.make_adamw_step(w, g, **st, max_norm=1.0, seed=9)

    w0, _, plain = fresh()
    plain(1, 1e-2)
    w1, _, other = fresh()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other(1, 1e-2)
    side.synchronize()
    w2, _, captured = fresh()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured(1, 1e-2)
    graph.replay()
    torch.cuda.synchronize()
    for a, b, c in zip(w0, w1, w2):
        assert torch.equal(a, b) and torch.equal(a, c)


def test_refusals(ctx):
    from paper_2506_00486_b200 import GGError, Segments, binding
    w, g = [torch.ones(300, device="cuda")], [torch.ones(300, device="cuda")]
    st, st8 = ctx.adamw_state(w), ctx.adamw_state(w, 8)
    before = ctx.launch_count
    one = torch.ones(1, device="cuda")
    with pytest.raises(ValueError):
        ctx.adamw_state(w, 4)
    for kw in (dict(g=[g[0][:299]]), dict(m=[st["m"][0][:299]]), dict(w_copy=[torch.zeros(7, dtype=torch.bfloat16, device="cuda")]),
               dict(weight_decay=torch.ones(2, device="cuda")), dict(weight_decay=one.double()), dict(grad_scale=torch.ones(2, device="cuda")),
               dict(grad_scale=one, max_norm=1.0)):
        with pytest.raises(ValueError):
            ctx.make_adamw_step(**{**dict(w=w, g=g, **st), **kw})
    for kw in (dict(m=[st["m"][0].double()]), dict(w_copy=[w[0]]), dict(scales=st8["scales"]), dict(w=[w[0].half()])):
        with pytest.raises(TypeError):
            ctx.make_adamw_step(**{**dict(w=w, g=g, **st), **kw})
    with pytest.raises(ValueError):
        ctx.make_adamw_step(w, g, st8["m"], st8["v"], scales=(one, one))
    for kw in (dict(beta1=1.0), dict(beta2=-0.1), dict(eps=-1.0), dict(eps=float("nan")), dict(weight_decay=float("inf")), dict(t=0),
               dict(lr=-1.0), dict(lr=float("nan")), dict(lr=float("inf"))):
        with pytest.raises(GGError) as e:
            ctx.gg_adamw_step(w, g, **{**dict(t=1, lr=1e-3), **st, **kw})
        assert e.value.status == 1, kw
    for bad in (0.0, -1.0, float("nan")):
        with pytest.raises(GGError):
            ctx.gg_grad_norm(g, bad)
    L, P = binding.lib(), binding.ctypes.byref
    step = ctx.make_adamw_step(w, g, **st)
    step.args.t, step.args.lr = 1, 1e-3
    odd = Segments([torch.zeros(304, dtype=torch.uint8, device="cuda")[1:301]])

    def status(**change):
        a = type(step.args).from_buffer_copy(step.args)
        for k, v in change.items():
            setattr(a, k, v)
        return L.gg_adamw_step(ctx._h, P(a), None)

    p = w[0].data_ptr()
    for change, want in ((dict(n_seg=-1), 1), (dict(w=None), 1), (dict(g=None), 1), (dict(m=None), 1), (dict(v=None), 1), (dict(state_bits=16), 1),
                         (dict(w_dtype=3), 2), (dict(g_dtype=-1), 2), (dict(g=odd.ptr), 3), (dict(m=odd.ptr), 3), (dict(v=odd.ptr), 3),
                         (dict(w_copy=odd.ptr), 3), (dict(decay=p + 2), 3), (dict(grad_scale=p + 1), 3), (dict(state_bits=8), 1),
                         (dict(state_bits=8, m_scale=p, v_scale=p + 3), 3)):
        assert status(**change) == want, change
    # more blocks than a scale can be numbered by: nothing is read, the check comes first
    huge = np.zeros(1, dtype=binding._SEG_DTYPE)
    huge["ptr"], huge["len"] = p, 1 << 40
    at = huge.ctypes.data
    assert status(w=at, g=at, m=at, v=at) == 4
    huge["len"] = -5
    assert status(w=at, g=at, m=at, v=at) == 1
    assert L.gg_adamw_step(None, P(step.args), None) == 1 and L.gg_adamw_step(ctx._h, None, None) == 1
    assert L.gg_grad_norm(None, None, 0, 0, 1.0, None, None, None) == 1
    assert L.gg_grad_norm(ctx._h, step._keep[1].ptr, 1, 0, 1.0, p + 4, None, None) == 3
    # nothing was enqueued, and nothing to do is no error
    assert ctx.launch_count == before and torch.equal(w[0], torch.ones(300, device="cuda"))
    ctx.gg_adamw_step([], [], [], [], t=1, lr=1e-3)
    empty = [torch.empty(0, device="cuda")]
    ctx.gg_adamw_step(empty, empty, empty, empty, t=1, lr=1e-3)
    assert ctx.launch_count == before
