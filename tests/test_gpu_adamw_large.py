"""The AdamW step over so many elements that a warp steps several blocks in a row: its ring of operands wraps, its scales come
from and go to several lanes, full blocks and short ones share a run, and blocks with inf, nan or large values stand in the
middle of one.  Against the 64-bit forms, computed on the device.

Tolerances: as in test_gpu_adamw.py.  u = 2^-24.  m and v are off by at most 4 u of the sum of their magnitudes, the update by
12 u of its own magnitude on top.  Codes and bf16 weights are the floor of a 64-bit position plus the stated noise: any whole
number that this floor can be when the position moves by the error of the fp32 value (a weight that the update nearly cancels
has an error of more than its own spacing)."""
import numpy as np
import pytest
import torch

from oracle import train_oracle as o

U = 2.0 ** -24
SEED = 0x1234567890
BLOCK = 256


@pytest.fixture(scope="module")
def ctx():
    import __graft_entry__ as entry
    entry.build()
    from paper_2506_00486_b200 import Context
    c = Context(0, guard=True)
    yield c
    c.check_guards()
    c.close()


# ---------------------------------------------- the 64-bit forms of train_oracle.py, on any device
def noise_for(n, t, segment, seed, shift, device):
    """The 16 random bits that each of n elements takes."""
    mask = 0xFFFFFFFF
    j = torch.arange((n + 7) // 8, device=device)
    c = [j & mask, j >> 32, torch.full_like(j, t & mask), torch.full_like(j, segment)]
    k = [seed & mask, seed >> 32 & mask]
    for _ in range(10):
        lo = [(v * m & mask) for v, m in ((c[0], 0xD2511F53), (c[2], 0xCD9E8D57))]
        hi = [(((v >> 16) * m + ((v & 0xFFFF) * m >> 16)) >> 16) & mask for v, m in ((c[0], 0xD2511F53), (c[2], 0xCD9E8D57))]
        c = [hi[1] ^ c[1] ^ k[0], lo[1], hi[0] ^ c[3] ^ k[1], lo[0]]
        k = [(k[0] + 0x9E3779B9) & mask, (k[1] + 0xBB67AE85) & mask]
    u = torch.stack([h for v in c for h in (v & 0xFFFF, v >> 16)], dim=1)
    return torch.roll(u, -shift, 1).reshape(-1)[:n]


def e4m3_position(y):
    a = y.abs()
    e = (torch.frexp(a).exponent - 1).clamp_min(-6)
    return torch.where(a < 2.0 ** -6, a * 512.0, (e + 6) * 8.0 + torch.ldexp(a, 3 - e))


def quantise(x, noise, keep_above):
    """(codes without sign, scales, positions + noise): a value that is not finite is left out of its block's scale and is code 127;
    values above `keep_above` (if not None) are never code 0."""
    finite = torch.isfinite(x)
    x = torch.where(finite, x, 0.0)
    pad = -x.numel() % BLOCK
    top = torch.nn.functional.pad(x.abs(), (0, pad)).view(-1, BLOCK).amax(1)
    fits = top > 2.0 ** -110
    factor = torch.where(fits, 448.0 / torch.where(fits, top, 1.0), 0.0).repeat_interleave(BLOCK)[:x.numel()]
    pos = e4m3_position(x * factor) + (noise.double() + 0.5) / 65536.0
    code = pos.floor().clamp_max(126)
    if keep_above is not None:
        code = torch.where((x > keep_above) & (code == 0), 1.0, code)
    return torch.where(finite, code, 127.0), torch.where(fits, top / 448.0, 0.0), pos


def adamw(w, g, m, v, t, lr, decay, b1=0.9, b2=0.999, eps=1e-8):
    m = b1 * m + (1.0 - b1) * g
    v = b2 * v + (1.0 - b2) * g * g
    return w - lr * decay * w - lr * (m / (1.0 - b1 ** t)) / (torch.sqrt(v / (1.0 - b2 ** t)) + eps), m, v


def test_the_forms_on_a_device_are_those_of_the_oracle():
    rng = np.random.default_rng(0)
    n = 1000
    for shift in (0, 2, 4):
        assert np.array_equal(noise_for(n, 9, 3, SEED, shift, "cpu").numpy(), o.noise_for(n, 9, 3, SEED, shift))
    x = rng.normal(size=n) * np.exp2(-25.0 * rng.random(n))
    noise = o.noise_for(n, 9, 3, SEED, 0)
    for keep in (False, True):
        want, scale, pos = o.quantise(np.abs(x), noise, keep)
        code, s, p = quantise(torch.from_numpy(np.abs(x)), torch.from_numpy(noise), 0.0 if keep else None)
        assert np.array_equal(code.numpy(), want) and np.array_equal(s.numpy(), scale)
        assert np.allclose(p.numpy(), pos, rtol=1e-13, atol=0.0)
    a = [rng.normal(size=n) for _ in range(3)] + [rng.random(n)]
    for got, want in zip(adamw(*(torch.from_numpy(v) for v in a), 5, 1e-3, 0.1), o.adamw(*a, 5, 1e-3, decay=0.1)):
        assert np.allclose(got.numpy(), want, rtol=1e-14, atol=1e-16)


# ------------------------------------------------------------------ the checks
def holds(ok, what):
    assert ok.all(), (what, int((~ok).sum()), torch.nonzero(~ok)[:5].view(-1).tolist())


def check_weight(w_new, w_old, w64, step64, dtype, noise):
    tol = 4 * U * w_old.abs() + 16 * U * step64 + 1e-37
    bad = ~torch.isfinite(w64)
    holds(torch.isnan(w_new) == torch.isnan(w64), "nan in w")
    w_new, w64, tol = (torch.where(bad, 0.0, t) for t in (w_new, w64, tol))
    if dtype == torch.float32:
        holds((w_new - w64).abs() <= tol, "w")
        return
    spacing = torch.ldexp(torch.ones_like(w64), torch.frexp(w64.abs().clamp_min(2.0 ** -126)).exponent - 8)
    pos, err, got = w64.abs() / spacing + noise.double() / 65536.0, tol / spacing, w_new / torch.copysign(spacing, w64)
    holds((got >= (pos - err).floor()) & (got <= (pos + err).floor()), "w")
    assert ((pos - err).floor() == (pos + err).floor()).sum() >= 0.98 * pos.numel()


def check_state8(codes, scales, x64, mag, noise, keep_above):
    want, scale, pos = quantise(x64, noise, keep_above)
    assert ((scales - scale).abs() <= 12 * U * scale + 1e-37).all()
    got = codes.to(torch.float64) % 128
    near = 5e-5 + 16.0 * (16 * U * mag / x64.abs().clamp_min(1e-300))
    off = (got - want).abs()
    holds((off == 0) | ((off == 1) & ((pos - pos.round()).abs() <= near)), "codes")
    clear = torch.isfinite(x64) & (x64.abs() > 16 * U * mag)
    holds(((codes >= 128) == torch.signbit(x64)) | ~clear, "signs")


def place(values, dtype, shift):
    """Copies of the tensors in one buffer each, `shift` elements after its start."""
    out = []
    for t in values:
        flat = torch.zeros(t.numel() + shift, dtype=dtype, device="cuda")
        flat[shift:].copy_(t)
        out.append(flat[shift:])
    return out


# Elements in all, for runs of 2, 5 and 8 blocks a warp (32 with bf16 weights and 8-bit states for the largest): a run has
# blocks / (SMs * 64) of them.
def lengths(total):
    small = [896, 5, 257, 4096, 0, 1023]
    big = [total // 2 + 3, total // 3 + 8, total - total // 2 - total // 3 - 11]
    return [big[0], *small, big[1], *small, big[2]]


SPECIAL = {1: float("inf"), 2: float("nan"), 3: 1e6, 4: -float("inf"), 5: 3e9}


def gradients(gen, lens, dtype):
    """Values over a wide range, zeros among them; in the first tensor some blocks in the middle of runs with an inf, a nan or a large value."""
    out = []
    for n in lens:
        g = torch.randn(n, generator=gen, device="cuda") * 1e-3 * torch.exp2(-20.0 * torch.rand(n, generator=gen, device="cuda"))
        g[::13] = 0.0
        out.append(g)
    for k, value in SPECIAL.items():
        for at in (k * 10_000 * BLOCK + 77, k * 1001 * BLOCK + 255):
            if at < lens[0]:
                out[0][at] = value
    return [g.to(dtype) for g in out]


@pytest.mark.gpu
@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("w_dtype,g_dtype", [("float32", "float32"), ("float32", "bfloat16"), ("bfloat16", "bfloat16"), ("bfloat16", "float32")])
@pytest.mark.parametrize("total", [6_000_000, 13_000_000, 30_000_000])
def test_runs_of_blocks_with_states_in_32_bits(ctx, total, w_dtype, g_dtype, shift):
    w_dtype, g_dtype = getattr(torch, w_dtype), getattr(torch, g_dtype)
    lens = lengths(total)
    gen = torch.Generator(device="cuda").manual_seed(total)
    w = place([0.02 * torch.randn(n, generator=gen, device="cuda") for n in lens], w_dtype, shift)
    g = place(gradients(gen, lens, g_dtype), g_dtype, shift)
    m = place([3e-4 * torch.randn(n, generator=gen, device="cuda") for n in lens], torch.float32, shift)
    v = place([1e-6 * torch.rand(n, generator=gen, device="cuda") for n in lens], torch.float32, shift)
    copy = place([torch.zeros(n, device="cuda") for n in lens], torch.bfloat16, shift)
    old = [[t.double() for t in ts] for ts in (w, g, m, v)]
    decay = torch.rand(len(lens), generator=gen, device="cuda") * 0.2
    ctx.gg_adamw_step(w, g, m, v, t=17, lr=1e-3, w_copy=copy, weight_decay=decay, seed=SEED)
    for i, n in enumerate(lens):
        w0, g0, m0, v0 = (ts[i] for ts in old)
        w1, m1, v1 = adamw(w0, g0, m0, v0, 17, 1e-3, float(decay[i]))
        m_mag = 0.9 * m0.abs() + 0.1 * g0.abs()
        for got, want, mag, what in ((m[i], m1, m_mag, "m"), (v[i], v1, v1, "v")):
            same = torch.where(torch.isfinite(want), (got.double() - want).abs() <= 4 * U * mag, got.double() == want)
            holds(same | (torch.isnan(want) & torch.isnan(got)), what)
        step = 1e-3 / (1 - 0.9 ** 17) * m_mag / (torch.sqrt(v1 / (1 - 0.999 ** 17)) + 1e-8)
        check_weight(w[i].double(), w0, w1, step, w_dtype, noise_for(n, 17, i, SEED, 2, "cuda") if w_dtype == torch.bfloat16 else None)
        ok = (copy[i].double() - w1).abs() <= 2.0 ** -8 * w1.abs() + 16 * U * step + 1e-37
        holds(ok | (torch.isnan(w1) & torch.isnan(copy[i])), "copy")


@pytest.mark.gpu
@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("w_dtype,g_dtype,total", [("float32", "float32", 6_000_000), ("float32", "bfloat16", 13_000_000), ("float32", "float32", 30_000_000),
                                                   ("bfloat16", "float32", 6_000_000), ("bfloat16", "bfloat16", 30_000_000),
                                                   ("bfloat16", "bfloat16", 90_000_000)])
def test_runs_of_blocks_with_states_in_8_bits(ctx, total, w_dtype, g_dtype, shift):
    w_dtype, g_dtype = getattr(torch, w_dtype), getattr(torch, g_dtype)
    lens = lengths(total)
    gen = torch.Generator(device="cuda").manual_seed(total)
    w = place([0.02 * torch.randn(n, generator=gen, device="cuda") for n in lens], w_dtype, shift)
    clean, special = ([torch.randn(n, generator=gen, device="cuda") * 1e-3 for n in lens], gradients(gen, lens, g_dtype))
    g = place(clean, g_dtype, shift)
    st = ctx.adamw_state(w, bits=8)
    st["m"], st["v"] = (place([t.view(torch.uint8) for t in st[k]], torch.uint8, shift) for k in ("m", "v"))
    copy = place([torch.zeros(n, device="cuda") for n in lens], torch.bfloat16, shift)
    step = ctx.make_adamw_step(w, g, **st, w_copy=copy, weight_decay=0.1, seed=SEED)
    first = np.cumsum([0] + [-(-n // BLOCK) for n in lens])
    step(1, 1e-3)                      # a state with something in every block
    for t_old, t_new in zip(g, special):
        t_old.copy_(t_new)

    def states(i, n):
        sl = slice(first[i], first[i + 1])
        codes = [st[k][i].view(torch.float8_e4m3fn).double() for k in ("m", "v")]
        return [c * s[sl].double().repeat_interleave(BLOCK)[:n] for c, s in zip(codes, st["scales"])]

    w_old, old = [t.double() for t in w], [states(i, n) for i, n in enumerate(lens)]
    step(2, 1e-3)
    for i, n in enumerate(lens):
        if n == 0:
            continue
        g0, (m0, r0) = g[i].double(), old[i]
        w1, m1, v1 = adamw(w_old[i], g0, m0, r0 * r0, 2, 1e-3, 0.1)
        m_mag, r1 = 0.9 * m0.abs() + 0.1 * g0.abs(), torch.sqrt(v1)
        upd = 1e-3 / (1 - 0.9 ** 2) * m_mag / (torch.sqrt(v1 / (1 - 0.999 ** 2)) + 1e-8)
        check_weight(w[i].double(), w_old[i], w1, 2 * upd, w_dtype, noise_for(n, 2, i, SEED, 2, "cuda") if w_dtype == torch.bfloat16 else None)
        ok = (copy[i].double() - w1).abs() <= 2.0 ** -8 * w1.abs() + 32 * U * upd + 1e-37
        holds(ok | (torch.isnan(w1) & torch.isnan(copy[i])), "copy")
        sl = slice(first[i], first[i + 1])
        check_state8(st["m"][i], st["scales"][0][sl].double(), m1, m_mag, noise_for(n, 2, i, SEED, 0, "cuda"), None)
        check_state8(st["v"][i], st["scales"][1][sl].double(), r1, r1, noise_for(n, 2, i, SEED, 4, "cuda"), 2.0 ** -62)


@pytest.mark.gpu
@pytest.mark.parametrize("w_dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("bits", [32, 8])
def test_every_length_up_to_two_blocks_and_its_neighbours(ctx, bits, w_dtype):
    # every end of a tensor, at every place of a vector, with what lies behind it
    w_dtype = getattr(torch, w_dtype)
    lens = list(range(1, 521))
    room = 544      # (a multiple of 32 bytes for every type: each tensor starts at a vector boundary)
    gen = torch.Generator(device="cuda").manual_seed(4)
    g = 1e-3 * torch.randn((len(lens), room), generator=gen, device="cuda")
    w = (0.02 * torch.randn((len(lens), room), generator=gen, device="cuda")).to(w_dtype)
    state = torch.float32 if bits == 32 else torch.uint8
    m, v = (torch.zeros((len(lens), room), dtype=state, device="cuda") for _ in range(2))
    copy = torch.zeros((len(lens), room), dtype=torch.bfloat16, device="cuda")
    beyond = torch.arange(room, device="cuda")[None, :] >= torch.tensor(lens, device="cuda")[:, None]
    for t in (m, v, copy):
        t[beyond] = 77
    before = [t.clone() for t in (w, m, v, copy)]
    scales = dict(scales=tuple(torch.zeros(sum(-(-n // BLOCK) for n in lens), device="cuda") for _ in range(2))) if bits == 8 else {}
    cut = [[t[i, :n] for i, n in enumerate(lens)] for t in (w, g, m, v, copy)]
    ctx.gg_adamw_step(cut[0], cut[1], cut[2], cut[3], t=1, lr=1e-3, w_copy=cut[4], weight_decay=0.1, seed=SEED, **scales)
    for t, old in zip((w, m, v, copy), before):
        assert torch.equal(t[beyond], old[beyond])
    s0 = 0
    for i, n in enumerate(lens):
        g0, w0 = g[i, :n].double(), before[0][i, :n].double()
        w1, m1, v1 = adamw(w0, g0, torch.zeros_like(g0), torch.zeros_like(g0), 1, 1e-3, 0.1)
        upd = 1e-3 / 0.1 * m1.abs() / (torch.sqrt(v1 / (1 - 0.999)) + 1e-8)
        check = (w[i, :n].double() - w1).abs() <= 4 * U * w0.abs() + 32 * U * upd + (2.0 ** -7 * w1.abs() if w_dtype == torch.bfloat16 else 0.0) + 1e-37
        holds(check, f"w of {n}")
        holds((copy[i, :n].double() - w1).abs() <= 2.0 ** -8 * w1.abs() + 32 * U * upd + 1e-37, f"copy of {n}")
        if bits == 32:
            holds((m[i, :n].double() - m1).abs() <= 4 * U * m1.abs(), f"m of {n}")
            holds((v[i, :n].double() - v1).abs() <= 4 * U * v1, f"v of {n}")
        else:
            s1 = s0 + -(-n // BLOCK)
            check_state8(m[i, :n], scales["scales"][0][s0:s1].double(), m1, m1.abs(), noise_for(n, 1, i, SEED, 0, "cuda"), None)
            check_state8(v[i, :n], scales["scales"][1][s0:s1].double(), torch.sqrt(v1), torch.sqrt(v1), noise_for(n, 1, i, SEED, 4, "cuda"), 2.0 ** -62)
            s0 = s1
