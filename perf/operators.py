"""The operators of a training step that are timed against their plain form: layer norm, its gradient, and the AdamW
step over many tensors with states in 32 or in 8 bits.

`run` computes a pass in elementary torch operations (`own` false) or through the library (`own` true); `exact` gives
the same outputs from the definitions in 64 bits.  A case's tensors of the AdamW step lie in flat buffers, every
tensor starting at a multiple of 256 elements, so that the plain form sees them as rows of 256.
"""
import math
import random

import torch

own = False

ACTIVATIONS = (16384, 4096)      # the activation matrix of the repository's benchmarks: 8 x 2048 tokens, hidden 4096
BUCKET = 25_000_000              # its gradient buckets
BLOCK = 256                      # elements that share one scale of an 8-bit state
BETA1, BETA2, EPS, LR = 0.9, 0.999, 1e-8, 1e-4
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "bf16": 2}
SEED = 0x5EED0F0D17              # seed of the rounding noise


# ---------------------------------------------------------------- the cases
def norm_case(name, op, rows, cols, dtype, w_dtype, pad=0, affine=True):
    return dict(name=name, op=op, rows=rows, cols=cols, dtype=dtype, w_dtype=w_dtype, pad=pad, affine=affine)


def adamw_case(name, tensors, bits, w_dtype, g_dtype, copy=False, clip=False, count=0, total=0, shape_seed=0):
    return dict(name=name, op="adamw", tensors=tensors, bits=bits, w_dtype=w_dtype, g_dtype=g_dtype, copy=copy, clip=clip,
                count=count, total=total, shape_seed=shape_seed)


def listed():
    return [
        # the norm of one new token of a small decoder: nothing but latency
        norm_case("ln_token", "layer_norm", 1, 896, "bf16", "bf16"),
        # an odd width with rows that are not aligned to anything but their element
        norm_case("ln_ragged", "layer_norm", 4099, 1023, "f32", "f32"),
        # a training batch of activations
        norm_case("ln_activations", "layer_norm", *ACTIVATIONS, "bf16", "bf16"),
        # the gradient for a short prompt: few rows, so the sums over the rows have little to run over
        norm_case("ln_grad_short", "layer_norm_grad", 33, 896, "bf16", "f32"),
        norm_case("ln_grad_ragged", "layer_norm_grad", 4099, 1023, "f32", "f32"),
        norm_case("ln_grad_activations", "layer_norm_grad", *ACTIVATIONS, "bf16", "bf16"),
        # the norm weights of a small decoder, stepped as a parameter group of their own: 49 short vectors
        adamw_case("adamw_vectors", "vectors", 32, "f32", "f32"),
        # a whole small decoder: fp32 weights with a bf16 copy for the next forward pass, bf16 gradients, clipped
        adamw_case("adamw_decoder", "decoder", 32, "f32", "bf16", copy=True, clip=True),
        # bf16 weights without a master copy, tensors of odd lengths
        adamw_case("adamw_mixed", "mixed", 32, "bf16", "bf16", count=37, total=30_000_001, shape_seed=1),
        adamw_case("adamw8_vectors", "vectors", 8, "f32", "f32"),
        # the gradient buckets of the repository's benchmarks
        adamw_case("adamw8_buckets", "buckets", 8, "f32", "f32"),
        # the least memory a step can have here: bf16 weights and gradients, 8-bit states
        adamw_case("adamw8_decoder", "decoder", 8, "bf16", "bf16"),
    ]


def log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("layer_norm", "layer_norm_grad", "adamw32", "adamw8"))
    if kind.startswith("layer_norm"):
        cols = log_uniform(rng, 16, 16384)
        if rng.random() < 0.5:
            cols = max(16, cols // 8 * 8)
        rows = log_uniform(rng, 1, min(65536, ACTIVATIONS[0] * ACTIVATIONS[1] // cols))
        case = norm_case("", kind, rows, cols, rng.choice(("f32", "bf16")), rng.choice(("f32", "bf16")), rng.choice((0, 0, 8, 5)),
                         rng.random() < 0.8)
    else:
        count = log_uniform(rng, 1, 200)
        total = log_uniform(rng, max(1000, 16 * count), 8 * BUCKET)
        bits = 32 if kind == "adamw32" else 8
        w_dtype = rng.choice(("f32", "bf16"))
        case = adamw_case("", "mixed", bits, w_dtype, rng.choice(("f32", "bf16")), copy=w_dtype == "f32" and rng.random() < 0.5,
                          clip=bits == 32 and rng.random() < 0.5, count=count, total=total, shape_seed=rng.randrange(1 << 30))
    del case["name"]
    return case


def lengths(case):
    """Lengths of a case's tensors and whether weight decay applies to each (it does to matrices)."""
    if case["tensors"] == "vectors":
        return [896] * 49, [False] * 49
    if case["tensors"] == "buckets":
        return [BUCKET] * 8, [True] * 8
    if case["tensors"] == "decoder":      # 24 layers, hidden 896, MLP 4864, two key/value heads of 64, vocabulary 151936
        layer = [896 * 896, 128 * 896, 128 * 896, 896 * 896] + [4864 * 896] * 3 + [896, 896]
        lens = [151936 * 896] + layer * 24 + [896]
        return lens, [n > 896 for n in lens]
    rng = random.Random(case["shape_seed"])     # lengths that differ by factors of up to 1000, odd ones among them
    share = [math.exp(rng.uniform(0.0, math.log(1000.0))) for _ in range(case["count"])]
    lens = [max(1, int(case["total"] * s / sum(share))) for s in share]
    return lens, [rng.random() < 0.8 for _ in lens]


def work(case):
    if case["op"] != "adamw":
        n, e, we = case["rows"] * case["cols"], BYTES[case["dtype"]], BYTES[case["w_dtype"]] * case["affine"]
        if case["op"] == "layer_norm":
            return {"bytes": 2 * n * e + 8 * case["rows"] + 2 * we * case["cols"], "flops": 8 * n}
        return {"bytes": 3 * n * e + 8 * case["rows"] + (we + 8 * case["affine"]) * case["cols"], "flops": 14 * n}
    n = sum(lengths(case)[0])
    state = 16 if case["bits"] == 32 else 4 + 16 / BLOCK
    return {"bytes": n * (2 * BYTES[case["w_dtype"]] + BYTES[case["g_dtype"]] + 2 * case["copy"] + state),
            "flops": n * (16 + 2 * case["clip"])}


# ------------------------------------------------------------- the inputs
_contexts = {}


def context():
    if "ctx" not in _contexts:
        from paper_2506_00486_b200 import Context
        _contexts["ctx"] = Context(torch.cuda.current_device())
    return _contexts["ctx"]


def norm_inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rows, cols, dtype, w_dtype = case["rows"], case["cols"], DTYPES[case["dtype"]], DTYPES[case["w_dtype"]]

    def matrix():      # `pad` more columns than the operator sees: rows with a stride
        return torch.randn((rows, cols + case["pad"]), generator=gen, device="cuda")

    x = matrix().add_(0.1)
    x = torch.where(torch.rand(x.shape, generator=gen, device="cuda") < 1e-3, 20.0 * x, x).to(dtype)[:, :cols]
    s = dict(case=case, x=x, weight=None, bias=None, eps=1e-5)
    if case["affine"]:
        s["weight"] = (1.0 + 0.1 * torch.randn(cols, generator=gen, device="cuda")).to(w_dtype)
        s["bias"] = (0.1 * torch.randn(cols, generator=gen, device="cuda")).to(w_dtype)
    if case["op"] == "layer_norm_grad":
        s["dy"] = (1e-2 * matrix()).to(dtype)[:, :cols]
        xf = x.float()       # what the forward pass left behind
        s["mean"] = xf.mean(1)
        s["rstd"] = 1.0 / torch.sqrt((xf - s["mean"][:, None]).square().mean(1) + s["eps"])
    return s


def adamw_inputs(case, seed):
    lens, decays = lengths(case)
    blocks = [-(-n // BLOCK) for n in lens]
    total = sum(blocks) * BLOCK
    gen = torch.Generator(device="cuda").manual_seed(seed)
    n_blocks = torch.tensor(blocks, device="cuda")
    first = torch.cumsum(n_blocks, 0) - n_blocks
    segment = torch.repeat_interleave(torch.arange(len(lens), device="cuda"), n_blocks)       # tensor of each block
    size = (10.0 ** (-5.0 + 3.0 * torch.rand(len(lens), generator=gen, device="cuda")))[segment][:, None]

    def noise():
        return torch.randn((total // BLOCK, BLOCK), generator=gen, device="cuda")

    s = dict(case=case, lens=lens, offsets=(first * BLOCK).tolist(), segment=segment, first=first, t=1000)
    s["decay"] = torch.tensor([0.1 * d for d in decays], device="cuda")
    w = noise().mul_(0.02)
    g = noise()
    g = g.mul_(g.abs()).mul_(size)               # heavier tails than a normal's
    m = noise().mul_(size).mul_(0.3)
    v = torch.rand((total // BLOCK, BLOCK), generator=gen, device="cuda").add_(0.5).mul_(size).mul_(size)
    for off, n, b in zip(s["offsets"], lens, blocks):
        if n < b * BLOCK:
            for t in (w, g, m, v):
                t.view(-1)[off + n:off + b * BLOCK] = 0.0
    s["w"], s["g"] = w.to(DTYPES[case["w_dtype"]]), g.to(DTYPES[case["g_dtype"]])
    del w, g
    if case["bits"] == 32:
        s["m"], s["v"] = m, v
    else:
        for name, value in (("m", m), ("v", v.sqrt_())):       # the 8-bit state holds the root of the second moment
            scale = value.abs().amax(1) / 448.0
            s[name] = (value / scale.clamp_min(1e-30)[:, None]).to(torch.float8_e4m3fn)
            s[name + "_scale"] = scale
        s["grad_scale"] = torch.full((1,), 0.5, device="cuda")
    if case["copy"]:
        s["copy"] = s["w"].to(torch.bfloat16)
    return s


def prepare(case, seed):
    s = norm_inputs(case, seed) if case["op"] != "adamw" else adamw_inputs(case, seed)
    if own:
        ctx = context()
        if case["op"] == "layer_norm":
            s["call"] = ctx.make_layer_norm(s["x"], s["weight"], s["bias"], eps=s["eps"])
        elif case["op"] == "layer_norm_grad":
            s["call"] = ctx.make_layer_norm_grad(s["dy"], s["x"], s["mean"], s["rstd"], s["weight"])
        else:
            from paper_2506_00486_b200 import Segments

            def segments(name):
                return Segments.slices(s[name].view(-1), s["offsets"], s["lens"])

            more = dict(scales=(s["m_scale"], s["v_scale"]), grad_scale=s["grad_scale"]) if case["bits"] == 8 else {}
            s["call"] = ctx.make_adamw_step(
                segments("w"), segments("g"), segments("m"), segments("v"), w_copy=segments("copy") if case["copy"] else None,
                beta1=BETA1, beta2=BETA2, eps=EPS, weight_decay=s["decay"], max_norm=1.0 if case["clip"] else None, seed=SEED, **more)
    return s


# ------------------------------------------------------------ the plain form
def philox(group, tensor, step, seed):
    """Philox4x32-10 at counter (group, step, tensor), key = seed: four words of 32 bits, as int64 tensors."""
    mask = 0xFFFFFFFF
    c = [group & mask, group >> 32, torch.full_like(group, step & mask), tensor]
    k0, k1 = seed & mask, seed >> 32 & mask
    for _ in range(10):
        p0, p1 = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(p1 >> 32 & mask) ^ c[1] ^ k0, p1 & mask, (p0 >> 32 & mask) ^ c[3] ^ k1, p0 & mask]
        k0, k1 = (k0 + 0x9E3779B9) & mask, (k1 + 0xBB67AE85) & mask
    return c


def rounding_noise(s, step):
    """16 random bits for each element, [blocks, 32, 8]: one Philox block covers 8 elements of a tensor."""
    segment = s["segment"]
    block = torch.arange(segment.numel(), device="cuda") - s["first"][segment]
    group = block[:, None] * (BLOCK // 8) + torch.arange(BLOCK // 8, device="cuda")
    words = philox(group, segment[:, None].expand_as(group), step, SEED)
    return torch.stack([half for w in words for half in (w & 0xFFFF, w >> 16)], -1).to(torch.int32)


def shifted(noise, by):
    """Each element takes the bits of the element `by` places on in its group of 8."""
    return torch.roll(noise, -by, -1).view(-1, BLOCK)


def to_bf16(x, noise):
    """fp32 to bf16, up or down with probabilities that keep the mean."""
    return ((x.view(torch.int32) + noise) & -65536).view(torch.float32).to(torch.bfloat16)


def to_e4m3(x, noise, keep_above_zero):
    """[blocks, 256] fp32 to e4m3 codes and a scale per block, up or down with probabilities that keep the mean."""
    amax = x.abs().amax(1, keepdim=True)
    fits = amax > 2.0 ** -110
    y = x * torch.where(fits, torch.full_like(amax, 448.0) / amax, torch.zeros_like(amax))
    a = y.abs()
    small = a < 2.0 ** -6                             # the subnormals of e4m3 have the spacing of its first binade
    a = torch.where(small, a + 2.0 ** -6, a)
    code = ((a.view(torch.int32) + (noise * 16 + 8)) >> 20) - torch.where(small, 968, 960)
    code = code.clamp_max(126)
    if keep_above_zero:
        code = torch.where((y > 0) & (code == 0), 1, code)
    code = code + 128 * torch.signbit(x)
    return code.to(torch.uint8).view(torch.float8_e4m3fn), torch.where(fits, amax * (1.0 / 448.0), 0.0).view(-1)


def plain_layer_norm(s):
    x = s["x"].float()
    mean = x.mean(1)
    x = x - mean[:, None]
    rstd = 1.0 / torch.sqrt((x * x).mean(1) + s["eps"])
    y = x * rstd[:, None]
    if s["weight"] is not None:
        y = y * s["weight"].float() + s["bias"].float()
    return dict(y=y.to(s["x"].dtype), mean=mean, rstd=rstd)


def plain_layer_norm_grad(s):
    xhat = (s["x"].float() - s["mean"][:, None]) * s["rstd"][:, None]
    dy = s["dy"].float()
    d = dy if s["weight"] is None else dy * s["weight"].float()
    dx = (d - d.mean(1, keepdim=True) - xhat * (d * xhat).mean(1, keepdim=True)) * s["rstd"][:, None]
    out = dict(dx=dx.to(s["x"].dtype))
    if s["weight"] is not None:
        out.update(dweight=(dy * xhat).sum(0), dbias=dy.sum(0))
    return out


def plain_adamw(s):
    case, t = s["case"], s["t"]
    out = dict(w=s["w"], m=s["m"], v=s["v"])
    g = s["g"].float()
    if case["clip"]:
        norm = torch.sqrt((g * g).sum())
        out["scale"] = torch.clamp(1.0 / norm, max=1.0).view(1)
        g = g * out["scale"]
    narrow = case["bits"] == 8
    if narrow:
        g = g * s["grad_scale"]
        m = s["m"].float() * s["m_scale"][:, None]
        r = s["v"].float() * s["v_scale"][:, None]
        v = r * r
    else:
        m, v = s["m"], s["v"]
    m = m * BETA1 + g * (1.0 - BETA1)
    v = v * BETA2 + (g * g) * (1.0 - BETA2)
    r = torch.sqrt(v)
    keep = (1.0 - LR * s["decay"])[s["segment"]][:, None]
    w = s["w"].float() * keep - (LR / (1.0 - BETA1 ** t)) * (m / (r * (1.0 / math.sqrt(1.0 - BETA2 ** t)) + EPS))
    noise = rounding_noise(s, t) if narrow or case["w_dtype"] == "bf16" else None
    s["w"].copy_(to_bf16(w, shifted(noise, 2)) if case["w_dtype"] == "bf16" else w)
    if narrow:
        for name, value, by in (("m", m, 0), ("v", r, 4)):
            code, scale = to_e4m3(value, shifted(noise, by), name == "v")
            s[name].copy_(code)
            s[name + "_scale"].copy_(scale)
            out[name + "_scale"] = s[name + "_scale"]
    else:
        s["m"].copy_(m)
        s["v"].copy_(v)
    if case["copy"]:
        out["copy"] = s["copy"].copy_(w)
    return out


def run(state):
    op = state["case"]["op"]
    if op == "adamw":
        state["t"] += 1
        if not own:
            return plain_adamw(state)
        made = state["call"](state["t"], LR)
        names = ["w", "m", "v"] + ["copy"] * state["case"]["copy"] + ["m_scale", "v_scale"] * (state["case"]["bits"] == 8)
        out = {n: state[n] for n in names}
        if state["case"]["clip"]:
            out["scale"] = made["scale"]
        return out
    if not own:
        return plain_layer_norm(state) if op == "layer_norm" else plain_layer_norm_grad(state)
    out = state["call"]()
    return {n: t for n, t in out.items() if t is not None}


# ------------------------------------------------------------ in 64 bits
def exact_norm(s):
    x = s["x"].double()
    if s["case"]["op"] == "layer_norm":
        var, mean = torch.var_mean(x, 1, correction=0, keepdim=True)
        y = (x - mean) / torch.sqrt(var + s["eps"])
        if s["weight"] is not None:
            y = torch.addcmul(s["bias"].double(), y, s["weight"].double())
        return dict(y=y, mean=mean.view(-1), rstd=(var + s["eps"]).pow(-0.5).view(-1))
    # the chain rule through y = w (x - mean) rstd + b, with the mean and rstd that the call is given
    xc, r, dy, n = x - s["mean"].double()[:, None], s["rstd"].double()[:, None], s["dy"].double(), x.shape[1]
    d = dy if s["weight"] is None else dy * s["weight"].double()
    along = (d * xc).sum(1, keepdim=True)
    out = dict(dx=r * d - (r / n) * d.sum(1, keepdim=True) - xc * (r ** 3 / n) * along)
    if s["weight"] is not None:
        out.update(dweight=torch.einsum("rc,rc,r->c", dy, xc, s["rstd"].double()), dbias=dy.sum(0))
    return out


def exact_e4m3(x, noise, keep_above_zero):
    top = x.abs().amax(1, keepdim=True)
    y = torch.where(top > 2.0 ** -110, x / top * 448.0, 0.0)
    exponent = torch.floor(torch.log2(y.abs().clamp_min(2.0 ** -60))).clamp_min(-6.0)
    spacing = torch.exp2(exponent - 3.0)
    q = (torch.floor(y.abs() / spacing + (noise.double() + 0.5) / 65536.0) * spacing).clamp_max(448.0)
    if keep_above_zero:
        q = torch.where((y > 0) & (q == 0), 2.0 ** -9, q)
    return torch.copysign(q, x), torch.where(top > 2.0 ** -110, top / 448.0, 0.0).view(-1)


def exact_adamw(s):
    case, t, out = s["case"], s["t"] + 1, {}
    g = s["g"].double()
    if case["clip"]:
        out["scale"] = (1.0 / torch.linalg.vector_norm(g)).clamp(max=1.0).view(1)
        g *= out["scale"]
    narrow = case["bits"] == 8
    if narrow:
        g *= s["grad_scale"].double()
        m, v = (s[n].double() * s[n + "_scale"].double()[:, None] for n in ("m", "v"))
        v = v.square_()
    else:
        m, v = s["m"].double(), s["v"].double()
    m = torch.lerp(g, m, BETA1)
    v = torch.lerp(g.square_(), v, BETA2)
    del g
    update = (m / (1.0 - BETA1 ** t)) / ((v / (1.0 - BETA2 ** t)).sqrt_() + EPS)
    w = s["w"].double()
    w = w - LR * (update + s["decay"].double()[s["segment"]][:, None] * w)
    del update
    if case["copy"]:
        out["copy"] = w
    if not narrow and case["w_dtype"] != "bf16":
        return dict(out, w=w, m=m, v=v)
    noise = rounding_noise(s, t)
    if case["w_dtype"] == "bf16":
        spacing = torch.exp2(torch.floor(torch.log2(w.abs().clamp_min(2.0 ** -126))) - 7.0)
        w = torch.copysign(torch.floor(w.abs() / spacing + shifted(noise, 2).double() / 65536.0) * spacing, w)
    if narrow:
        m, out["m_scale"] = exact_e4m3(m, shifted(noise, 0), False)
        v, out["v_scale"] = exact_e4m3(v.sqrt_(), shifted(noise, 4), True)
    return dict(out, w=w, m=m, v=v)


def exact(case, seed):
    if case["op"] == "adamw":
        return exact_adamw(adamw_inputs(case, seed))
    return exact_norm(norm_inputs(case, seed))
