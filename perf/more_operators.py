"""The operators of a training step around its matrix products that are timed against their plain form: the softmax cross
entropy over a vocabulary and its gradient, the gated half of a feed-forward block and its gradient, and dropout.

`run` computes a pass in elementary torch operations (`own` false) or through the library (`own` true); `exact` gives
the same outputs from the definitions in 64 bits.
"""
import math

import numpy as np
import torch

own = False

SMALL = dict(width=896, hidden=4864, vocab=151936)       # the small decoder of the repository's initialisation workload
LARGE = dict(width=4096, hidden=11008, vocab=32000)      # the decoder of its weight sweep
TOKENS = 16384                                           # 8 x 2048 tokens, its activation matrix
IGNORED = -100                                           # the target of a position that has none
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "bf16": 2}
SEED = 0x5EED0F0D17                                      # of the dropout mask
MOST_FLOPS = 3.3e12


# ---------------------------------------------------------------- the cases
def loss_case(name, op, rows, width, vocab, ignored=0.05, pad=0):
    return dict(name=name, op=op, rows=rows, width=width, vocab=vocab, ignored=ignored, pad=pad)


def gated_case(name, op, rows, width, hidden, act="silu", keep=False, pad=0):
    return dict(name=name, op=op, rows=rows, width=width, hidden=hidden, act=act, keep=keep, pad=pad)


def dropout_case(name, rows, cols, dtype, p, residual, pad=0, t=1, tensor_id=0):
    return dict(name=name, op="dropout", rows=rows, cols=cols, dtype=dtype, p=p, residual=residual, pad=pad, t=t, tensor_id=tensor_id)


def listed():
    return [
        # the log-probability of one token of a small decoder: one pass over its output matrix
        loss_case("loss_token", "cross_entropy", 1, SMALL["width"], SMALL["vocab"], ignored=0.0),
        # a short evaluation batch: no size is a multiple of a tile, a quarter of the positions is padding
        loss_case("loss_ragged", "cross_entropy", 517, 1000, 32003, ignored=0.25),
        # the loss of a training batch
        loss_case("loss_batch", "cross_entropy", TOKENS, LARGE["width"], LARGE["vocab"]),
        # the gradient for a short prompt (tuning on a few tokens): nearly all of it is the gradient of the output matrix
        loss_case("loss_grad_short", "cross_entropy_grad", 33, SMALL["width"], SMALL["vocab"], ignored=0.1),
        # a training micro-batch of a small decoder, whose vocabulary outweighs its layers
        loss_case("loss_grad_decoder", "cross_entropy_grad", 4096, SMALL["width"], SMALL["vocab"]),
        # one new token of a small decoder: nothing but latency
        gated_case("gated_token", "gated_linear", 1, SMALL["width"], SMALL["hidden"]),
        # a serving batch of single tokens: one pass over both matrices
        gated_case("gated_tokens", "gated_linear", 64, LARGE["width"], LARGE["hidden"]),
        # the forward pass of a training batch, which keeps both projections for the backward pass
        gated_case("gated_batch", "gated_linear", TOKENS, LARGE["width"], LARGE["hidden"], keep=True),
        # an odd hidden width: rows that start on no vector boundary
        gated_case("gated_grad_ragged", "gated_linear_grad", 1023, 1000, 2731, act="gelu", keep=True),
        gated_case("gated_grad_batch", "gated_linear_grad", TOKENS // 2, LARGE["width"], LARGE["hidden"], keep=True),
        # an odd width, as the last piece of a sharded activation has it
        dropout_case("dropout_ragged", 4099, 1023, "f32", 0.5, False, t=7, tensor_id=3),
        # the end of a residual branch over a training batch
        dropout_case("dropout_activations", TOKENS, LARGE["width"], "bf16", 0.1, True, t=1000, tensor_id=11),
    ]


def log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def maybe_round(rng, n, to):
    return max(to, n // to * to) if rng.random() < 0.5 else n


def draw(rng):
    op = rng.choice(("cross_entropy", "cross_entropy_grad", "gated_linear", "gated_linear_grad", "dropout"))
    if op == "dropout":
        cols = maybe_round(rng, log_uniform(rng, 1, 16384), 8)
        rows = log_uniform(rng, 1, max(1, min(65536, TOKENS * LARGE["width"] // cols)))
        case = dropout_case("", rows, cols, rng.choice(("f32", "bf16")), round(rng.uniform(0.0, 0.9), 3), rng.random() < 0.5,
                            rng.choice((0, 0, 8, 5)), rng.randrange(1, 1 << 40), rng.randrange(1 << 16))
    else:
        width = maybe_round(rng, log_uniform(rng, 64, LARGE["width"]), 64)
        other = maybe_round(rng, log_uniform(rng, 1000, SMALL["vocab"]) if "entropy" in op else log_uniform(rng, 100, 16384), 64)
        each = 2 * width * other * (1 if "entropy" in op else 2) * {"cross_entropy": 1, "cross_entropy_grad": 3, "gated_linear": 1, "gated_linear_grad": 2}[op]
        rows = maybe_round(rng, log_uniform(rng, 1, max(1, min(TOKENS, int(MOST_FLOPS / each)))), 64 if rng.random() < 0.5 else 1)
        rows = max(1, min(rows, int(MOST_FLOPS / each)))
        pad = rng.choice((0, 0, 8, 5))
        if "entropy" in op:
            case = loss_case("", op, rows, width, other, round(rng.uniform(0.0, 0.5), 2), pad)
        else:
            keep = op == "gated_linear_grad" or rng.random() < 0.5
            case = gated_case("", op, rows, width, other, rng.choice(("silu", "gelu", "gelu_tanh", "relu")), keep, pad)
    del case["name"]
    return case


def work(case):
    op, rows = case["op"], case["rows"]
    if op == "dropout":
        n = rows * case["cols"]
        return {"bytes": n * BYTES[case["dtype"]] * (2 + case["residual"]), "flops": 2 * n}
    width = case["width"]
    if "entropy" in op:
        product, operands = 2 * rows * width * case["vocab"], 2 * (rows * width + case["vocab"] * width)
        if op == "cross_entropy":
            return {"bytes": operands + 16 * rows, "flops": product}
        return {"bytes": 2 * operands + 16 * rows, "flops": 3 * product}     # the logits, and the two products of their gradient
    hidden = case["hidden"]
    product, operands = 4 * rows * width * hidden, 2 * (rows * width + 2 * hidden * width)
    if op == "gated_linear":
        return {"bytes": operands + 2 * rows * hidden * (1 + 2 * case["keep"]), "flops": product}
    return {"bytes": 2 * operands + 6 * rows * hidden, "flops": 2 * product}


# ------------------------------------------------------------- the inputs
_contexts = {}


def context():
    if "ctx" not in _contexts:
        from paper_2506_00486_b200 import Context
        _contexts["ctx"] = Context(torch.cuda.current_device())
    return _contexts["ctx"]


def matrix(gen, rows, cols, scale, dtype, pad=0):
    """Rows of cols elements, `pad` elements apart from one another."""
    return torch.randn((rows, cols + pad), generator=gen, device="cuda").mul_(scale).to(dtype)[:, :cols]


def loss_inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rows, width, vocab = case["rows"], case["width"], case["vocab"]
    s = dict(case=case)
    s["w"] = matrix(gen, vocab, width, 0.02, torch.bfloat16, case["pad"])
    target = torch.randint(0, vocab, (rows,), generator=gen, device="cuda")
    # a model that has learnt something: a position's features lean towards its target
    toward = s["w"][target].float()
    lean = 8.0 * torch.rand((rows, 1), generator=gen, device="cuda")
    h = torch.randn((rows, width + case["pad"]), generator=gen, device="cuda")
    h[:, :width] += toward * (lean / toward.square().sum(1, keepdim=True).sqrt())
    s["h"] = h.to(torch.bfloat16)[:, :width]
    ignored = torch.rand(rows, generator=gen, device="cuda") < case["ignored"]
    s["target"] = torch.where(ignored, IGNORED, target)
    if case["op"] == "cross_entropy_grad":       # what the forward pass left behind, and the weight of each position in the mean
        logits = s["h"].float() @ s["w"].float().t()
        most = logits.amax(1)
        s["lse"] = logits.sub_(most[:, None]).exp_().sum(1).log_() + most
        s["dloss"] = torch.full((rows,), 1.0 / max(1, rows - int(case["ignored"] * rows)), device="cuda")
    return s


def gated_inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rows, width, hidden = case["rows"], case["width"], case["hidden"]
    s = dict(case=case)
    s["x"] = matrix(gen, rows, width, 1.0, torch.bfloat16, case["pad"])
    for name in ("w_gate", "w_up"):
        s[name] = matrix(gen, hidden, width, 1.2 / math.sqrt(width), torch.bfloat16, case["pad"])
    if case["op"] == "gated_linear_grad":        # what the forward pass left behind
        for name, w in (("gate", "w_gate"), ("up", "w_up")):
            s[name] = (s["x"].float() @ s[w].float().t()).to(torch.bfloat16)
        s["dh"] = matrix(gen, rows, hidden, 1e-2, torch.bfloat16, case["pad"])
    return s


def dropout_inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(case=case, seed=SEED + seed, residual=None)
    s["x"] = matrix(gen, case["rows"], case["cols"], 1.0, DTYPES[case["dtype"]], case["pad"])
    if case["residual"]:
        s["residual"] = matrix(gen, case["rows"], case["cols"], 4.0, DTYPES[case["dtype"]], case["pad"])
    return s


def inputs(case, seed):
    return (loss_inputs if "entropy" in case["op"] else gated_inputs if "gated" in case["op"] else dropout_inputs)(case, seed)


def prepare(case, seed):
    s = inputs(case, seed)
    if own:
        ctx, op = context(), case["op"]
        if op == "cross_entropy":
            s["call"] = ctx.make_cross_entropy(s["h"], s["w"], s["target"])
        elif op == "cross_entropy_grad":
            s["call"] = ctx.make_cross_entropy_grad(s["dloss"], s["h"], s["w"], s["target"], s["lse"])
        elif op == "gated_linear":
            s["call"] = ctx.make_gated_linear(s["x"], s["w_gate"], s["w_up"], act=case["act"], keep=case["keep"])
        elif op == "gated_linear_grad":
            s["call"] = ctx.make_gated_linear_grad(s["dh"], s["x"], s["w_gate"], s["w_up"], s["gate"], s["up"], act=case["act"])
        else:
            s["call"] = ctx.make_dropout(s["x"], case["p"], residual=s["residual"], seed=s["seed"], tensor_id=case["tensor_id"])
    return s


# ------------------------------------------------------------ the plain form
def plain_loss(s):
    logits = s["h"].float() @ s["w"].float().t()
    most = logits.amax(1)
    lse = torch.exp(logits - most[:, None]).sum(1).log() + most
    there = s["target"] >= 0
    at = torch.gather(logits, 1, s["target"].clamp_min(0)[:, None])[:, 0]
    return dict(loss=torch.where(there, lse - at, 0.0), lse=lse)


def plain_loss_grad(s):
    h, w = s["h"].float(), s["w"].float()
    there = s["target"] >= 0
    d = torch.exp(h @ w.t() - s["lse"][:, None])
    row = torch.arange(d.shape[0], device="cuda")
    d[row, s["target"].clamp_min(0)] -= 1.0
    d = d * torch.where(there, s["dloss"], 0.0)[:, None]
    return dict(dh=(d @ w).to(torch.bfloat16), dw=(d.t() @ h).to(torch.bfloat16))


def activation(a, act):
    """act(a) and its derivative."""
    if act == "silu":
        s = 1.0 / (1.0 + torch.exp(-a))
        return a * s, s * (1.0 + a * (1.0 - s))
    if act == "relu":
        on = (a > 0).to(a.dtype)
        return a * on, on
    if act == "gelu":
        cdf = 0.5 * (1.0 + torch.erf(a * math.sqrt(0.5)))
        return a * cdf, cdf + a * torch.exp(-0.5 * a * a) * (1.0 / math.sqrt(2.0 * math.pi))
    c, k = math.sqrt(2.0 / math.pi), 0.044715
    t = torch.tanh(c * (a + k * a * a * a))
    return 0.5 * a * (1.0 + t), 0.5 * (1.0 + t) + 0.5 * a * (1.0 - t * t) * c * (1.0 + 3.0 * k * a * a)


def plain_gated(s):
    x = s["x"].float()
    gate, up = x @ s["w_gate"].float().t(), x @ s["w_up"].float().t()
    out = dict(h=(activation(gate, s["case"]["act"])[0] * up).to(torch.bfloat16))
    if s["case"]["keep"]:
        out.update(gate=gate.to(torch.bfloat16), up=up.to(torch.bfloat16))
    return out


def plain_gated_grad(s):
    x, dh, up = s["x"].float(), s["dh"].float(), s["up"].float()
    value, slope = activation(s["gate"].float(), s["case"]["act"])
    dgate, dup = dh * up * slope, dh * value
    return dict(dx=(dgate @ s["w_gate"].float() + dup @ s["w_up"].float()).to(torch.bfloat16),
                dw_gate=(dgate.t() @ x).to(torch.bfloat16), dw_up=(dup.t() @ x).to(torch.bfloat16))


def philox(c0, c1, c2, c3, seed):
    """Philox4x32-10, key = seed: four words of 32 bits, as int64 tensors."""
    mask = 0xFFFFFFFF
    c = [c0, c1, c2, c3]
    k0, k1 = seed & mask, seed >> 32 & mask
    for _ in range(10):
        p0, p1 = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(p1 >> 32 & mask) ^ c[1] ^ k0, p1 & mask, (p0 >> 32 & mask) ^ c[3] ^ k1, p0 & mask]
        k0, k1 = (k0 + 0x9E3779B9) & mask, (k1 + 0xBB67AE85) & mask
    return c


def plain_dropout(s):
    case = s["case"]
    rows, cols = case["rows"], case["cols"]
    groups = -(-cols // 8)                       # 128 bits for eight elements of a row
    j = torch.arange(rows * groups, device="cuda")
    words = philox(j & 0xFFFFFFFF, j >> 32, torch.full_like(j, case["t"] & 0xFFFFFFFF), torch.full_like(j, case["tensor_id"]), s["seed"])
    bits = torch.stack([half for w in words for half in (w & 0xFFFF, w >> 16)], 1).view(rows, groups * 8)[:, :cols]
    least = int(case["p"] * 65536.0 + 0.5)
    y = torch.where(bits >= least, s["x"].float() * (65536.0 / (65536 - least)), 0.0)
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return dict(y=y.to(s["x"].dtype))


PLAIN = dict(cross_entropy=plain_loss, cross_entropy_grad=plain_loss_grad, gated_linear=plain_gated, gated_linear_grad=plain_gated_grad,
             dropout=plain_dropout)


def run(state):
    case = state["case"]
    if not own:
        return PLAIN[case["op"]](state)
    out = state["call"](case["t"]) if case["op"] == "dropout" else state["call"]()
    return {n: t for n, t in out.items() if t is not None}


# ------------------------------------------------------------ in 64 bits
def exact_loss(s):
    logits = torch.einsum("rc,vc->rv", s["h"].double(), s["w"].double())
    lse = torch.logsumexp(logits, 1)
    rows = torch.nonzero(s["target"] >= 0)[:, 0]
    if s["case"]["op"] == "cross_entropy":
        loss = torch.zeros_like(lse)
        loss[rows] = lse[rows] - logits[rows, s["target"][rows]]
        return dict(loss=loss, lse=lse)
    # the chain rule through loss = lse - logit, with the lse that the call is given, over the rows that count
    p = torch.exp(logits[rows] - s["lse"][rows].double()[:, None])
    p[torch.arange(rows.numel(), device="cuda"), s["target"][rows]] -= 1.0
    p *= s["dloss"][rows].double()[:, None]
    dh = torch.zeros(s["h"].shape, dtype=torch.float64, device="cuda")
    dh[rows] = p @ s["w"].double()
    return dict(dh=dh, dw=torch.einsum("rv,rc->vc", p, s["h"][rows].double()))


def exact_act(a, act):
    """act(a) in 64 bits; its derivative comes from autograd."""
    if act == "silu":
        return a * torch.sigmoid(a)
    if act == "relu":
        return torch.clamp(a, min=0.0)
    if act == "gelu":
        return a * 0.5 * torch.special.erfc(-a / math.sqrt(2.0))
    # (1 + tanh z) / 2 = sigmoid(2 z)
    return a * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (a + 0.044715 * a ** 3))


def exact_gated(s):
    act = s["case"]["act"]
    x, wg, wu = (s[n].double() for n in ("x", "w_gate", "w_up"))
    if s["case"]["op"] == "gated_linear":
        gate, up = torch.einsum("rc,fc->rf", x, wg), torch.einsum("rc,fc->rf", x, wu)
        out = dict(h=exact_act(gate, act) * up)
        return dict(out, gate=gate, up=up) if s["case"]["keep"] else out
    with torch.enable_grad():
        gate, up = (s[n].double().requires_grad_(True) for n in ("gate", "up"))
        dgate, dup = torch.autograd.grad(exact_act(gate, act) * up, (gate, up), s["dh"].double())
    return dict(dx=torch.einsum("rf,fc->rc", dgate, wg) + torch.einsum("rf,fc->rc", dup, wu),
                dw_gate=torch.einsum("rf,rc->fc", dgate, x), dw_up=torch.einsum("rf,rc->fc", dup, x))


def exact_dropout(s):
    """The mask on the host, in unsigned words of 64 bits."""
    case, low = s["case"], np.uint64(0xFFFFFFFF)
    groups = (case["cols"] + 7) // 8
    at = np.arange(case["rows"] * groups, dtype=np.uint64)
    a, b = at & low, at >> np.uint64(32)
    c, d = np.full_like(at, case["t"] % 2 ** 32), np.full_like(at, case["tensor_id"])
    k, l = s["seed"] % 2 ** 32, s["seed"] // 2 ** 32 % 2 ** 32
    for r in range(10):
        u, v = a * np.uint64(0xD2511F53), c * np.uint64(0xCD9E8D57)
        a, b = v // np.uint64(2 ** 32) ^ b ^ np.uint64((k + r * 0x9E3779B9) % 2 ** 32), v & low
        c, d = u // np.uint64(2 ** 32) ^ d ^ np.uint64((l + r * 0xBB67AE85) % 2 ** 32), u & low
    bits = np.stack((a, b, c, d), 1).astype("<u4").view("<u2").reshape(case["rows"], groups * 8)[:, :case["cols"]]
    dropped = round(case["p"] * 65536)
    kept = torch.from_numpy(bits >= dropped).cuda()
    y = s["x"].double() * kept / (1.0 - dropped / 65536)
    return dict(y=y if s["residual"] is None else y + s["residual"].double())


def exact(case, seed):
    s = inputs(case, seed)
    return (exact_loss if "entropy" in case["op"] else exact_gated if "gated" in case["op"] else exact_dropout)(s)
