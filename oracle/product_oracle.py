"""The vocabulary loss, the gated block, their gradients and dropout in plain 64-bit numpy, from the formulas.

Test infrastructure only, and apart from the library: arrays in, arrays out, no blocking and no tricks."""
import math

import numpy as np

from oracle.train_oracle import philox4x32_10

_erfc = np.vectorize(math.erfc, otypes=[np.float64])


# ------------------------------------------------------------- vocabulary loss
def cross_entropy(h, w, target):
    """(loss, lse, logits) of the rows of h; a negative target has loss 0, one beyond the vocabulary nan."""
    logits = np.asarray(h, dtype=np.float64) @ np.asarray(w, dtype=np.float64).T
    most = logits.max(axis=1)
    lse = np.log(np.exp(logits - most[:, None]).sum(axis=1)) + most
    loss = np.zeros(len(target))
    for r, t in enumerate(target):
        if t >= 0:
            loss[r] = lse[r] - logits[r, t] if t < logits.shape[1] else np.nan
    return loss, lse, logits


def cross_entropy_grad(dloss, h, w, target, lse):
    """(dh, dw, d) with d the gradient of the logits, for the lse that is given."""
    h, w = np.asarray(h, dtype=np.float64), np.asarray(w, dtype=np.float64)
    d = np.exp(h @ w.T - np.asarray(lse, dtype=np.float64)[:, None])
    for r, t in enumerate(target):
        if t < 0:
            d[r] = 0.0
            continue
        if t < w.shape[0]:
            d[r, t] -= 1.0
        d[r] *= dloss[r] if t < w.shape[0] else np.nan
    return d @ w, d.T @ h, d


# ---------------------------------------------------------------- gated block
def activation(a, act):
    """(act(a), its derivative)."""
    a = np.asarray(a, dtype=np.float64)
    if act == "relu":
        return np.where(a > 0, a, 0.0), np.where(a > 0, 1.0, 0.0)
    if act == "silu":
        s = 1.0 / (1.0 + np.exp(-a))
        return a * s, s + a * s * (1.0 - s)
    if act == "gelu":
        cdf = 0.5 * _erfc(-a / math.sqrt(2.0))
        return a * cdf, cdf + a * np.exp(-0.5 * a * a) / math.sqrt(2.0 * math.pi)
    c, k = math.sqrt(2.0 / math.pi), 0.044715
    s = 1.0 / (1.0 + np.exp(-2.0 * c * (a + k * a ** 3)))       # (1 + tanh z) / 2, which cancels for negative z
    return a * s, s + a * s * (1.0 - s) * 2.0 * c * (1.0 + 3.0 * k * a * a)


def gated_linear(x, w_gate, w_up, act):
    """(h, gate, up)."""
    x, w_gate, w_up = (np.asarray(t, dtype=np.float64) for t in (x, w_gate, w_up))
    gate, up = x @ w_gate.T, x @ w_up.T
    return activation(gate, act)[0] * up, gate, up


def gated_linear_grad(dh, x, w_gate, w_up, gate, up, act):
    """(dx, dw_gate, dw_up, dgate, dup)."""
    dh, x, w_gate, w_up, gate, up = (np.asarray(t, dtype=np.float64) for t in (dh, x, w_gate, w_up, gate, up))
    value, slope = activation(gate, act)
    dgate, dup = dh * up * slope, dh * value
    return dgate @ w_gate + dup @ w_up, dgate.T @ x, dup.T @ x, dgate, dup


# -------------------------------------------------------------------- dropout
def dropout_bits(rows, cols, t, tensor_id, seed, first=0):
    """The 16 random bits of each element of `rows` rows from row `first` on: [rows, cols] integers."""
    groups = (cols + 7) // 8
    j = np.arange(rows * groups, dtype=np.uint64) + np.uint64(first * groups)
    same = np.zeros_like(j)
    w = philox4x32_10((j & np.uint64(0xFFFFFFFF), j >> np.uint64(32), same + np.uint64(t % 2 ** 32), same + np.uint64(tensor_id)),
                      (seed & 0xFFFFFFFF, seed >> 32 & 0xFFFFFFFF))
    bits = np.stack([h for v in w for h in (v & 0xFFFF, v >> 16)], axis=1)
    return bits.reshape(rows, groups * 8)[:, :cols].astype(np.int64)


def dropout(x, p, bits, residual=None):
    least = int(math.floor(p * 65536 + 0.5))
    y = np.where(bits >= least, np.asarray(x, dtype=np.float64), 0.0) / (1.0 - least / 65536.0)
    return y if residual is None else y + residual
