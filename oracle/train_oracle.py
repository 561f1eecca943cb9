"""Layer norm, its gradient, the gradient norm and the AdamW step in plain 64-bit numpy, from the formulas.

Test infrastructure only, and apart from the library: arrays in, arrays out, no blocking and no tricks."""
import numpy as np

BLOCK = 256


# ------------------------------------------------------------------- layer norm
def layer_norm(x, weight=None, bias=None, eps=1e-5):
    """(y, mean, rstd) of the rows of x."""
    x = np.asarray(x, dtype=np.float64)
    mean = x.mean(axis=1)
    rstd = 1.0 / np.sqrt(((x - mean[:, None]) ** 2).mean(axis=1) + eps)
    y = (x - mean[:, None]) * rstd[:, None]
    if weight is not None:
        y = y * weight
    if bias is not None:
        y = y + bias
    return y, mean, rstd


def layer_norm_grad(dy, x, mean, rstd, weight=None):
    """(dx, dweight, dbias)."""
    dy, x = np.asarray(dy, dtype=np.float64), np.asarray(x, dtype=np.float64)
    xhat = (x - mean[:, None]) * rstd[:, None]
    d = dy if weight is None else dy * weight
    dx = rstd[:, None] * (d - d.mean(axis=1, keepdims=True) - xhat * (d * xhat).mean(axis=1, keepdims=True))
    return dx, (dy * xhat).sum(axis=0), dy.sum(axis=0)


# ---------------------------------------------------------------- random numbers
def philox4x32_10(counter, key):
    """counter: four uint32 arrays, key: two ints; four uint32 arrays."""
    c = [np.asarray(v, dtype=np.uint64) for v in counter]
    k = [int(v) for v in key]
    low = np.uint64(0xFFFFFFFF)
    for _ in range(10):
        p0, p1 = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(p1 >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), p1 & low, (p0 >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), p0 & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return [v.astype(np.uint32) for v in c]


def rounding_noise(n, t, segment, seed):
    """The 16 random bits of elements 0 .. n-1 of a segment, in groups of 8: [ceil(n / 8), 8] integers."""
    j = np.arange((n + 7) // 8, dtype=np.uint64)
    same = np.zeros_like(j)
    w = philox4x32_10((j & np.uint64(0xFFFFFFFF), j >> np.uint64(32), same + np.uint64(t & 0xFFFFFFFF), same + np.uint64(segment)),
                      (seed & 0xFFFFFFFF, seed >> 32 & 0xFFFFFFFF))
    return np.stack([h for v in w for h in (v & 0xFFFF, v >> 16)], axis=1).astype(np.int64)


def noise_for(n, t, segment, seed, shift):
    """The bits that element e takes: those of place e + shift (modulo 8) in its group."""
    return np.roll(rounding_noise(n, t, segment, seed), -shift, axis=1).reshape(-1)[:n]


# ------------------------------------------------------------------------ rounding
def e4m3_position(y):
    """Where |y| lies on the e4m3 grid, as a real code: code k stands at position k, and in between it is linear."""
    a = np.abs(y)
    e = np.maximum(np.floor(np.log2(np.maximum(a, 2.0 ** -40))), -6.0)
    return np.where(a < 2.0 ** -6, a * 512.0, (e + 6.0) * 8.0 + a / 2.0 ** (e - 3.0))


def e4m3_value(code):
    """The value of e4m3 codes (0 .. 255); 127 and 255 are nan."""
    k, s = np.asarray(code).astype(np.int64) & 127, np.asarray(code).astype(np.int64) >> 7
    e = np.maximum(k >> 3, 1)
    v = np.where(k < 8, k / 512.0, (8 + (k & 7)) * 2.0 ** (e - 10.0))
    v = np.where(k == 127, np.nan, v)
    return np.where(s == 1, -v, v)


def block_tops(x):
    """Largest magnitude of every block of 256 (the last may be short)."""
    return np.array([np.abs(x[i:i + BLOCK]).max() for i in range(0, x.size, BLOCK)])


def quantise(x, noise, keep_above_zero):
    """(codes, scales, positions + noise) of a state: floor of the last is the code."""
    top = block_tops(x)
    fits = top > 2.0 ** -110
    factor = np.repeat(np.where(fits, 448.0 / np.where(fits, top, 1.0), 0.0), BLOCK)[:x.size]
    pos = e4m3_position(x * factor) + (noise + 0.5) / 65536.0
    code = np.minimum(np.floor(pos), 126)
    if keep_above_zero:
        code = np.where((x * factor > 0) & (code == 0), 1, code)
    return (code + 128 * np.signbit(x)).astype(np.uint8), np.where(fits, top / 448.0, 0.0), pos


# --------------------------------------------------------------------------- AdamW
def grad_norm(gs):
    return float(np.sqrt(sum((np.asarray(g, dtype=np.float64) ** 2).sum() for g in gs)))


def adamw(w, g, m, v, t, lr, beta1=0.9, beta2=0.999, eps=1e-8, decay=0.0):
    """(w, m, v) after step t; v is the second moment itself."""
    w, g, m, v = (np.asarray(a, dtype=np.float64) for a in (w, g, m, v))
    m = beta1 * m + (1.0 - beta1) * g
    v = beta2 * v + (1.0 - beta2) * g * g
    mhat, vhat = m / (1.0 - beta1 ** t), v / (1.0 - beta2 ** t)
    return w - lr * decay * w - lr * mhat / (np.sqrt(vhat) + eps), m, v
