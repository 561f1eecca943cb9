"""Shared by the tests of the operators around matrix products: matrices with strides, and bounds on sums.

A product of bf16 values is exact in fp32.  The tensor cores add 16 of them and the sum so far at once, each term cut at 24
bits below the largest of them or better, so one such step is off by at most 17 * 2^-24 of sum|terms|, and a sum of n terms by
(n / 16 + 1) steps of that: SUM(n) * sum|terms| with SUM(n) = (n + 32) * 1.0625 * 2^-24.  A bf16 value is half a unit off, 2^-8 relative (2^-9 of
the next power of two)."""
import numpy as np
import torch

U, BF16 = 2.0 ** -24, 2.0 ** -8


def SUM(n):
    return (n + 32) * 1.0625 * U


def host(t):
    return None if t is None else t.double().cpu().numpy()


def matrix(gen, rows, cols, pad=0, shift=0, scale=1.0, dtype=torch.bfloat16):
    """A [rows, cols] view with row stride cols + pad that starts `shift` elements into its buffer."""
    flat = torch.full((rows * (cols + pad) + shift + 8,), 7.0, dtype=dtype, device="cuda")
    t = flat[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    t.copy_(torch.randn((rows, cols), generator=gen, device="cuda") * scale)
    return t


def around(t, shift):
    """The buffer of matrix() without the elements of t, as bits."""
    flat = t.as_strided((t._base.numel(),), (1,), 0).clone()
    inner = flat[shift:shift + t.shape[0] * t.stride(0)].view(t.shape[0], t.stride(0)) if t.shape[0] else flat[:0].view(0, 1)
    inner[:, :t.shape[1]] = 0
    return flat


def near(got, want, tol, what=""):
    got = host(got) if isinstance(got, torch.Tensor) else got
    off = np.abs(got - want) - tol
    assert np.all(off <= 0), (what, float(off.max()), np.unravel_index(np.argmax(off), off.shape))
