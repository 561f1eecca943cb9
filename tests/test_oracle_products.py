"""Pins of the 64-bit forms of the vocabulary loss, the gated block and dropout: closed forms, differences, torch in fp64."""
import math

import numpy as np
import pytest
import torch

from oracle import product_oracle as o


def test_loss_of_known_logits():
    # logits ln 1, ln 2, ln 5 of one feature: the probabilities are 1/8, 2/8, 5/8
    w = np.log(np.array([[1.0], [2.0], [5.0]]))
    loss, lse, _ = o.cross_entropy(np.ones((4, 1)), w, [0, 1, 2, -100])
    assert np.allclose(lse, math.log(8.0), rtol=1e-15) and np.allclose(loss, [math.log(8), math.log(4), math.log(1.6), 0.0], rtol=1e-14)
    assert np.isnan(o.cross_entropy(np.ones((1, 1)), w, [3])[0][0])
    _, _, d = o.cross_entropy_grad([2.0, 1.0], np.ones((2, 1)), w, [1, -1], lse[:2])
    assert np.allclose(d, [[0.25, -1.5, 1.25], [0.0, 0.0, 0.0]], atol=1e-15)


def test_loss_and_gradient_against_torch_and_differences():
    rng = np.random.default_rng(0)
    h, w, target, g = rng.normal(size=(6, 5)), rng.normal(size=(9, 5)), [3, -100, 0, 8, 3, 3], rng.normal(size=6)
    loss, lse, _ = o.cross_entropy(h, w, target)
    th, tw = (torch.tensor(t, requires_grad=True) for t in (h, w))
    want = torch.nn.functional.cross_entropy(th @ tw.t(), torch.tensor(target), reduction="none")
    assert np.allclose(loss, want.detach().numpy(), rtol=1e-13, atol=1e-13)
    want.backward(torch.tensor(g))
    dh, dw, _ = o.cross_entropy_grad(g, h, w, target, lse)
    assert np.allclose(dh, th.grad.numpy(), atol=1e-13) and np.allclose(dw, tw.grad.numpy(), atol=1e-13)
    e = 1e-6     # (central differences: e^2 f''' / 6 and 1e-16 |f| / e are below 1e-9)
    for at in ((0, 0), (3, 4), (1, 2)):
        step = np.zeros_like(h)
        step[at] = e
        diff = sum(gi * (a - b) for gi, a, b in zip(g, o.cross_entropy(h + step, w, target)[0], o.cross_entropy(h - step, w, target)[0])) / (2 * e)
        assert diff == pytest.approx(dh[at], abs=1e-8)


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh", "relu"])
def test_activations(act):
    a = np.linspace(-9.0, 9.0, 1001)
    value, slope = o.activation(a, act)
    t = torch.tensor(a, requires_grad=True)
    f = {"silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu, "relu": torch.nn.functional.relu,
         "gelu_tanh": lambda v: torch.nn.functional.gelu(v, approximate="tanh")}[act](t)
    f.sum().backward()
    # torch's 1 + tanh is off by 2^-53, which its derivative multiplies by at most |a| c (1 + 3 k a^2) = 9 * 0.8 * 12 here
    assert np.allclose(value, f.detach().numpy(), rtol=1e-12, atol=1e-14) and np.allclose(slope, t.grad.numpy(), rtol=1e-12, atol=2e-14)


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh", "relu"])
def test_gated_block_against_torch(act):
    rng = np.random.default_rng(1)
    x, wg, wu, dh = (rng.normal(size=s) for s in ((4, 3), (7, 3), (7, 3), (4, 7)))
    h, gate, up = o.gated_linear(x, wg, wu, act)
    dx, dwg, dwu, _, _ = o.gated_linear_grad(dh, x, wg, wu, gate, up, act)
    tx, tg, tu = (torch.tensor(t, requires_grad=True) for t in (x, wg, wu))
    f = {"silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu, "relu": torch.nn.functional.relu,
         "gelu_tanh": lambda v: torch.nn.functional.gelu(v, approximate="tanh")}[act]
    want = f(tx @ tg.t()) * (tx @ tu.t())
    want.backward(torch.tensor(dh))
    for got, ref in ((h, want.detach()), (dx, tx.grad), (dwg, tg.grad), (dwu, tu.grad)):
        assert np.allclose(got, ref.numpy(), rtol=1e-12, atol=1e-13)


def test_dropout_bits():
    # the first block of counter 0, key 0 is the known answer 6627e8d5 e169c58d bc57ac4c 9b00dbd8
    assert o.dropout_bits(1, 8, 0, 0, 0).tolist() == [[0xE8D5, 0x6627, 0xC58D, 0xE169, 0xAC4C, 0xBC57, 0xDBD8, 0x9B00]]
    # a row starts a block of its own; rows can be drawn from any row on
    whole = o.dropout_bits(5, 11, 3, 2, 99)
    assert np.array_equal(whole[3:], o.dropout_bits(2, 11, 3, 2, 99, first=3))
    bits = o.dropout_bits(100, 1000, 7, 1, 5)
    for p in (0.0, 0.1, 0.5, 0.9):
        kept = o.dropout(np.ones(bits.shape), p, bits)
        q = math.floor(p * 65536 + 0.5) / 65536
        n = bits.size      # (the mean of n elements is off by more than 5 standard deviations once in a million)
        assert abs(kept.mean() - 1.0) <= 5 * math.sqrt(q / (1 - q) / n) + 1e-12
    assert np.array_equal(o.dropout(np.ones((1, 8)), 0.5, np.array([[0, 32767, 32768, 65535, 1, 2, 3, 40000]]), 3.0), [[3.0, 3.0, 5.0, 5.0, 3.0, 3.0, 3.0, 5.0]])
