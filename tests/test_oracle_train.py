"""Pins of the 64-bit forms of layer norm and the AdamW step: closed forms, differences, known answers."""
import os

import numpy as np
import pytest
import torch

from oracle import train_oracle as o

HERE = os.path.dirname(os.path.abspath(__file__))


def test_layer_norm_of_a_known_row():
    # 1, 2, 3, 6: mean 3, variance (4 + 1 + 0 + 9) / 4
    y, mean, rstd = o.layer_norm(np.array([[1.0, 2.0, 3.0, 6.0]]), np.array([1.0, 1.0, 1.0, 2.0]), np.array([0.0, 0.0, 5.0, 0.0]), eps=0.0)
    assert mean[0] == 3.0 and rstd[0] == pytest.approx(3.5 ** -0.5, rel=1e-15)
    assert np.allclose(y[0], np.array([-2.0, -1.0, 0.0, 6.0]) / np.sqrt(3.5) + np.array([0.0, 0.0, 5.0, 0.0]), rtol=1e-14)


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 7), (5, 3), (4, 32)])
def test_layer_norm_gradient_against_differences(rows, cols):
    rng = np.random.default_rng(rows * 100 + cols)
    x, dy, w, b = rng.normal(1.0, 2.0, (rows, cols)), rng.normal(size=(rows, cols)), rng.normal(size=cols), rng.normal(size=cols)
    _, mean, rstd = o.layer_norm(x, w, b)
    dx, dw, db = o.layer_norm_grad(dy, x, mean, rstd, w)

    def loss(x_, w_, b_):
        return (dy * o.layer_norm(x_, w_, b_)[0]).sum()

    h = 1e-5      # central differences: h^2 f''' / 6 and 1e-16 |f| / h are both below 1e-8 for these sizes (rstd up to 1 / sqrt(eps) with one column)
    for i in np.ndindex(x.shape):
        e = np.zeros_like(x)
        e[i] = h
        assert (loss(x + e, w, b) - loss(x - e, w, b)) / (2 * h) == pytest.approx(dx[i], abs=1e-6)
    for c in range(cols):
        e = np.zeros(cols)
        e[c] = h
        assert (loss(x, w + e, b) - loss(x, w - e, b)) / (2 * h) == pytest.approx(dw[c], abs=1e-6)
        assert (loss(x, w, b + e) - loss(x, w, b - e)) / (2 * h) == pytest.approx(db[c], abs=1e-6)


def test_philox_known_answers():
    for line in open(os.path.join(HERE, "golden", "philox4x32_10_kat.txt")):
        words = [int(v, 16) for v in line.split("#")[0].split()]
        if not words:
            continue
        got = o.philox4x32_10([np.array([v]) for v in words[:4]], words[4:6])
        assert [int(v[0]) for v in got] == words[6:10]


def test_e4m3_values_are_those_of_the_type():
    codes = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(o.e4m3_value(codes), want, equal_nan=True)
    finite = codes[:127]
    assert np.array_equal(o.e4m3_position(want[:127]), finite.astype(np.float64))


def test_stochastic_rounding_keeps_the_mean_and_exact_values():
    rng = np.random.default_rng(3)
    noise = np.arange(65536)
    for top, x in ((448.0, 17.3), (448.0, 0.0011), (448.0, 2.0 ** -6 - 1e-5), (448.0, 300.0)):
        block = np.full(65536, x)
        block[::256] = top
        code, _, _ = o.quantise(block, noise, False)
        got = o.e4m3_value(code)[np.arange(65536) % 256 != 0]
        spacing = max(2.0 ** (np.floor(np.log2(x)) - 3), 2.0 ** -9)
        # every 256th value of the noise is left out: the mean of the rest is off by less than 1/256 of the spacing
        assert abs(got.mean() - x) <= spacing / 256 + 1e-12
    grid = o.e4m3_value(rng.integers(0, 127, 256).astype(np.uint8))
    grid[0] = 448.0
    code, scale, _ = o.quantise(grid, rng.integers(0, 65536, 256), False)
    assert np.array_equal(o.e4m3_value(code) * scale[0], grid)


def test_noise_of_the_three_roundings_is_that_of_other_elements():
    u = o.rounding_noise(64, 5, 2, 77)
    assert u.shape == (8, 8) and u.min() >= 0 and u.max() < 65536
    assert np.array_equal(o.noise_for(64, 5, 2, 77, 4).reshape(8, 8)[:, :4], u[:, 4:])
    assert np.array_equal(o.noise_for(61, 5, 2, 77, 2), np.roll(u, -2, axis=1).reshape(-1)[:61])


def test_adamw_first_step_is_the_sign_of_the_gradient():
    g = np.array([3.0, -1e-3, 0.0])
    w, m, v = o.adamw(np.array([1.0, 1.0, 1.0]), g, np.zeros(3), np.zeros(3), 1, 0.1, eps=0.0 + 1e-30, decay=0.5)
    assert np.allclose(w, 1.0 - 0.05 - 0.1 * np.sign(g), rtol=1e-12)
    assert np.allclose(m, 0.1 * g) and np.allclose(v, 0.001 * g * g)


def test_adamw_matches_the_other_formulation_over_steps():
    # torch.optim.AdamW in fp64: decay first, then the step
    rng = np.random.default_rng(9)
    w = rng.normal(size=50)
    p = torch.nn.Parameter(torch.from_numpy(w.copy()))
    opt = torch.optim.AdamW([p], lr=1e-2, betas=(0.8, 0.95), eps=1e-6, weight_decay=0.1)
    m, v = np.zeros(50), np.zeros(50)
    for t in range(1, 8):
        g = rng.normal(size=50)
        p.grad = torch.from_numpy(g)
        opt.step()
        w, m, v = o.adamw(w, g, m, v, t, 1e-2, 0.8, 0.95, 1e-6, 0.1)
        assert np.allclose(p.detach().numpy(), w, rtol=1e-11, atol=1e-13)
