"""The fp64 oracle of the operators of gated recurrent blocks: gradients against differences, roundings against their definition."""
import numpy as np
import pytest
import torch

from oracle import blocks


def directional(f, at, along, step=1e-6):
    return (f(at + step * along) - f(at - step * along)) / (2 * step)


def test_norm_adjoint_is_the_derivative():
    rng = np.random.default_rng(0)
    x, r, g, dy, ds = (rng.standard_normal(s) for s in ((5, 13), (5, 13), 13, (5, 13), (5, 13)))
    s, y, rstd = blocks.norm_forward(x, r, g, 1e-3)

    def loss(x_, r_, g_):
        s_, y_, _ = blocks.norm_forward(x_, r_, g_, 1e-3)
        return (y_ * dy).sum() + (s_ * ds).sum()

    dx, dg = blocks.norm_adjoint(s, g, rstd, dy, ds)
    for k in range(3):
        along, gain = rng.standard_normal((5, 13)), rng.standard_normal(13)
        # (central differences with step 1e-6: 1e-12 of the third derivative and 1e-10 of rounding, for numbers of order 10)
        assert abs(directional(lambda t: loss(t, r, g), x, along) - (dx * along).sum()) < 1e-7
        assert abs(directional(lambda t: loss(x, t, g), r, along) - (dx * along).sum()) < 1e-7
        assert abs(directional(lambda t: loss(x, r, t), g, gain) - (dg * gain).sum()) < 1e-7


@pytest.mark.parametrize("sigmoid", [False, True])
def test_scan_adjoint_is_the_derivative(sigmoid):
    rng = np.random.default_rng(1)
    n, T, C = 3, 7, 4
    lengths = np.array([7, 0, 4])
    a = rng.standard_normal((n, T, C)) if sigmoid else rng.uniform(0.3, 1.1, (n, T, C))
    x, h0, dh, dhT = (rng.standard_normal(s) for s in ((n, T, C), (n, C), (n, T, C), (n, C)))

    def loss(a_, x_, h0_):
        h, hT = blocks.scan_forward(a_, x_, h0_, lengths, sigmoid)
        return (h * dh).sum() + (hT * dhT).sum()

    h, hT = blocks.scan_forward(a, x, h0, lengths, sigmoid)
    assert np.array_equal(hT[1], h0[1]) and not h[1].any() and not h[2, 4:].any()
    da, dx, dh0 = blocks.scan_adjoint(a, x, h, h0, lengths, dh, dhT, sigmoid)
    for _ in range(3):
        along, start = rng.standard_normal(a.shape), rng.standard_normal(h0.shape)
        assert abs(directional(lambda t: loss(t, x, h0), a, along) - (da * along).sum()) < 1e-7
        assert abs(directional(lambda t: loss(a, t, h0), x, along) - (dx * along).sum()) < 1e-7
        assert abs(directional(lambda t: loss(a, x, t), h0, start) - (dh0 * start).sum()) < 1e-7


def test_codes_round_as_the_format_does():
    values = torch.cat([torch.linspace(-448, 448, 20001), torch.linspace(-0.05, 0.05, 20001)])
    got = blocks.round_e4m3(values.double().numpy())
    assert np.array_equal(got, values.to(torch.float8_e4m3fn).view(torch.uint8).numpy())
    table = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(blocks.e4m3_values(), table, equal_nan=True)


def test_scales_are_the_smallest_that_hold_the_block():
    for top, byte in ((448.0, 127), (449.0, 128), (224.0, 126), (0.0, 1), (2.0 ** -140, 1), (np.inf, 255)):
        assert blocks.scale_byte(np.array([top, -top / 3, 0.0])) == byte
    assert blocks.scale_byte(np.array([np.nan, 448.0])) == 127


def test_adamw_follows_the_gradient_of_a_parabola():
    p, m, v = np.full(3, 2.0), np.zeros(3), np.zeros(3)
    for t in range(1, 400):
        p, m, v = blocks.adamw(p, 2 * p, m, v, 0.05, 0.9, 0.99, 1e-8, 0.0, t)
    assert np.abs(p).max() < 1e-2
    q, _, _ = blocks.adamw(np.full(1, 2.0), np.zeros(1), np.zeros(1), np.zeros(1), 0.1, 0.9, 0.99, 1e-8, 0.5, 1)
    assert q[0] == pytest.approx(2.0 * 0.95)  # decay alone
