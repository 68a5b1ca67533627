"""What the microscaled reference itself rests on: the formats' printed values, and gradients against differences (no GPU)."""
import numpy as np
import pytest

import mx_reference as R


def test_printed_values_of_the_4_bit_form():
    # the largest value 6 gives e = 2, so s = 0: the grid itself, its ties, and what saturates
    x = np.array([[6, 0.5, 1, 1.5, 2, 3, 4, -6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 0.250001, -0.25, 5.01]])
    codes, scales = R.encode(x, 4)
    assert scales.tolist() == [[127]]
    assert R.decode(codes, scales, 4).tolist() == [[6, 0.5, 1, 1.5, 2, 3, 4, -6, 0, 1, 1, 2, 2, 4, 4, 0.5, 0, 6]]
    assert R.quantised(np.array([[7.9, 0.9]]), 4).tolist() == [[6, 1]]


def test_printed_values_of_the_8_bit_form():
    x = np.array([[1.0, 1.5 / 64, 2.5 / 64, -1.999, 1.999, 1 / 128]])
    assert (64 * R.quantised(x, 8)).tolist() == [[64, 2, 2, -127, 127, 0]]


@pytest.mark.parametrize("bits", (4, 8))
def test_scales(bits):
    down = 2 if bits == 4 else 0
    for e in (-149, -130, -126, -125, -1, 0, 5, 127):
        _, s = R.encode(np.array([[2.0 ** e]]), bits)
        assert s[0, 0] == max(e - down, -127) + 127
    _, s = R.encode(np.array([[0.0] * 32 + [np.nan] + [1.0] * 31 + [np.inf]]), bits)
    assert s.tolist() == [[0, 255, 255]]


@pytest.mark.parametrize("bits", (4, 8))
def test_error_is_at_most_half_a_step(bits):
    x = np.random.default_rng(1).standard_normal((16, 96))
    q = R.quantised(x, bits)
    top = np.repeat(np.abs(x).reshape(16, 3, 32).max(2), 32, 1)
    power = 2.0 ** np.floor(np.log2(top))
    # steps: 8 bits 1/64 of the power; 4 bits 1/2 of it at the top, and 7/4 to 2 of it saturate at 3/2 (6/4)
    assert np.all(np.abs(q - x) <= (power / 128 * (1 + 1e-12) if bits == 8 else power / 2))


@pytest.mark.parametrize("name", ("silu", "gelu"))
def test_slope_is_the_differences(name):
    v, h = np.linspace(-9, 9, 181), 1e-5
    d = (R.function(name, v + h) - R.function(name, v - h)) / (2 * h)
    assert np.max(np.abs(d - R.slope(name, v))) < 1e-9


def test_norm_grad_is_the_differences():
    g = np.random.default_rng(2)
    x, dy, gamma, beta = g.standard_normal((3, 17)), g.standard_normal((3, 17)), g.standard_normal(17), g.standard_normal(17)
    loss = lambda x, gamma, beta: (R.norm(x, gamma, beta, 1e-5)[0] * dy).sum()      # noqa: E731
    _, mean, rstd = R.norm(x, gamma, beta, 1e-5)
    dx, dgamma, dbeta = R.norm_grad(dy, x, mean, rstd, gamma)
    h = 1e-6
    for i in range(3):
        for j in range(17):
            e = np.zeros_like(x)
            e[i, j] = h
            assert abs((loss(x + e, gamma, beta) - loss(x - e, gamma, beta)) / (2 * h) - dx[i, j]) < 1e-7
    for j in range(17):
        e = np.zeros(17)
        e[j] = h
        assert abs((loss(x, gamma + e, beta) - loss(x, gamma - e, beta)) / (2 * h) - dgamma[j]) < 1e-7
        assert abs((loss(x, gamma, beta + e) - loss(x, gamma, beta - e)) / (2 * h) - dbeta[j]) < 1e-7
