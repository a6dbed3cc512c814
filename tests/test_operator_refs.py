"""The definitions that the operators' GPU tests compare with, held to differences and to the spectrum."""
import numpy as np
import pytest

import _operator_refs as R


@pytest.mark.parametrize("kind", ["none", "relu", "silu"])
@pytest.mark.parametrize("shape,groups", [((1, 1, 1, 2), 1), ((2, 2, 3, 6), 3), ((1, 2, 4, 4), 4)])
def test_groupnorm_gradients_are_those_of_differences(shape, groups, kind):
    rng = np.random.default_rng(3)
    x, dy = rng.standard_normal(shape), rng.standard_normal(shape)
    gamma, beta = 1 + 0.2 * rng.standard_normal((shape[0], shape[3])), 0.2 * rng.standard_normal((shape[0], shape[3]))
    eps = 1e-2

    def loss(x, gamma, beta):
        return (R.gn_forward(x, gamma, beta, groups, eps, kind)[0] * dy).sum()

    _, mean, rstd, z = R.gn_forward(x, gamma, beta, groups, eps, kind)
    assert np.abs(z).min() > 1e-3  # ReLU's corner is not between the two points of a difference
    got = R.gn_backward(x, dy, gamma, beta, mean, rstd, groups, kind)[:3]
    h = 1e-6
    for i, (arr, grad) in enumerate(zip((x, gamma, beta), got)):
        for at in np.ndindex(arr.shape):
            lo, hi = arr.copy(), arr.copy()
            lo[at] -= h
            hi[at] += h
            args = [[x, gamma, beta], [x, gamma, beta]]
            args[0][i], args[1][i] = hi, lo
            d = (loss(*args[0]) - loss(*args[1])) / (2 * h)
            assert abs(d - grad[at]) <= 1e-6 * max(1, abs(d)) + 2e-8 / h * 1e-6, (i, at)


@pytest.mark.parametrize("rows,cols", [(5, 5), (4, 9), (9, 4), (1, 7), (7, 1)])
def test_direction_is_the_quintic_of_the_singular_values(rows, cols):
    rng = np.random.default_rng(rows * 16 + cols)
    x = rng.standard_normal((2, rows, cols))
    x[1] = 0
    o = R.direction(x, 5)
    u, s, vt = np.linalg.svd(x[0], full_matrices=False)
    s = s / np.sqrt((s ** 2).sum())
    for _ in range(5):
        s = R.A * s + R.B * s ** 3 + R.C * s ** 5
    assert np.abs(o[0] - (u * s) @ vt).max() <= 1e-9  # 3.4445^5 of 64-bit roundings, with room
    assert not o[1].any()
