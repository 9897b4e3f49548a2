"""The 64-bit definitions of the operators between the products: gradients against differences, values against what can be said by hand."""
import numpy as np
import pytest

from oracle import train_oracle as orc


def _slope(f, x, v, h=1e-5):
    """d f(x + t v) / dt at t = 0, by central differences in 64 bits."""
    return (f(x + h * v) - f(x - h * v)) / (2 * h)


@pytest.mark.parametrize("n,k", [(1, 2), (3, 5), (7, 33)])
def test_layer_norm_gradient_is_the_slope(n, k):
    rng = np.random.default_rng(n * 100 + k)
    x, dy, v = (rng.standard_normal((n, k)) for _ in range(3))
    gamma, beta, w = (rng.standard_normal(k) for _ in range(3))
    _, m, r = orc.layer_norm(x, gamma, beta)
    dx, dgamma, dbeta = orc.layer_norm_backward(dy, x, gamma, m, r)
    loss = lambda x_, g_, b_: (orc.layer_norm(x_, g_, b_)[0] * dy).sum()  # noqa: E731
    # the error of a central difference is h^2 times a third derivative, below 1e-10 times (r^3 <= 3e7 for a row of two near values)
    assert (dx * v).sum() == pytest.approx(_slope(lambda t: loss(t, gamma, beta), x, v), rel=1e-5, abs=1e-6)
    assert (dgamma * w).sum() == pytest.approx(_slope(lambda t: loss(x, t, beta), gamma, w), rel=1e-7, abs=1e-8)
    assert (dbeta * w).sum() == pytest.approx(_slope(lambda t: loss(x, gamma, t), beta, w), rel=1e-7, abs=1e-8)


def test_layer_norm_by_hand():
    y, m, r = orc.layer_norm([[1.0, 3.0], [5.0, 5.0]], [2.0, 2.0], [0.5, 0.5], eps=0.25)
    assert np.allclose(m, [2, 5]) and np.allclose(r, [1.25 ** -0.5, 2.0])
    assert np.allclose(y, [[0.5 - 2 * 1.25 ** -0.5, 0.5 + 2 * 1.25 ** -0.5], [0.5, 0.5]])
