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


def test_kept_values_by_hand():
    x = np.zeros((3, 34))
    x[0, :4] = [64.0, -0.4, 0.5, 1.5]       # step 1: ties to even, nothing becomes zero
    x[0, 32:] = [127.75, 3e-3]              # step 1 again: 128 does not fit 8 bits
    x[1, 0], x[1, 33] = np.inf, -2.0 ** -140  # the smallest step is 2^-126
    q, e = orc.keep(x)
    assert q[0, :5].tolist() == [64, -1, 1, 2, 0] and q[0, 32:].tolist() == [127, 1] and e[0].tolist() == [0, 0]
    assert e[1].tolist() == [128, -126] and not q[1, :32].any() and q[1, 33] == -1 and not q[2].any()
    v = orc.kept_values(q, e)
    assert np.isnan(v[1, :32]).all() and v[1, 33] == -(2.0 ** -126) and v[0, 1] == -1


def test_kept_values_are_within_a_step_and_keep_the_sign():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((200, 70)) * np.exp2(rng.integers(-100, 100, (200, 1)))
    q, e = orc.keep(x)
    v, step = orc.kept_values(q, e), np.repeat(np.ldexp(1.0, e), 32, axis=1)[:, :70]
    assert np.all(np.abs(v - x) <= step) and np.array_equal(np.sign(v), np.sign(x))
    plain = (np.abs(x) >= step / 2) & (np.abs(x) <= 127.5 * step)
    assert np.all(np.abs(v - x)[plain] <= step[plain] / 2)


def test_weight_and_relu_gradients_are_the_slopes():
    """Of a loss that is linear in Y = X~ W, and in relu(Z) with X~ = relu(Z) kept."""
    rng = np.random.default_rng(2)
    z, w, dy, v = rng.standard_normal((9, 40)), rng.standard_normal((40, 5)), rng.standard_normal((9, 5)), rng.standard_normal((40, 5))
    q, e = orc.keep(np.maximum(z, 0))
    x = orc.kept_values(q, e)
    assert (orc.weight_grad(q, e, dy) * v).sum() == pytest.approx(_slope(lambda t: (x @ t * dy).sum(), w, v), rel=1e-7)
    g, u = rng.standard_normal(z.shape), rng.standard_normal(z.shape)
    assert (orc.relu_backward(q, e, g) * u).sum() == pytest.approx(_slope(lambda t: (np.maximum(t, 0) * g).sum(), z, u, 1e-9), rel=1e-5)


@pytest.mark.parametrize("n,c", [(1, 2), (4, 7), (3, 50)])
def test_log_probability_gradient_is_the_slope(n, c):
    rng = np.random.default_rng(c)
    z, v = 2 * rng.standard_normal((n, c)), rng.standard_normal((n, c))
    labels, a, h = rng.integers(-1, c, n), rng.standard_normal(n), rng.standard_normal(n)
    logp, entropy, stats, _, _ = orc.log_probs(z, labels)
    dz = orc.log_probs_backward(z, labels, stats, entropy, a, h)
    loss = lambda t: (orc.log_probs(t, labels)[0] * a + orc.log_probs(t, labels)[1] * h).sum()  # noqa: E731
    assert (dz * v).sum() == pytest.approx(_slope(loss, z, v), rel=1e-6, abs=1e-8)


def test_log_probabilities_by_hand():
    inf = np.inf
    z = np.array([[0.0, 0.0, 0.0], [np.log(3.0), 0.0, -inf], [-inf, -inf, -inf], [0.0, np.nan, 1.0], [inf, 0.0, 1.0], [5.0, 5.0, 6.0]])
    logp, entropy, stats, values, columns = orc.log_probs(z, [1, 0, 2, 0, 3, 7], top=4)
    assert np.allclose(logp[:2], [-np.log(3), np.log(0.75)]) and logp[2] == -inf and np.isnan(logp[3]) and logp[4] == 0 and logp[5] == 0
    assert np.allclose(entropy[:3], [np.log(3), np.log(4) - 0.75 * np.log(3), 0]) and np.isnan(entropy[3:5]).all()
    assert np.allclose(stats[:2], [[0, np.log(3)], [np.log(3), np.log(4 / 3)]]) and (stats[2] == -inf).all() and np.isnan(stats[3:5]).all()
    assert columns.tolist() == [[0, 1, 2, -1], [0, 1, -1, -1], [-1] * 4, [-1] * 4, [-1] * 4, [2, 0, 1, -1]]
    assert np.allclose(values[1, :2], np.log([0.75, 0.25])) and (values[1, 2:] == -inf).all() and np.isnan(values[3]).all()
    dz = orc.log_probs_backward(z[:3], [1, 0, 2], stats[:3], entropy[:3], [1.0, 1.0, 1.0], [0.0, 0.0, 1.0])
    assert np.allclose(dz, [[-1 / 3, 2 / 3, -1 / 3], [0.25, -0.25, 0], [0, 0, 0]])
