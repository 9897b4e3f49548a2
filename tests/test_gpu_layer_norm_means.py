"""Layer norm of rows whose mean has no exact sum: equal values, and values that differ by a few units of their last place."""
import numpy as np
import pytest

from oracle import train_oracle as orc
from test_gpu_layer_norm import DEPTH, U, _matrix, _numbers, env  # noqa: F401

pytestmark = pytest.mark.gpu
EPS = float(np.float32(1e-5))


@pytest.mark.parametrize("name", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("k", [3, 5, 7, 33, 100, 300, 500, 1000, 3001, 4095, 8191, 12289, 16383, 20001, 70001])
def test_equal_values_come_out_as_beta(env, name, k):  # noqa: F811
    """A sum of k equal values is off by up to DEPTH units of its last place, and the mean with it; the deviations from that mean are whole units, and so is their sum (90 x 70,001 < 2^24), so
    their mean is exact, and nothing is left of them."""
    torch, cbm = env
    rng = np.random.default_rng(k)
    X, _ = _matrix(torch, np.repeat([[0.1], [3000.1], [30000.1], [-1e-3], [7 / 3]], k, axis=1), name, 3)
    gamma, beta = (torch.from_numpy(rng.standard_normal(k).astype(np.float32)).cuda() for _ in range(2))
    Y, mean, rstd = torch.empty_like(X), torch.empty(5, device="cuda"), torch.empty(5, device="cuda")
    cbm.cbm_layer_norm(X, gamma, beta, 1e-5, Y, mean, rstd)
    assert torch.equal(Y, beta.to(X.dtype).expand(5, k)) and torch.equal(mean, X[:, 0].float())
    off = (DEPTH * U * np.abs(_numbers(mean))) ** 2  # squares of the deviations from the first mean, added up with DEPTH roundings
    assert np.all(np.abs(_numbers(rstd) * EPS ** 0.5 - 1) <= 0.5 * (DEPTH + 4) * U * off / EPS + 4 * U)


@pytest.mark.parametrize("k", [3, 7, 33, 100, 500, 1000, 4095])
def test_equal_values_without_eps_have_no_norm(env, k):  # noqa: F811
    """Nothing is left of the deviations, as above, so the variance is 0."""
    torch, cbm = env
    X = torch.tensor([0.1, 3000.1, 30000.1, -1e-3], device="cuda")[:, None].expand(4, k).contiguous()
    Y, rstd = torch.empty_like(X), torch.empty(4, device="cuda")
    cbm.cbm_layer_norm(X, None, None, 0.0, Y, None, rstd)
    assert bool(Y.isnan().all()) and bool(rstd.isinf().all())


@pytest.mark.parametrize("k", [5, 33, 100, 500, 1000, 3001, 8191, 16383, 20001, 70001])
def test_deviations_of_a_few_units_of_the_last_place(env, k):  # noqa: F811
    """The mean's error e goes into neither the deviations (but for DEPTH roundings of it) nor the variance (but for DEPTH roundings of e^2)."""
    torch, cbm = env
    rng = np.random.default_rng(k)
    base = np.float32(30000.1)
    x = base + rng.integers(-3, 4, (6, k)) * float(np.spacing(base))
    X, _ = _matrix(torch, x, "f32", 1)
    Y, mean, rstd = torch.empty_like(X), torch.empty(6, device="cuda"), torch.empty(6, device="cuda")
    cbm.cbm_layer_norm(X, None, None, 1e-5, Y, mean, rstd)
    x = _numbers(X)
    y, m, r = orc.layer_norm(x, eps=EPS)
    e, var = DEPTH * U * np.abs(m), r ** -2.0
    rel = 0.5 * (DEPTH + 6) * U * (1 + e * e / var) + 4 * U
    of_mean = (DEPTH + 4) * U * (np.abs(x - m[:, None]).mean(axis=1) + e)  # of the deviations' mean
    assert np.all(np.abs(_numbers(rstd) - r) <= rel * r)
    assert np.all(np.abs(_numbers(mean) - m) <= of_mean + U * np.abs(m))
    assert np.all(np.abs(_numbers(Y) - y) <= (of_mean * r)[:, None] + np.abs(y) * (rel + 4 * U)[:, None])


@pytest.mark.parametrize("k", [5, 100, 1000, 5000, 20001])
def test_the_mean_of_a_row_that_is_not_finite(env, k):  # noqa: F811
    """What the definition gives: an infinity of one sign is the mean, anything else that is not finite has none; values near the type's largest keep theirs."""
    torch, cbm = env
    X = torch.randn((5, k), device="cuda")
    X[0, 0], X[1, k - 1], X[2, k // 2] = float("inf"), float("-inf"), float("nan")
    X[3, 0] = torch.finfo(torch.float32).min
    X[3, 1:] = 0.0
    Y, mean, rstd = torch.empty_like(X), torch.empty(5, device="cuda"), torch.empty(5, device="cuda")
    cbm.cbm_layer_norm(X, None, None, 1e-5, Y, mean, rstd)
    assert float(mean[0]) == float("inf") and float(mean[1]) == float("-inf") and bool(mean[2].isnan())
    assert bool(Y[:3].isnan().all()) and bool(rstd[:3].isnan().all())
    # the variance passes the largest value: r = 0
    assert float(mean[3]) == pytest.approx(torch.finfo(torch.float32).min / k, rel=1e-6) and float(rstd[3]) == 0.0 and not bool(Y[3].any())
    assert bool(Y[4].isfinite().all())


@pytest.mark.parametrize("k", [3, 7, 100, 1000, 3001, 16383, 65535])
def test_equal_values_of_any_size_that_the_header_names(env, k):  # noqa: F811
    torch, cbm = env
    X = (torch.tensor([1.1, -1.9, 4 / 3], device="cuda")[:, None] * torch.tensor([2.0 ** -50, 2.0 ** -30, 1.0, 2.0 ** 40, 2.0 ** 69], device="cuda")).reshape(-1, 1).expand(15, k).contiguous()
    Y, mean, rstd = torch.empty_like(X), torch.empty(15, device="cuda"), torch.empty(15, device="cuda")
    cbm.cbm_layer_norm(X, None, None, 1e-5, Y, mean, rstd)
    assert not bool(Y.any()) and torch.equal(mean, X[:, 0])
    cbm.cbm_layer_norm(X, None, None, 0.0, Y, None, rstd)
    assert bool(Y.isnan().all()) and bool(rstd.isinf().all())


@pytest.mark.parametrize("name", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("k", [2, 3, 5, 8, 9, 17, 33, 64, 100, 129, 257, 300, 500, 512])
def test_a_corrected_row_leaves_the_others_their_bits(env, name, k):  # noqa: F811
    """Rows that share a wave with one whose mean is corrected come out as they do without it."""
    torch, cbm = env
    rng = np.random.default_rng(k)
    x = rng.standard_normal((200, k)) * 3 + 0.7
    X, _ = _matrix(torch, x, name, 0)
    x[::9] = 1000.1 + rng.standard_normal((23, k))
    other, _ = _matrix(torch, x, name, 0)
    got = []
    for t in (X, other):
        Y, mean, rstd = torch.empty_like(t), torch.empty(200, device="cuda"), torch.empty(200, device="cuda")
        cbm.cbm_layer_norm(t, None, None, 1e-5, Y, mean, rstd)
        got.append((Y, mean, rstd))
    rest = torch.arange(200, device="cuda") % 9 != 0
    assert all(torch.equal(a[rest], b[rest]) for a, b in zip(*got))
