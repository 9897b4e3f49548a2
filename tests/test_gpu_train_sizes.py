"""The operators between the products at sizes where work is dealt out otherwise: more rows than a grid has at once, few rows of thousands of columns, shares of the rows
that do not divide, as many equal scores as there is room for.  Bounds are those of the tests beside it."""
import numpy as np
import pytest

from oracle import train_oracle as orc
from test_gpu_checkpoint import _grad, _kept, _room
from test_gpu_layer_norm import DEPTH, ROUNDING, U, _forward_bound, _matrix, _numbers, _untouched, env  # noqa: F401
from test_gpu_log_probs import _check, _scores

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,k,name", [(600001, 1, "f32"), (600001, 3, "f32"), (600001, 4, "f32"), (300001, 5, "f16"), (600001, 8, "bf16"), (70001, 20, "f32"), (300, 16161, "bf16"),
                                      (515, 8200, "f32"), (1100, 5561, "f16")])
def test_layer_norm(env, n, k, name):  # noqa: F811
    torch, cbm = env
    rng = np.random.default_rng(n + k)
    X, _ = _matrix(torch, rng.standard_normal((n, k)) + 0.7, name, 1)
    Y, whole = _matrix(torch, np.zeros((n, k)), name, 3)
    gamma, beta = (torch.from_numpy(rng.standard_normal(k).astype(np.float32)).cuda() for _ in range(2))
    mean, rstd = (torch.full((n,), np.nan, device="cuda") for _ in range(2))
    cbm.cbm_layer_norm(X, gamma, beta, 1e-5, Y, mean, rstd)
    x, g = _numbers(X), _numbers(gamma)
    y, m, r = orc.layer_norm(x, g, _numbers(beta), float(np.float32(1e-5)))
    by, bm, br = _forward_bound(x, (y, (x - m[:, None]) * r[:, None]), m, r, g, name)
    assert np.all(np.abs(_numbers(Y) - y) <= by) and np.all(np.abs(_numbers(mean) - m) <= bm) and np.all(np.abs(_numbers(rstd) - r) <= br)
    _untouched(torch, Y, whole, 0)


# both sides of every size at which sums go into the same launch, and more partial sums than slices of a join
@pytest.mark.parametrize("n,k,name", [(208, 12062, "bf16"), (217, 12100, "f32"), (1024, 2560, "bf16"), (1025, 2560, "f32"), (1024, 2561, "f16"), (2048, 256, "f32"), (2049, 256, "f16"),
                                      (2048, 257, "bf16"), (600, 16160, "bf16"), (70, 20001, "f16"), (40001, 3, "f32"), (40001, 8, "bf16")])
def test_layer_norm_backward(env, n, k, name):  # noqa: F811
    torch, cbm = env
    rng = np.random.default_rng(n + k)
    X, _ = _matrix(torch, rng.standard_normal((n, k)) + 0.7, name, 1)
    dY, _ = _matrix(torch, rng.standard_normal((n, k)), name, 2)
    dX, whole = _matrix(torch, np.zeros((n, k)), name, 3)
    gamma = torch.from_numpy(rng.standard_normal(k).astype(np.float32)).cuda()
    x, dy, g = _numbers(X), _numbers(dY), _numbers(gamma)
    _, m, r = orc.layer_norm(x, eps=1e-5)
    mean, rstd = (torch.from_numpy(a.astype(np.float32)).cuda() for a in (m, r))
    dgamma, dbeta = (torch.full((k,), np.nan, device="cuda") for _ in range(2))
    workspace = torch.full((cbm.cbm_layer_norm_workspace_bytes(n, k),), 255, dtype=torch.uint8, device="cuda")
    cbm.cbm_layer_norm_backward(dY, X, gamma, mean, rstd, dX, dgamma, dbeta, workspace)
    dx, dg, db = orc.layer_norm_backward(dy, x, g, _numbers(mean), _numbers(rstd))
    h, u = (x - _numbers(mean)[:, None]) * _numbers(rstd)[:, None], dy * g
    size = np.abs(u) + np.abs(u).mean(axis=1, keepdims=True) + np.abs(h) * np.abs(u * h).mean(axis=1, keepdims=True)
    bound = _numbers(rstd)[:, None] * (DEPTH + 20) * U * size
    assert np.all(np.abs(_numbers(dX) - dx) <= bound + ROUNDING[name] * (np.abs(dx) + bound) + (2.0 ** -25 if name == "f16" else 0.0))
    # at most n / 16 + 64 additions on the way of a row's share into a column's sum
    depth = 10 + min(n, max(150, n / 16 + 64))
    assert np.all(np.abs(_numbers(dgamma) - dg) <= depth * U * np.abs(dy * h).sum(axis=0))
    assert np.all(np.abs(_numbers(dbeta) - db) <= depth * U * np.abs(dy).sum(axis=0))
    _untouched(torch, dX, whole, 0)


@pytest.mark.parametrize("n,k,name", [(300000, 7, "f32"), (300001, 8, "bf16"), (200001, 15, "f16"), (70001, 64, "f32"), (45003, 100, "f32"), (70001, 33, "f32"), (30001, 200, "f32")])
def test_kept_and_restored(env, n, k, name):  # noqa: F811
    torch, cbm = env
    rng = np.random.default_rng(n + k)
    X, _ = _matrix(torch, rng.standard_normal((n, k)) * np.exp2(rng.integers(-12, 8, (n, 1))), name, 1)
    Q, E, wq, we = _room(torch, n, k, 3)
    cbm.cbm_checkpoint_save(X, Q, E)
    q, e = orc.keep(_numbers(X))
    got_q, got_e = _kept(Q, E)
    assert np.array_equal(got_q, q) and np.array_equal(got_e, e)
    assert bool((wq[:, k:] == 77).all()) and bool((we[:, E.shape[1]:] == 77).all()), "wrote outside the columns"
    B, whole = _matrix(torch, np.zeros((n, k)), "f32", 2)
    cbm.cbm_checkpoint_restore(Q, E, B)
    assert np.array_equal(_numbers(B), orc.kept_values(q, e))
    _untouched(torch, B, whole, 0)
    dY, _ = _matrix(torch, rng.standard_normal((n, k)), name, 1)
    dX, whole = _matrix(torch, np.zeros((n, k)), name, 2)
    cbm.cbm_checkpoint_relu_backward(Q, E, dY, dX)
    assert np.array_equal(_numbers(dX), orc.relu_backward(q, e, _numbers(dY)))
    _untouched(torch, dX, whole, 0)


# tiles of 128 x 64 and less that do not divide the card, 2 to 512 shares
@pytest.mark.parametrize("name", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,k,c", [(13613, 323, 359), (114720, 13, 5), (40001, 60, 20), (2151, 207, 245), (6001, 572, 94), (3001, 884, 35), (1000, 1500, 900), (9001, 64, 33)])
def test_weight_gradient_of_whole_numbers_is_exact(env, name, n, k, c):  # noqa: F811
    torch, cbm = env
    rng = np.random.default_rng(n)
    q, e = rng.integers(-9, 10, (n, k)), rng.integers(-1, 2, (n, -(-k // 32)))  # products are multiples of 1/2; a sum's size is below 6 sqrt(n) 40 < 2^20
    Q, E, _, _ = _room(torch, n, k, 1)
    Q.copy_(torch.from_numpy(q))
    E.copy_(torch.from_numpy(e + 127))
    dY, _ = _matrix(torch, rng.integers(-8, 9, (n, c)).astype(np.float64), name, 1)
    assert np.array_equal(_grad(torch, cbm, Q, E, dY, c), orc.weight_grad(q, e, _numbers(dY)))


@pytest.mark.parametrize("name", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("c", [257, 513, 1024, 1025, 2047, 2048, 2049, 4096])
def test_as_many_equal_scores_as_there_is_room_for(env, name, c):  # noqa: F811
    torch, cbm = env
    rng = np.random.default_rng(c)
    z = rng.integers(-8, 0, (9, c)) / 4.0
    for row, equal in enumerate((1, 2, 31, 64, 255, 256, 257, c - 1)):
        z[row, rng.permutation(c)[:equal]] = 3.0
    z[8] = np.where(rng.random(c) < 0.9, -np.inf, 1.0)
    Z, _ = _matrix(torch, z, name, 1)
    labels = rng.integers(0, c, 9)
    for top in (1, 2, 20, 32):
        _check(torch, Z, labels, _scores(torch, cbm, Z, labels, top), top)


# a wave a row: many rows of more columns than stay in registers; the largest scores in a few lanes' columns, equal ones, masks
@pytest.mark.parametrize("n,c,name", [(1024, 2049, "f32"), (1500, 4096, "f32"), (1024, 4097, "f32"), (1025, 2049, "bf16"), (1024, 5003, "f16"), (1100, 8192, "bf16"), (1100, 8193, "f16")])
def test_many_rows_of_scores(env, n, c, name):  # noqa: F811
    torch, cbm = env
    rng = np.random.default_rng(n + c)
    z = 3 * rng.standard_normal((n, c))
    z[::7] = rng.integers(-2, 3, z[::7].shape)
    z[1::7, : c // 2] = -np.inf
    z[2::7] = np.where(np.arange(c) % 512 < 8, 20.0 + rng.random(c), z[2::7])
    z[3], z[10], z[17, 5], z[24, 0] = 1.5, -np.inf, np.nan, np.inf
    z[31] = np.arange(c) / 512.0
    Z, _ = _matrix(torch, z, name, 3)
    labels = rng.integers(-1, c + 1, n)
    for top in (0, 1, 8, 32):
        _check(torch, Z, labels, _scores(torch, cbm, Z, labels, top), top)
