"""Slopes that are kept in 16 bits between the products of a backward pass: what decides their size, at sizes whose products are not small (those keep slopes in fp32), against 64 bits."""
import math

import numpy as np
import pytest

from oracle import train_oracle as orc
from test_gpu_gated_linear import SUM, TYPES, _near, _rounded
from test_gpu_layer_norm import ROUNDING, _matrix, _numbers, env  # noqa: F401

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def _classes(torch, n, d, c, name):
    rng = np.random.default_rng(n + d + c)
    X, W = _matrix(torch, rng.standard_normal((n, d)), name, 0)[0], _matrix(torch, 3 * rng.standard_normal((d, c)) / math.sqrt(d), name, 0)[0]
    labels = rng.integers(0, c, n)
    labels[::3], labels[1::7] = -1, c
    return rng, X, W, torch.from_numpy(labels).cuda()


def _classes_backward(torch, cbm, X, W, L, stats, dlogp):
    dX, dW = torch.empty_like(X), torch.empty_like(W)
    ws = torch.full((cbm.cbm_linear_log_probs_backward_workspace_bytes(X.shape[0], *W.shape, X.dtype),), 255, dtype=torch.uint8, device="cuda")
    cbm.cbm_linear_log_probs_backward(X, W, L, stats, dlogp, dX, dW, workspace=ws)
    return dX, dW


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("n,d,c", [(9001, 17, 300), (20003, 65, 47), (70001, 9, 20), (2304, 320, 4096)])
def test_rows_without_a_label_or_a_distribution_say_nothing_about_the_rest(env, name, n, d, c):  # noqa: F811
    """Their dlogp is as large as it may be, or infinite: the same bits as with zeros there, and those are the gradients."""
    torch, cbm = env
    rng, X, W, L = _classes(torch, n, d, c, name)
    labels = L.cpu().numpy()
    stats = torch.from_numpy(orc.log_probs(_numbers(X) @ _numbers(W), labels)[2].astype(np.float32)).cuda()
    nothing = np.zeros(n, dtype=bool)
    nothing[5::11] = True  # rows with a label of which every class is ruled out
    stats[torch.from_numpy(nothing).cuda()] = -math.inf
    given = (labels >= 0) & (labels < c) & ~nothing
    a = np.where(given, rng.uniform(-1.5e-4, -0.5e-4, n), 0.0).astype(np.float32)
    want = _classes_backward(torch, cbm, X, W, L, stats, torch.from_numpy(a).cuda())
    for large in (1e9, 3e38, math.inf):
        got = _classes_backward(torch, cbm, X, W, L, stats, torch.from_numpy(np.where(given, a, np.float32(large))).cuda())
        assert all(torch.equal(p, q) for p, q in zip(got, want))
    x, w, st = _numbers(X), _numbers(W), _numbers(stats)
    z = x @ w
    with np.errstate(invalid="ignore"):
        p = np.where(given[:, None], np.exp(z - st[:, :1] - st[:, 1:]), 0.0)
        away = np.where(given[:, None], np.abs(z - st[:, :1]) + np.abs(st[:, 1:]), 0.0)
    hot = np.zeros((n, c))
    hot[np.flatnonzero(given), labels[given]] = 1.0
    dz = a.astype(np.float64)[:, None] * (hot - p)
    # p: its score, three roundings of the exponent, exp2's unit in the last place; two roundings of the difference; the type's, where fp16's smallest values are those of 2^15 over the largest |dlogp|
    size = np.abs(a).astype(np.float64)[:, None] * (1.01 * p * (SUM(d) * (np.abs(x) @ np.abs(w)) + 6 * U * away + 4 * U) + 2 * U) + 2 * U * np.abs(dz)
    least = 2.0 ** -25 * 2.0 ** -15 * float(np.abs(a).max()) if name == "f16" else 0.0
    off = given[:, None] * (size + ROUNDING[name] * (np.abs(dz) + size) + least)
    _near(want[0], dz @ w.T, _rounded(dz @ w.T, SUM(c) * ((np.abs(dz) + off) @ np.abs(w.T)) + off @ np.abs(w.T), name))
    _near(want[1], x.T @ dz, _rounded(x.T @ dz, SUM(n) * (np.abs(x.T) @ (np.abs(dz) + off)) + np.abs(x.T) @ off, name))
