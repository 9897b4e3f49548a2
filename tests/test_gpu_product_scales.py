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


# sizes of dH, U, X and the weights: dG and dU beyond fp16's largest value, below its smallest, of one entry alone beyond it, and as they usually are; the gradients can be held in all of them
SLOPES = {"large": (300.0, 300.0, 1e-4, 1e-3), "tiny": (2.0 ** -14, 2.0 ** -12, 512.0, 512.0), "small": (2.0 ** -18, 1.0, 1.0, 1.0), "usual": (0.01, 1.0, 1.0, 0.2), "near one": (1.0, 1.0, 1.0, 0.2)}


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("sizes", SLOPES)
@pytest.mark.parametrize("n,k,m,act", [(20003, 65, 47, "relu"), (9001, 17, 300, "silu"), (5000, 64, 264, "gelu"), (4100, 136, 1024, "silu")])
def test_slopes_of_a_gated_layer_of_any_size(env, name, sizes, n, k, m, act):  # noqa: F811
    torch, cbm = env
    of_dh, of_u, of_x, of_w = SLOPES[sizes]
    rng = np.random.default_rng(n + len(sizes))
    dH, X, Wg, Wu, G, U_ = (_matrix(torch, s * rng.standard_normal(shape), name, 0)[0]
                            for s, shape in ((of_dh, (n, m)), (of_x, (n, k)), (of_w, (k, m)), (of_w, (k, m)), (2.0, (n, m)), (of_u, (n, m))))
    outs = [torch.empty_like(t) for t in (X, Wg, Wu)]
    ws = torch.full((cbm.cbm_gated_linear_backward_workspace_bytes(n, k, m, X.dtype),), 255, dtype=torch.uint8, device="cuda")
    cbm.cbm_gated_linear_backward(dH, X, Wg, Wu, G, U_, *outs, activation=act, workspace=ws)
    dh, x, wg, wu, g, u = (_numbers(t) for t in (dH, X, Wg, Wu, G, U_))
    dx, dwg, dwu, dg, du = orc.gated_linear_backward(dh, x, wg, wu, g, u, act)
    assert max(np.abs(v).max() for v in (dx, dwg, dwu)) < 60000  # (fp16 holds the gradients)
    # the activation: exp's argument is off by |g| 2^-24 of it, erfc's by g^2 2^-23; the type's rounding, where fp16's smallest values are those of the largest slope at 2^3
    of = (np.abs(g) + (np.minimum(g * g, 64.0) if act == "gelu" else 0.0) + 16) * 2 * U * (np.abs(g) + 1)
    least = 2.0 ** -28 * max(np.abs(dg).max(), np.abs(du).max()) if name == "f16" else 0.0
    half = ROUNDING[name]
    of_dg, of_du = (b + half * (np.abs(v) + b) + least for v, b in ((dg, np.abs(dh * u) * of + 3 * U * np.abs(dg)), (du, np.abs(dh) * of + 2 * U * np.abs(du))))
    bound = sum(SUM(2 * m + 128) * ((np.abs(v) + o) @ np.abs(w.T)) + o @ np.abs(w.T) for v, o, w in ((dg, of_dg, wg), (du, of_du, wu)))
    _near(outs[0], dx, _rounded(dx, bound, name))
    for got, want, v, o in ((outs[1], dwg, dg, of_dg), (outs[2], dwu, du, of_du)):
        _near(got, want, _rounded(want, SUM(n) * (np.abs(x.T) @ (np.abs(v) + o)) + np.abs(x.T) @ o, name))


@pytest.mark.parametrize("n,k,m", [(9001, 17, 300), (4100, 136, 1024)])
def test_slopes_of_a_gated_layer_that_are_not_finite_or_nothing(env, n, k, m):  # noqa: F811
    """In fp16: rows without such a slope come out as if there were none, whatever the others' size, and slopes of zero give zeros."""
    torch, cbm = env
    rng = np.random.default_rng(n)
    dH, X, Wg, Wu, G, U_ = (_matrix(torch, s * rng.standard_normal(shape), "f16", 0)[0]
                            for s, shape in ((1e-4, (n, m)), (1.0, (n, k)), (0.2, (k, m)), (0.2, (k, m)), (2.0, (n, m)), (1.0, (n, m))))
    ws = torch.empty(cbm.cbm_gated_linear_backward_workspace_bytes(n, k, m, X.dtype), dtype=torch.uint8, device="cuda")
    rows = torch.ones(n, dtype=torch.bool, device="cuda")
    rows[[3, n - 1]] = False
    some = []
    for bad in (0.0, math.nan, math.inf):
        dH[[3, n - 1]] = bad
        outs = [torch.ones_like(t) for t in (X, Wg, Wu)]
        cbm.cbm_gated_linear_backward(dH, X, Wg, Wu, G, U_, *outs, workspace=ws)
        some.append(outs[0])
    assert torch.equal(some[0][rows], some[1][rows]) and torch.equal(some[0][rows], some[2][rows])
    assert not bool(some[0][~rows].any()) and not bool(some[1][~rows].isfinite().any()) and not bool(some[2][~rows].isfinite().any())
    assert bool(some[0][rows].isfinite().all()) and bool(some[0][rows].any())
    cbm.cbm_gated_linear_backward(dH.zero_(), X, Wg, Wu, G, U_, *outs, workspace=ws)
    assert not any(bool(t.any()) for t in outs)
