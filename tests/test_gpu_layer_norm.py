"""Layer norm forward and backward through the C ABI against the definition in 64 bits: every width at which a kernel's shape changes, types, strides, empty
inputs, values that are not finite, refusals."""
import ctypes
import math

import numpy as np
import pytest

from oracle import train_oracle as orc

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
ROUNDING = {"f32": U, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}  # half a unit of the last of 24, 8, 11 bits
# Additions on the way of one value into a row's sum: at most 64 in a lane (rows of up to 70,000 values), 6 in a wave, 16 over waves.
DEPTH = 90
WIDTHS = [1, 2, 3, 4, 5, 7, 8, 9, 15, 16, 17, 31, 32, 33, 47, 63, 64, 65, 100, 127, 128, 129, 255, 256, 257, 500, 511, 512, 513, 1000, 1023, 1024, 1025, 2047, 2048, 2049, 4095, 4096,
          4097, 8192, 8193, 16385, 40000, 70001]


@pytest.fixture(scope="module")
def env():
    import torch

    import paper_2409_02208_amd as cbm

    assert torch.cuda.is_available(), "this test needs the MI355X"
    return torch, cbm


def _type(torch, name):
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[name]


def _matrix(torch, values, name, pad, offset=0):
    """`values` as a device matrix of the type, with `pad` columns of NaN after each row and `offset` elements before the first."""
    n, k = values.shape
    whole = torch.full((offset + n * (k + pad),), math.nan, dtype=_type(torch, name), device="cuda")
    t = whole[offset:].view(n, k + pad)[:, :k]
    t.copy_(torch.from_numpy(np.ascontiguousarray(values, dtype=np.float32)))
    return t, whole


def _numbers(t):
    return t.double().cpu().numpy()


def _untouched(torch, t, whole, offset):
    n, k = t.shape
    rows = whole[offset:].view(n, -1)
    assert bool(rows[:, k:].isnan().all()) and bool(whole[:offset].isnan().all()), "wrote outside the columns"


def _forward_bound(x, y, m, r, gamma, name):
    x, g = np.abs(x), np.abs(gamma)
    dm = (DEPTH + 2) * U * x.mean(axis=1)
    var = (r ** -2.0)  # with eps in it
    rel = 0.5 * ((DEPTH + 6) * U + (dm * dm) / var) + 3 * U  # of r
    h = np.abs(y[1])
    bound = g * (dm * r)[:, None] * 1.01 + g * h * (rel + 4 * U)[:, None] + 2 * U * np.abs(y[0])
    return bound + ROUNDING[name] * (np.abs(y[0]) + bound) + (2.0 ** -25 if name == "f16" else 0.0), dm + U * np.abs(m), rel * r


@pytest.mark.parametrize("name", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("k", WIDTHS)
def test_forward(env, name, k):
    torch, cbm = env
    rng = np.random.default_rng(k)
    for n, pad, offset in ((1, 0, 0), (5, 3, 1), (67, 0, 0)) + (((2500, 8, 8),) if k <= 600 else ()):
        X, _ = _matrix(torch, rng.standard_normal((n, k)) + 0.7, name, pad, offset)
        Y, whole = _matrix(torch, np.zeros((n, k)), name, pad, offset)
        gamma, beta = (torch.from_numpy(rng.standard_normal(k).astype(np.float32)).cuda() for _ in range(2))
        mean, rstd = (torch.full((n,), math.nan, device="cuda") for _ in range(2))
        for g, b in ((gamma, beta), (None, beta), (gamma, None)):
            cbm.cbm_layer_norm(X, g, b, 1e-5, Y, mean, rstd)
            x, gn = _numbers(X), np.ones(k) if g is None else _numbers(g)
            y, m, r = orc.layer_norm(x, gn, None if b is None else _numbers(b), float(np.float32(1e-5)))
            by, bm, br = _forward_bound(x, (y, (x - m[:, None]) * r[:, None]), m, r, gn, name)
            assert np.all(np.abs(_numbers(Y) - y) <= by), (n, pad)
            assert np.all(np.abs(_numbers(mean) - m) <= bm) and np.all(np.abs(_numbers(rstd) - r) <= br), (n, pad)
            _untouched(torch, Y, whole, offset)
        first = Y.clone()
        cbm.cbm_layer_norm(X, gamma, None, 1e-5, Y)  # without statistics
        assert torch.equal(first, Y)


def test_large_means_keep_the_variance(env):
    """The second pass is over deviations: a mean of 3000 beside deviations of 1 costs the 2^-24 of the mean, not its square."""
    torch, cbm = env
    rng = np.random.default_rng(5)
    for k in (64, 100, 1000, 5000, 20000):
        X, _ = _matrix(torch, rng.standard_normal((9, k)) + 3000.0, "f32", 0)
        Y, mean, rstd = torch.empty_like(X), torch.empty(9, device="cuda"), torch.empty(9, device="cuda")
        cbm.cbm_layer_norm(X, None, None, 1e-5, Y, mean, rstd)
        y, m, r = orc.layer_norm(_numbers(X), eps=float(np.float32(1e-5)))
        by, _, br = _forward_bound(_numbers(X), (y, y), m, r, np.ones(k), "f32")
        assert np.all(np.abs(_numbers(Y) - y) <= by) and np.all(np.abs(_numbers(rstd) - r) <= br)
        assert by.max() < 0.04


def test_equal_values_and_no_eps(env):
    torch, cbm = env
    for k in (3, 8, 33, 300, 3000):
        X = torch.full((4, k), 2.0, device="cuda")
        X[1] = 0.0
        Y, beta = torch.empty_like(X), torch.arange(k, device="cuda", dtype=torch.float32)
        rstd = torch.empty(4, device="cuda")
        cbm.cbm_layer_norm(X, None, beta, 1e-5, Y, None, rstd)
        assert torch.equal(Y, beta.expand(4, k)) and torch.allclose(rstd, torch.full_like(rstd, 1e-5 ** -0.5))
        cbm.cbm_layer_norm(X, None, beta, 0.0, Y, None, rstd)
        assert bool(Y.isnan().all()) and bool(rstd.isinf().all())


@pytest.mark.parametrize("k", [5, 64, 100, 1000, 3001, 20001])
def test_values_that_are_not_finite_stay_in_their_row(env, k):
    torch, cbm = env
    X = torch.randn((6, k), device="cuda")
    clean = torch.empty_like(X)
    cbm.cbm_layer_norm(X, None, None, 1e-5, clean)
    X[1, k - 1], X[3, 0], X[4, k // 2] = math.nan, math.inf, -math.inf
    Y = torch.empty_like(X)
    cbm.cbm_layer_norm(X, None, None, 1e-5, Y)
    for row in range(6):
        assert bool(Y[row].isnan().all()) if row in (1, 3, 4) else torch.equal(Y[row], clean[row])
    dX, dY = torch.empty_like(X), torch.randn_like(X)
    mean, rstd = torch.zeros(6, device="cuda"), torch.ones(6, device="cuda")
    cbm.cbm_layer_norm_backward(dY, X, None, mean, rstd, dX, None, None, None)
    for row in range(6):
        assert bool(dX[row].isfinite().all()) == (row not in (1, 3, 4))


@pytest.mark.parametrize("name", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("k", WIDTHS)
def test_backward(env, name, k):
    torch, cbm = env
    rng = np.random.default_rng(k + 1)
    for n, pad, offset in ((1, 0, 0), (5, 3, 1), (67, 0, 0)) + (((5000, 8, 8),) if k <= 600 else ()):
        X, _ = _matrix(torch, rng.standard_normal((n, k)) + 0.7, name, pad, offset)
        dY, _ = _matrix(torch, rng.standard_normal((n, k)), name, pad + 1, offset)
        dX, whole = _matrix(torch, np.zeros((n, k)), name, pad, offset)
        gamma = torch.from_numpy(rng.standard_normal(k).astype(np.float32)).cuda()
        x = _numbers(X)
        _, m, r = orc.layer_norm(x)
        mean, rstd = (torch.from_numpy(a.astype(np.float32)).cuda() for a in (m, r))
        dgamma, dbeta = (torch.full((k,), math.nan, device="cuda") for _ in range(2))
        workspace = torch.full((cbm.cbm_layer_norm_workspace_bytes(n, k),), 255, dtype=torch.uint8, device="cuda")  # (NaN all over)
        for g in (gamma, None):
            cbm.cbm_layer_norm_backward(dY, X, g, mean, rstd, dX, dgamma, dbeta, workspace)
            gn = np.ones(k) if g is None else _numbers(g)
            dy = _numbers(dY)
            dx, dg, db = orc.layer_norm_backward(dy, x, gn, _numbers(mean), _numbers(rstd))
            r64 = _numbers(rstd)[:, None]
            h, u = (x - _numbers(mean)[:, None]) * r64, dy * gn
            size = np.abs(u) + np.abs(u).mean(axis=1, keepdims=True) + np.abs(h) * np.abs(u * h).mean(axis=1, keepdims=True)
            bound = r64 * (DEPTH + 20) * U * size
            assert np.all(np.abs(_numbers(dX) - dx) <= bound + ROUNDING[name] * (np.abs(dx) + bound) + (2.0 ** -25 if name == "f16" else 0.0)), (n, pad)
            # at most 80 rows a lane, 4 steps over a wave's rows, 8 waves, 16 + 32 partial sums
            assert np.all(np.abs(_numbers(dgamma) - dg) <= 150 * U * np.abs(dy * h).sum(axis=0)), (n, pad)
            assert np.all(np.abs(_numbers(dbeta) - db) <= 150 * U * np.abs(dy).sum(axis=0)), (n, pad)
            _untouched(torch, dX, whole, offset)
        # any of the outputs may be left out, and what is left has the same bits
        again, g2, b2 = torch.zeros_like(dX), torch.zeros_like(dgamma), torch.zeros_like(dbeta)
        cbm.cbm_layer_norm_backward(dY, X, None, mean, rstd, again, None, None, None)
        cbm.cbm_layer_norm_backward(dY, X, None, mean, rstd, None, g2, None, workspace)
        cbm.cbm_layer_norm_backward(dY, X, None, mean, rstd, None, None, b2, workspace)
        assert torch.equal(again, dX) and torch.equal(g2, dgamma) and torch.equal(b2, dbeta)


def test_gradient_is_the_slope_of_the_forward_pass(env):
    torch, cbm = env
    rng = np.random.default_rng(3)
    n, k = 40, 75
    x, dy, v = (rng.standard_normal((n, k)).astype(np.float32) for _ in range(3))
    gamma, beta, w = (rng.standard_normal(k).astype(np.float32) for _ in range(3))
    X, dY, G = (torch.from_numpy(a).cuda() for a in (x, dy, gamma))
    Y, dX = torch.empty_like(X), torch.empty_like(X)
    mean, rstd = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    dg, db = torch.empty(k, device="cuda"), torch.empty(k, device="cuda")
    cbm.cbm_layer_norm(X, G, torch.from_numpy(beta).cuda(), 1e-5, Y, mean, rstd)
    workspace = torch.empty(cbm.cbm_layer_norm_workspace_bytes(n, k), dtype=torch.uint8, device="cuda")
    cbm.cbm_layer_norm_backward(dY, X, G, mean, rstd, dX, dg, db, workspace)
    loss = lambda x_, g_, b_: (orc.layer_norm(x_, g_, b_)[0] * dy).sum()  # noqa: E731
    h = 1e-5
    x, gamma, beta = (a.astype(np.float64) for a in (x, gamma, beta))
    # 3,000 terms of size 1 with 2^-24 x DEPTH each at most, and h^2
    assert (_numbers(dX) * v).sum() == pytest.approx((loss(x + h * v, gamma, beta) - loss(x - h * v, gamma, beta)) / (2 * h), abs=2e-3)
    assert (_numbers(dg) * w).sum() == pytest.approx((loss(x, gamma + h * w, beta) - loss(x, gamma - h * w, beta)) / (2 * h), abs=2e-3)
    assert (_numbers(db) * w).sum() == pytest.approx((loss(x, gamma, beta + h * w) - loss(x, gamma, beta - h * w)) / (2 * h), abs=2e-3)


def test_no_rows(env):
    torch, cbm = env
    X = torch.empty((0, 12), device="cuda")
    cbm.cbm_layer_norm(X, None, None, 1e-5, X.clone())
    dg, db = torch.ones(12, device="cuda"), torch.ones(12, device="cuda")
    none = torch.empty(0, device="cuda")
    cbm.cbm_layer_norm_backward(X, X.clone(), None, none, none, X.clone(), dg, db, None)
    assert not bool(dg.any()) and not bool(db.any())


def test_more_than_2_to_the_31_values(env):
    """Offsets beyond 32 bits: the last rows of a matrix of 2.2e9 values."""
    torch, cbm = env
    n, k = 1 << 21, 1056
    X = torch.empty((n, k), dtype=torch.float16, device="cuda")
    X[:4], X[-300:] = torch.randn((4, k), device="cuda"), torch.randn((300, k), device="cuda")
    X[4:-300] = 1.0
    Y = torch.empty_like(X)
    mean, rstd = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    cbm.cbm_layer_norm(X, None, None, 1e-5, Y, mean, rstd)
    small = torch.empty((300, k), dtype=torch.float16, device="cuda")
    cbm.cbm_layer_norm(X[-300:].clone(), None, None, 1e-5, small)
    assert torch.equal(Y[-300:], small)
    dX, dY = torch.empty_like(X), Y
    cbm.cbm_layer_norm_backward(dY, X, None, mean, rstd, dX, None, None, None)
    cbm.cbm_layer_norm_backward(dY[-300:].clone(), X[-300:].clone(), None, mean[-300:].clone(), rstd[-300:].clone(), small, None, None, None)
    assert torch.equal(dX[-300:], small)


def test_graph_capture_replays(env):
    torch, cbm = env
    n, k = 3000, 100
    X, dY, G = torch.randn((n, k), device="cuda"), torch.randn((n, k), device="cuda"), torch.randn(k, device="cuda")
    outs = [torch.empty((n, k), device="cuda"), torch.empty(n, device="cuda"), torch.empty(n, device="cuda"), torch.empty((n, k), device="cuda"), torch.empty(k, device="cuda"),
            torch.empty(k, device="cuda")]
    workspace = torch.empty(cbm.cbm_layer_norm_workspace_bytes(n, k), dtype=torch.uint8, device="cuda")

    def step():
        cbm.cbm_layer_norm(X, G, None, 1e-5, outs[0], outs[1], outs[2])
        cbm.cbm_layer_norm_backward(dY, X, G, outs[1], outs[2], outs[3], outs[4], outs[5], workspace)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in range(3):
        X.copy_(torch.randn((n, k), device="cuda") + seed)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outs]
        for t in outs:
            t.fill_(math.nan)
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, outs))


def test_refusals(env):
    torch, cbm = env
    X, Y = torch.zeros((4, 8), device="cuda"), torch.zeros((4, 8), device="cuda")
    v = torch.zeros(8, device="cuda")
    s, s2 = torch.zeros(4, device="cuda"), torch.zeros(4, device="cuda")
    ws = torch.zeros(cbm.cbm_layer_norm_workspace_bytes(4, 8), dtype=torch.uint8, device="cuda")
    for bad in (lambda: cbm.cbm_layer_norm(X.cpu(), None, None, 1e-5, Y), lambda: cbm.cbm_layer_norm(X.double(), None, None, 1e-5, Y),
                lambda: cbm.cbm_layer_norm(X, None, None, 1e-5, Y[:, :4]), lambda: cbm.cbm_layer_norm(X, None, None, 1e-5, Y.bfloat16()),
                lambda: cbm.cbm_layer_norm(X, v[:4], None, 1e-5, Y), lambda: cbm.cbm_layer_norm(X, v.half(), None, 1e-5, Y),
                lambda: cbm.cbm_layer_norm(X.t(), None, None, 1e-5, Y.t()), lambda: cbm.cbm_layer_norm(X, None, None, 1e-5, Y, s[:2]),
                lambda: cbm.cbm_layer_norm_backward(X, X[:2], None, s, s2, Y, None, None, None),
                lambda: cbm.cbm_layer_norm_backward(X, X, None, s[:1], s2, Y, None, None, None)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: cbm.cbm_layer_norm(X, None, None, -1.0, Y), lambda: cbm.cbm_layer_norm(X, None, None, math.nan, Y), lambda: cbm.cbm_layer_norm(X, None, None, 1e-5, X),
                lambda: cbm.cbm_layer_norm(X, None, None, math.inf, Y), lambda: cbm.cbm_layer_norm(X, v, None, 1e-5, Y, s, s),
                lambda: cbm.cbm_layer_norm_backward(X, X, None, s, s2, X, None, None, None), lambda: cbm.cbm_layer_norm_backward(X, X, None, s, s2, None, None, None, None),
                lambda: cbm.cbm_layer_norm_backward(X, X, None, s, s2, Y, v, None, None), lambda: cbm.cbm_layer_norm_backward(X, X, None, s, s2, Y, v, None, ws[:-1]),
                lambda: cbm.cbm_layer_norm_backward(X, X, None, s, s2, Y, v, v, ws)):
        with pytest.raises(cbm.CbmError) as e:
            bad()
        assert e.value.status == 1
    # through the C ABI: types, sizes and leading dimensions that no tensor has
    from paper_2409_02208_amd import binding

    lib, p, q = binding._lib(), X.data_ptr(), Y.data_ptr()
    call = lambda n, k, t, ldx, ldy, x=p, y=q: lib.cbm_layer_norm(n, k, t, x, ldx, None, None, 1e-5, y, ldy, None, None, None)  # noqa: E731
    assert [call(4, 8, 3, 8, 8), call(-1, 8, 0, 8, 8), call(4, 0, 0, 8, 8), call(4, 8, 0, 7, 8), call(4, 8, 0, 8, 7), call(4, 8, 0, 8, 8, None), call(4, 8, 0, 8, 8, p + 1)] == [1] * 7
    assert call(4, (1 << 24) + 1, 0, 1 << 31, 1 << 31) == 5 and call(1 << 40, 8, 0, 1 << 40, 8) == 5
    assert cbm.cbm_layer_norm_workspace_bytes(4, 0) == 0 and isinstance(ctypes.c_size_t(ws.numel()).value, int)
    assert not bool(Y.any()) and not bool(X.any())
