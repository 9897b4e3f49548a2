"""The orthogonal update through the C ABI against the iteration in 64 bits: shapes from one value to several tiles, tall and wide, types, strides, in place, zeros, values that are
not finite, refusals."""
import math

import numpy as np
import pytest

from oracle import train_oracle as orc
from test_gpu_gated_linear import TYPES
from test_gpu_layer_norm import ROUNDING, _matrix, _numbers, _type, _untouched, env  # noqa: F401

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
A, B, C = 3.4445, -4.7750, 2.0315
SHAPES = [(1, 1), (1, 7), (7, 1), (2, 2), (3, 5), (8, 8), (16, 31), (33, 32), (47, 64), (64, 64), (64, 128), (65, 63), (100, 47), (128, 128), (129, 130), (257, 64), (64, 257), (200, 300),
          (500, 129), (1, 1000), (2000, 3), (40, 1500)]


def _error_bound(x, steps, abc=(A, B, C), eps=1e-7):
    """Of Z in the Frobenius norm.  A step's products have sums of K terms: off by (K + 16) 2^-24 |P| |Q|, whose norm is at most that of the factors' norms' product.  A step f carries an
    earlier error on by at most the largest slope of a s + b s^3 + c s^5 on the singular values up to the largest (an odd polynomial of a matrix changes by no more than its slope)."""
    z = np.asarray(x, dtype=np.float64)
    z = z.T if z.shape[0] > z.shape[1] else z
    z = z / (np.linalg.norm(z) + eps)
    m, n = z.shape
    error = 4 * U
    for _ in range(steps):
        s = np.linalg.svd(z, compute_uv=False)
        top = s[0] + error
        grid = np.linspace(0, top, 2001) ** 2
        slope = np.abs(abc[0] + 3 * abc[1] * grid + 5 * abc[2] * grid * grid).max()
        gram, size = z @ z.T, np.linalg.norm(z)
        of_gram = (n + 16) * U * size * size
        p = abc[1] * gram + abc[2] * gram @ gram
        of_p = (abs(abc[1]) + 2 * abs(abc[2]) * top * top) * of_gram + (m + 20) * U * (abs(abc[2]) * np.linalg.norm(gram) ** 2 + abs(abc[1]) * np.linalg.norm(gram))
        error = slope * error + of_p * top + (m + 20) * U * (np.linalg.norm(p) * size + abs(abc[0]) * size)
        z = abc[0] * z + p @ z
    return error


def _check(torch, cbm, x, name, pad=0, offset=0, in_place=False, **more):
    X, whole_x = _matrix(torch, x, name, pad, offset)
    exact = _numbers(X)
    Y, whole = (X, whole_x) if in_place else _matrix(torch, np.zeros(x.shape), name, pad, offset)
    ws = torch.full((cbm.cbm_orthogonalise_workspace_bytes(*x.shape, _type(torch, name)),), 255, dtype=torch.uint8, device="cuda")
    cbm.cbm_orthogonalise(X, Y, workspace=ws, **more)
    _untouched(torch, Y, whole, offset)
    want = orc.orthogonalise(exact, **more)
    scale = abs(more.get("scale", 1.0))
    of_z = scale * _error_bound(exact, more.get("steps", 5), more.get("coefficients", (A, B, C)), more.get("eps", 1e-7)) + U * np.linalg.norm(want)
    bound = of_z + ROUNDING[name] * (np.linalg.norm(want) + of_z) + (2.0 ** -25 * math.sqrt(x.size) if name == "f16" else 0.0)
    off = np.linalg.norm(_numbers(Y) - want)
    assert off <= bound, (off, bound)
    return Y, want


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("m,n", SHAPES)
def test_against_64_bits(env, name, m, n):  # noqa: F811
    torch, cbm = env
    rng = np.random.default_rng(m + 1000 * n)
    for i, (pad, offset, in_place) in enumerate(((0, 0, False), (3, 1, True), (8, 8, False))):
        x = 10.0 ** (-i) * rng.standard_normal((m, n))
        if min(m, n) > 8:
            x += rng.standard_normal((m, 2)) @ rng.standard_normal((2, n))
        _check(torch, cbm, x, name, pad, offset, in_place)


@pytest.mark.parametrize("m,n", [(64, 64), (48, 200), (300, 70), (130, 129)])
def test_singular_values(env, m, n):  # noqa: F811
    """From 1 / 500 of the norm up they come out between 0.65 and 1.25 (the iteration's own range, 0.68 to 1.21, and a margin for its roundings), with the directions kept."""
    torch, cbm = env
    rng = np.random.default_rng(5)
    u, v = np.linalg.qr(rng.standard_normal((m, min(m, n))))[0], np.linalg.qr(rng.standard_normal((n, min(m, n))))[0]
    s = np.geomspace(1.0, 1 / 60, min(m, n))
    assert s[-1] / np.linalg.norm(s) >= 1 / 500
    Y, _ = _check(torch, cbm, (u * s) @ v.T, "f32")
    y = _numbers(Y)
    got = np.linalg.svd(y, compute_uv=False)
    assert got.min() > 0.65 and got.max() < 1.25
    core = u.T @ y @ v
    assert np.abs(core - np.diag(np.diag(core))).max() < 1e-3


@pytest.mark.parametrize("m,n", [(20, 33), (150, 140), (64, 64)])
def test_steps_coefficients_and_scale(env, m, n):  # noqa: F811
    torch, cbm = env
    x = np.random.default_rng(6).standard_normal((m, n))
    _check(torch, cbm, x, "f32", steps=0)
    _check(torch, cbm, x, "f32", steps=1, scale=-0.25)
    _check(torch, cbm, x, "f32", steps=3, coefficients=(1.875, -1.25, 0.375), scale=2.0)
    _check(torch, cbm, x, "bf16", steps=2, eps=0.5)


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("m,n", [(5, 9), (64, 64), (130, 70)])
def test_zeros_and_values_that_are_not_finite(env, name, m, n):  # noqa: F811
    torch, cbm = env
    ws = torch.empty(cbm.cbm_orthogonalise_workspace_bytes(m, n, _type(torch, name)), dtype=torch.uint8, device="cuda")
    X, Y = torch.zeros((m, n), dtype=_type(torch, name), device="cuda"), torch.ones((m, n), dtype=_type(torch, name), device="cuda")
    cbm.cbm_orthogonalise(X, Y, workspace=ws)
    assert not bool(Y.any())
    cbm.cbm_orthogonalise(X, Y, eps=0.0, workspace=ws)
    assert bool(Y.isnan().all())
    for odd in (math.nan, math.inf):
        X.fill_(1.0)
        X[m // 2, n - 1] = odd
        cbm.cbm_orthogonalise(X, Y, workspace=ws)
        assert bool(Y.isnan().all())


@pytest.mark.parametrize("size", [1e-30, 1e-12, 1e12, 1e30])
@pytest.mark.parametrize("m,n", [(30, 40), (140, 150)])
def test_sizes_whose_squares_leave_fp32(env, size, m, n):  # noqa: F811
    torch, cbm = env
    _check(torch, cbm, size * np.random.default_rng(7).standard_normal((m, n)), "f32", eps=0.0)


def test_captured(env):  # noqa: F811
    torch, cbm = env
    for m, n in ((64, 64), (100, 300)):
        X, Y = torch.randn((m, n), device="cuda"), torch.empty((m, n), device="cuda")
        ws = torch.empty(cbm.cbm_orthogonalise_workspace_bytes(m, n, torch.float32), dtype=torch.uint8, device="cuda")
        step = lambda: cbm.cbm_orthogonalise(X, Y, workspace=ws)  # noqa: E731
        step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        for seed in range(3):
            X.copy_(torch.randn((m, n), device="cuda") * (seed + 1))
            graph.replay()
            torch.cuda.synchronize()
            got = Y.clone()
            Y.fill_(-5)
            step()
            torch.cuda.synchronize()
            assert torch.equal(got, Y)


def test_refusals(env):  # noqa: F811
    torch, cbm = env
    X, Y = torch.zeros((30, 20), device="cuda"), torch.ones((30, 20), device="cuda")
    ws = torch.zeros(cbm.cbm_orthogonalise_workspace_bytes(30, 20, torch.float32), dtype=torch.uint8, device="cuda")
    for bad in (lambda: cbm.cbm_orthogonalise(X.cpu(), Y, workspace=ws), lambda: cbm.cbm_orthogonalise(X, Y[:, :19], workspace=ws), lambda: cbm.cbm_orthogonalise(X, Y.half(), workspace=ws),
                lambda: cbm.cbm_orthogonalise(X.t(), Y.t(), workspace=ws), lambda: cbm.cbm_orthogonalise(X, Y, coefficients=(1.0, 2.0), workspace=ws),
                lambda: cbm.cbm_orthogonalise(X, Y, steps=1 << 40, workspace=ws)):
        with pytest.raises((ValueError, OverflowError)):
            bad()
    for bad in (lambda: cbm.cbm_orthogonalise(X, Y), lambda: cbm.cbm_orthogonalise(X, Y, workspace=ws[:-1]), lambda: cbm.cbm_orthogonalise(X, Y, steps=-1, workspace=ws),
                lambda: cbm.cbm_orthogonalise(X, Y, steps=101, workspace=ws), lambda: cbm.cbm_orthogonalise(X, Y, eps=-1.0, workspace=ws), lambda: cbm.cbm_orthogonalise(X, Y, eps=math.nan, workspace=ws),
                lambda: cbm.cbm_orthogonalise(X, Y, scale=math.inf, workspace=ws), lambda: cbm.cbm_orthogonalise(X, Y, coefficients=(1.0, math.nan, 0.0), workspace=ws),
                lambda: cbm.cbm_orthogonalise(X[:29], X[1:], workspace=ws), lambda: cbm.cbm_orthogonalise(X[:0], Y[:0], workspace=ws)):
        with pytest.raises(cbm.CbmError) as e:
            bad()
        assert e.value.status == 1
    from paper_2409_02208_amd import binding

    lib = binding._lib()
    call = lambda m=30, n=20, t=0, ld=20: lib.cbm_orthogonalise(m, n, t, X.data_ptr(), ld, 5, None, 0.0, 1.0, Y.data_ptr(), ld, ws.data_ptr(), ws.numel(), None)  # noqa: E731
    assert [call(m=0), call(n=-1), call(t=3), call(ld=19)] == [1] * 4
    assert [call(m=65537), call(n=65537, ld=70000)] == [5, 5]
    torch.cuda.synchronize()
    assert bool((Y == 1).all())


def test_coefficients_that_diverge_are_refused(env):  # noqa: F811
    torch, cbm = env
    for m, n in ((8, 8), (200, 150)):
        X, Y = torch.ones((m, n), device="cuda"), torch.full((m, n), 3.0, device="cuda")
        ws = torch.empty(cbm.cbm_orthogonalise_workspace_bytes(m, n, torch.float32), dtype=torch.uint8, device="cuda")
        for abc, steps in (((100.0, 0.0, 0.0), 6), ((1e20, 0.0, 0.0), 2), ((0.0, 0.0, 1e31), 1), ((3.0, 3.0, 3.0), 100), ((2.0, -3.0, 50.0), 2), ((0.0, 1.0, 0.0), 1)):
            with pytest.raises(cbm.CbmError) as e:
                cbm.cbm_orthogonalise(X, Y, steps=steps, coefficients=abc, workspace=ws)
            assert e.value.status == 5
        assert bool((Y == 3).all())
        cbm.cbm_orthogonalise(X, Y, steps=100, workspace=ws)  # (the usual ones stay)
        assert bool(Y.isfinite().all())


@pytest.mark.parametrize("m,n", [(30, 20), (150, 200)])
def test_large_and_small_coefficients(env, m, n):  # noqa: F811
    torch, cbm = env
    x = np.random.default_rng(8).standard_normal((m, n))
    for abc, steps in (((10.0, 0.0, 0.0), 6), ((0.01, 0.0, 0.0), 6), ((1.5, -0.5, 0.0), 12), ((1e25, 0.0, 0.0), 1)):
        _check(torch, cbm, x, "f32", steps=steps, coefficients=abc)


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("m,n", [(1, 129), (31, 129), (3, 255), (32, 256), (256, 17), (32, 257), (20, 511), (512, 32), (1, 512), (33, 130), (64, 256), (256, 64), (250, 63), (34, 255), (513, 32), (257, 33), (65, 129)])
def test_thin_matrices(env, name, m, n):  # noqa: F811
    """Short sides of up to 32 and 64 with long ones up to 512 and 256, and the next beyond."""
    torch, cbm = env
    x = np.random.default_rng(m + 1000 * n).standard_normal((m, n))
    for pad, offset, in_place in ((0, 0, False), (5, 3, True)):
        _check(torch, cbm, x, name, pad, offset, in_place)
