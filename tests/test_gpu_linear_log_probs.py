"""Log probabilities of a layer's classes without their scores, and their gradients, through the C ABI against the definition in 64 bits: sizes around every tile, chunk and piece,
rows without a label, scores that rule classes out, refusals."""
import math

import numpy as np
import pytest

from oracle import train_oracle as orc
from test_gpu_gated_linear import SUM, TYPES, _gpu, _near, _rounded, _within
from test_gpu_layer_norm import _matrix, _numbers, _type, _untouched, env  # noqa: F401

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
SIZES = [(1, 1, 1), (2, 3, 2), (5, 7, 3), (33, 8, 4), (128, 9, 7), (129, 31, 8), (3, 33, 31), (64, 64, 33), (31, 65, 47), (127, 63, 64), (257, 100, 65), (1, 128, 127), (70, 130, 128),
         (5, 40, 129), (300, 17, 300), (1, 500, 1000), (40, 24, 5003), (2, 1030, 257), (1000, 12, 20)]


def _inputs(torch, n, d, c, name, pad, offset, bits=64, spread=3.0):
    rng = np.random.default_rng(n + 3 * d + 7 * c)
    X, _ = _matrix(torch, rng.standard_normal((n, d)), name, pad, offset)
    W, _ = _matrix(torch, spread * rng.standard_normal((d, c)) / math.sqrt(d), name, pad, offset)
    labels = rng.integers(-1, c + 1, n)
    return X, W, torch.from_numpy(labels).to(torch.int64 if bits == 64 else torch.int32).cuda()


def _forward(torch, cbm, X, W, L):
    n, c = X.shape[0], W.shape[1]
    logp, stats = torch.full((n,), math.nan, device="cuda"), torch.full((n, 2), math.nan, device="cuda")
    ws = torch.full((cbm.cbm_linear_log_probs_workspace_bytes(n, X.shape[1], c, X.dtype),), 255, dtype=torch.uint8, device="cuda")
    cbm.cbm_linear_log_probs(X, W, L, logp, stats, workspace=ws)
    return logp, stats


def _score_bound(x, w):
    return SUM(x.shape[1]) * (np.abs(x) @ np.abs(w))


def _check_forward(X, W, L, logp, stats):
    x, w, labels = _numbers(X), _numbers(W), L.cpu().numpy()
    z = x @ w
    want = orc.log_probs(z, labels)
    of_z = _score_bound(x, w)
    largest = np.max(of_z, axis=1)
    d = np.abs(z - z.max(axis=1)[:, None])
    p = np.exp(-d) / np.exp(-d).sum(axis=1)[:, None]
    # a term of the sum: its score, its argument's three roundings, exp2's unit in the last place, once more for each joining; c additions at most, in shares
    of_l = (p * (of_z + U * (6 * d + 40))).sum(axis=1) + largest + (z.shape[1] / 32 + 40) * U + 3 * U * np.abs(want[2][:, 1])
    _near(stats[:, 0], want[2][:, 0], largest + U * np.abs(want[2][:, 0]))
    _near(stats[:, 1], want[2][:, 1], of_l)
    given = (labels >= 0) & (labels < z.shape[1])
    of_chosen = np.where(given, of_z[np.arange(len(labels)), np.where(given, labels, 0)], 0.0)
    _near(logp, want[0], np.where(given, of_chosen + largest + of_l + 4 * U * (np.abs(want[0]) + np.abs(want[2][:, 1])), 0.0))


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("n,d,c", SIZES)
def test_forward(env, name, n, d, c):  # noqa: F811
    torch, cbm = env
    for pad, offset, bits in ((0, 0, 64), (3, 1, 32), (8, 8, 64)):
        X, W, L = _inputs(torch, n, d, c, name, pad, offset, bits)
        _check_forward(X, W, L, *_forward(torch, cbm, X, W, L))


def _backward(torch, cbm, X, W, L, pad, offset, size=1.0, outputs=(True, True), equal=False):
    n, c = X.shape[0], W.shape[1]
    name = {torch.float32: "f32", torch.bfloat16: "bf16", torch.float16: "f16"}[X.dtype]
    stats = torch.from_numpy(orc.log_probs(_numbers(X) @ _numbers(W), L.cpu().numpy())[2].astype(np.float32)).cuda() if n else torch.zeros((0, 2), device="cuda")
    rng = np.random.default_rng(n)
    dlogp = torch.from_numpy((size * (np.ones(n) if equal else rng.uniform(-1.5, 0.5, n))).astype(np.float32)).cuda()
    (dX, whole_x), (dW, whole_w) = (_matrix(torch, np.zeros(s), name, pad, offset) for s in (tuple(X.shape), tuple(W.shape)))
    ws = torch.full((cbm.cbm_linear_log_probs_backward_workspace_bytes(n, X.shape[1], c, X.dtype),), 255, dtype=torch.uint8, device="cuda")
    cbm.cbm_linear_log_probs_backward(X, W, L, stats, dlogp, dX if outputs[0] else None, dW if outputs[1] else None, workspace=ws)
    _untouched(torch, dX, whole_x, offset)
    _untouched(torch, dW, whole_w, offset)
    return stats, dlogp, dX, dW


def _check_backward(X, W, L, stats, dlogp, dX, dW, name, outputs=(True, True)):
    x, w, labels, st, a = _numbers(X), _numbers(W), L.cpu().numpy(), _numbers(stats), _numbers(dlogp)
    dx, dw, dz = orc.linear_log_probs_backward(x, w, labels, st, a)
    z = x @ w
    with np.errstate(invalid="ignore"):
        away = np.where(st[:, :1] > -np.inf, np.abs(z - st[:, :1]) + np.abs(st[:, 1:]), 0.0)
        p = np.where(st[:, :1] > -np.inf, np.exp(z - st[:, :1] - st[:, 1:]), 0.0)
    given = ((labels >= 0) & (labels < w.shape[1]))[:, None]
    # p: its score, three roundings of the exponent, exp2's unit in the last place; two roundings of the difference; the type's (fp16: of dz at 2^15 over the largest |dlogp|)
    least = {"f32": 2.0 ** -126, "bf16": 2.0 ** -126, "f16": 2.0 ** -25 * 2.0 ** -15 * (np.abs(a).max() if len(a) else 0.0)}[name]
    of_dz = np.abs(a)[:, None] * (1.01 * p * (_score_bound(x, w) + 6 * U * away + 4 * U) + 2 * U) + 2 * U * np.abs(dz)
    half = {"f32": U, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}[name]
    of_dz = given * (of_dz + half * (np.abs(dz) + of_dz) + least)
    for on, got, want, bound in ((outputs[0], dX, dx, SUM(w.shape[1]) * ((np.abs(dz) + of_dz) @ np.abs(w.T)) + of_dz @ np.abs(w.T)),
                                 (outputs[1], dW, dw, SUM(x.shape[0]) * (np.abs(x.T) @ (np.abs(dz) + of_dz)) + np.abs(x.T) @ of_dz)):
        if on:
            _near(got, want, _rounded(want, bound, name))
        else:
            assert not bool(got.any())


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("n,d,c", SIZES + [(3000, 9, 5), (2600, 70, 130)])
def test_backward(env, name, n, d, c):  # noqa: F811
    torch, cbm = env
    for i, (pad, offset, bits) in enumerate(((0, 0, 64), (5, 1, 32), (8, 8, 64))):
        X, W, L = _inputs(torch, n, d, c, name, pad, offset, bits)
        on = ((True, True), (True, False), (False, True))[i] if n % 2 else (True, True)
        _check_backward(X, W, L, *_backward(torch, cbm, X, W, L, pad, offset, outputs=on, equal=i == 2), name, on)


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("n,d,c", [(40001, 31, 8), (20003, 65, 47), (9001, 17, 300), (5001, 63, 130), (65, 40, 16400)])
def test_many_rows_or_classes(env, name, n, d, c):  # noqa: F811
    """Tiles through LDS, where most sizes above are small."""
    torch, cbm = env
    for i, (pad, offset, bits) in enumerate(((0, 0, 64), (5, 1, 32), (8, 8, 64))):
        X, W, L = _inputs(torch, n, d, c, name, pad, offset, bits)
        _check_forward(X, W, L, *_forward(torch, cbm, X, W, L))
        on = ((True, True), (True, False), (False, True))[i]
        _check_backward(X, W, L, *_backward(torch, cbm, X, W, L, pad, offset, outputs=on, equal=i == 2), name, on)


@pytest.mark.parametrize("name", TYPES)
def test_pieces_of_the_classes(env, name):  # noqa: F811
    """More rows than 512 MiB hold scores for: several pieces, the last one short."""
    torch, cbm = env
    n, d, c = 262147 if name == "f32" else 524309, 4, 1100
    X, W, L = _inputs(torch, n, d, c, name, 0, 0)
    stats = torch.empty((n, 2), device="cuda")
    z = X.double() @ W.double()
    stats[:, 0] = z.amax(dim=1)
    stats[:, 1] = torch.logsumexp(z, dim=1) - z.amax(dim=1)
    dlogp = torch.full((n,), -1.0 / n, device="cuda")
    given = (L >= 0) & (L < c)
    dX, dW = torch.empty_like(X), torch.empty_like(W)
    ws = torch.full((cbm.cbm_linear_log_probs_backward_workspace_bytes(n, d, c, X.dtype),), 255, dtype=torch.uint8, device="cuda")
    cbm.cbm_linear_log_probs_backward(X, W, L, stats, dlogp, dX, dW, workspace=ws)
    dz = torch.exp(z - stats.double().sum(1, keepdim=True)).neg_()
    del z
    dz[torch.arange(n, device="cuda"), L.clamp(0, c - 1)] += 1.0
    dz *= (dlogp * given).double()[:, None]
    # the largest rounding by far is the type's of each dz and of the results; in the 2-norm terms of either sign add up to less than twice each
    tol = {"f32": 1e-5, "bf16": 2.0 ** -7, "f16": 2.0 ** -10}[name]
    for got, want in ((dX, dz @ W.double().t().contiguous()), (dW, X.double().t().contiguous() @ dz)):
        least = 2.0 ** -24 * math.sqrt(want.numel()) if name == "f16" else 0.0
        assert float((got.double() - want).norm()) <= tol * float(want.norm()) + least


def test_small_gradients_in_fp16_are_not_lost(env):  # noqa: F811
    """dlogp of 1e-7 of rows of equal weight: dz itself is below fp16's smallest value, the gradients are not where they add up."""
    torch, cbm = env
    X, W, L = _inputs(torch, 600, 20, 300, "f16", 0, 0)
    _check_backward(X, W, L, *_backward(torch, cbm, X, W, L, 0, 0, size=1e-5), "f16")


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("n", [1, 130, 9001])
def test_a_mean_is_not_rounded_alike_in_every_row(env, name, n):  # noqa: F811
    """The same dlogp in every row, which the type would round by almost half a step; scores of zero, so that p is 2^-10 everywhere and a label's 1 - p is at most that far from a value of the type."""
    torch, cbm = env
    d, c = 40, 1024
    rng = np.random.default_rng(n)
    X, W = _matrix(torch, rng.standard_normal((n, d)), name, 0)[0], _matrix(torch, np.zeros((d, c)), name, 0)[0]
    L = torch.from_numpy(rng.integers(0, c, n)).cuda()
    stats = torch.tensor([0.0, math.log(c)], device="cuda").repeat(n, 1)
    half = {"f32": U, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}[name]
    a = -(1 + 0.97 * half) * 2.0 ** -7
    dX, dW = torch.ones_like(X), torch.empty_like(W)
    ws = torch.empty(cbm.cbm_linear_log_probs_backward_workspace_bytes(n, d, c, X.dtype), dtype=torch.uint8, device="cuda")
    cbm.cbm_linear_log_probs_backward(X, W, L, stats, torch.full((n,), a, device="cuda"), dX, dW, workspace=ws)
    x = _numbers(X)
    dz = np.full((n, c), -float(np.float32(a)) / c)
    dz[np.arange(n), L.cpu().numpy()] += float(np.float32(a))
    # 1 - p: 2^-10 where the type lacks it; p: the logarithm's rounding and the exponential's; the factor's two; then the sum and the result's own rounding
    size = np.abs(dz) * (12 * U + (2.0 ** -10 if name == "bf16" else 0.0))
    least = 2.0 ** -25 * 2.0 ** -15 * abs(a) if name == "f16" else 0.0
    _near(dW, x.T @ dz, _rounded(x.T @ dz, SUM(n) * (np.abs(x.T) @ np.abs(dz)) + np.abs(x.T) @ (size + least), name))
    assert not bool(dX.any())


@pytest.mark.parametrize("name", TYPES)
def test_slopes_that_are_not_finite_or_nothing(env, name):  # noqa: F811
    """A row's infinite or missing slope is its own (and that of the weights' sums), and none at all leaves zeros."""
    torch, cbm = env
    n, d, c = 200, 24, 300
    X, W, L = _inputs(torch, n, d, c, name, 0, 0)
    L.clamp_(0, c - 1)
    ws = torch.empty(cbm.cbm_linear_log_probs_backward_workspace_bytes(n, d, c, X.dtype), dtype=torch.uint8, device="cuda")
    stats = _forward(torch, cbm, X, W, L)[1]
    a, rows = -torch.rand(n, device="cuda") - 0.1, torch.ones(n, dtype=torch.bool, device="cuda")
    some = []
    for bad in (0.0, math.nan, math.inf):
        a[[3, 150]] = bad
        dX, dW = torch.empty_like(X), torch.empty_like(W)
        cbm.cbm_linear_log_probs_backward(X, W, L, stats, a, dX, dW, workspace=ws)
        some.append(dX)
    rows[[3, 150]] = False
    assert torch.equal(some[0][rows], some[1][rows]) and torch.equal(some[0][rows], some[2][rows])
    assert not bool(some[0][~rows].any()) and not bool(some[1][~rows].isfinite().any()) and not bool(some[2][~rows].isfinite().any())
    for size in (0.0, 1e-42):
        cbm.cbm_linear_log_probs_backward(X, W, L, stats, torch.full_like(a, size), dX, dW, workspace=ws)
        assert float(dX.abs().max()) <= 1e-38 and float(dW.abs().max()) <= 1e-38


def test_backward_against_differences(env):  # noqa: F811
    torch, cbm = env
    X, W, L = _inputs(torch, 5, 4, 6, "f32", 0, 0)
    x, w, labels = _numbers(X), _numbers(W), L.cpu().numpy()
    _, dlogp, dX, dW = _backward(torch, cbm, X, W, L, 0, 0)
    loss = lambda x, w: (orc.log_probs(x @ w, labels)[0] * _numbers(dlogp)).sum()  # noqa: E731
    step = 1e-5
    for i, got in enumerate((dX, dW)):
        want = np.zeros(got.shape)
        for at in np.ndindex(*got.shape):
            both = []
            for s in (step, -step):
                p = [x.copy(), w.copy()]
                p[i][at] += s
                both.append(loss(*p))
            want[at] = (both[0] - both[1]) / (2 * step)
        assert np.abs(_numbers(got) - want).max() <= 1e-5 * max(1.0, np.abs(want).max())  # (differences: step^2 and 2^-53 / step, sums of fp32)


@pytest.mark.parametrize("name", ["bf16", "f16"])
def test_classes_ruled_out(env, name):  # noqa: F811
    """A last feature of one and a weight of -infinity rule a class out; with all of them ruled out a row has no distribution.  In 16 bits, where a sum with an infinite term is infinite."""
    torch, cbm = env
    rng = np.random.default_rng(4)
    n, d, c = 40, 9, 150
    x, w = rng.standard_normal((n, d)), rng.standard_normal((d, c))
    x[:, -1] = 1.0
    w[-1, rng.random(c) < 0.3] = -math.inf
    labels = rng.integers(0, c, n)
    X, W, L = _matrix(torch, x, name, 0)[0], _matrix(torch, w, name, 0)[0], torch.from_numpy(labels).cuda()
    for W_, every in ((W, False), (torch.full_like(W, -math.inf), True)):
        if every:
            W_[:-1] = 0.0
        logp, stats = _forward(torch, cbm, X, W_, L)
        z = _numbers(X) @ _numbers(W_) if not every else np.full((n, c), -np.inf)
        want = orc.log_probs(z, labels)
        same = lambda a, b: np.all((a == b) | (np.abs(a - b) <= 1e-4))  # noqa: E731  (which classes are left, not the roundings)
        with np.errstate(invalid="ignore"):
            assert same(_numbers(logp), want[0]) and same(_numbers(stats), want[2])
    # nothing comes back from a row without a distribution
    dX, dW = torch.ones_like(X), torch.ones_like(W)
    empty = torch.full((n, 2), -math.inf, device="cuda")
    ws = torch.empty(cbm.cbm_linear_log_probs_backward_workspace_bytes(n, d, c, X.dtype), dtype=torch.uint8, device="cuda")
    cbm.cbm_linear_log_probs_backward(X, torch.zeros_like(W), L, empty, torch.ones(n, device="cuda"), dX, dW, workspace=ws)
    assert not bool(dX.any()) and not bool(dW.any())


@pytest.mark.parametrize("name", TYPES)
def test_values_that_are_not_finite(env, name):  # noqa: F811
    torch, cbm = env
    X, W, L = _inputs(torch, 200, 20, 300, name, 0, 0)
    L.clamp_(0, 299)
    L[7] = -1
    logp, stats = _forward(torch, cbm, X, W, L)
    X[5, 3], X[7, 0], X[150, 19] = math.nan, math.nan, math.inf
    again, odd = _forward(torch, cbm, X, W, L)
    rows = torch.ones(200, dtype=torch.bool, device="cuda")
    rows[[5, 7, 150]] = False
    assert torch.equal(logp[rows], again[rows]) and torch.equal(stats[rows], odd[rows])
    assert bool(odd[~rows].isnan().all()) and bool(again[[5, 150]].isnan().all()) and float(again[7]) == 0.0


@pytest.mark.parametrize("name", TYPES)
def test_no_rows(env, name):  # noqa: F811
    torch, cbm = env
    X, W, L = _inputs(torch, 0, 12, 9, name, 0, 0)
    _forward(torch, cbm, X, W, L)
    dW = torch.full_like(W, 3)
    cbm.cbm_linear_log_probs_backward(X, W, L, torch.zeros((0, 2), device="cuda"), torch.zeros(0, device="cuda"), None, dW,
                                      workspace=torch.empty(cbm.cbm_linear_log_probs_backward_workspace_bytes(0, 12, 9, _type(torch, name)), dtype=torch.uint8, device="cuda"))
    assert not bool(dW.any())


def test_agrees_with_log_probs_of_the_scores(env):  # noqa: F811
    """Small whole numbers: scores are exact either way, so both calls see the same."""
    torch, cbm = env
    g = torch.Generator(device="cuda").manual_seed(2)
    X, W = (torch.randint(-3, 4, s, device="cuda", generator=g).float() for s in ((150, 24), (24, 700)))
    L = torch.randint(0, 700, (150,), device="cuda", generator=g)
    logp, stats = _forward(torch, cbm, X, W, L)
    other, st = torch.empty_like(logp), torch.empty_like(stats)
    cbm.cbm_log_probs((X.double() @ W.double()).float(), L, other, None, st)
    assert torch.equal(stats[:, 0], st[:, 0])
    # both sum 700 terms of one in another order, below 200 roundings each
    assert float((stats - st).abs().max()) <= 400 * U * 2 and float((logp - other).abs().max()) <= 400 * U * 2 + 4 * U * float(other.abs().max())


def test_captured_and_on_streams(env):  # noqa: F811
    torch, cbm = env
    n, d, c = 300, 40, 700
    for dtype in (torch.float16, torch.float32):
        X, W, L = (t.to(dtype) if t.is_floating_point() else t for t in _inputs(torch, n, d, c, "f32", 0, 0))
        one = torch.ones(n, device="cuda")
        new = lambda: [torch.empty(n, device="cuda"), torch.empty((n, 2), device="cuda"), torch.empty_like(X), torch.empty_like(W)]  # noqa: E731
        need = max(cbm.cbm_linear_log_probs_workspace_bytes(n, d, c, dtype), cbm.cbm_linear_log_probs_backward_workspace_bytes(n, d, c, dtype))
        ws = [torch.empty(need, dtype=torch.uint8, device="cuda") for _ in range(3)]
        outs = new()

        def step(o, w, stream=None):
            cbm.cbm_linear_log_probs(X, W, L, o[0], o[1], workspace=w, stream=stream)
            cbm.cbm_linear_log_probs_backward(X, W, L, o[1], one, o[2], o[3], workspace=w, stream=stream)

        step(outs, ws[0])
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step(outs, ws[0])
        streams = [torch.cuda.Stream() for _ in range(2)]
        for seed in range(3):
            X.copy_(torch.randn((n, d), device="cuda") * (seed + 1))
            graph.replay()
            torch.cuda.synchronize()
            got, apart = [t.clone() for t in outs], [new() for _ in range(2)]
            torch.cuda.synchronize()
            for s, o, w in zip(streams, apart, ws[1:]):
                step(o, w, s)
            torch.cuda.synchronize()
            for o in apart:
                assert all(torch.equal(a, b) for a, b in zip(got, o))


def test_refusals(env):  # noqa: F811
    torch, cbm = env
    X, W, L = torch.zeros((4, 6), device="cuda"), torch.zeros((6, 50), device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda")
    logp, st = torch.ones(4, device="cuda"), torch.ones((4, 2), device="cuda")
    ws = torch.zeros(cbm.cbm_linear_log_probs_workspace_bytes(4, 6, 50, torch.float32), dtype=torch.uint8, device="cuda")
    wb = torch.zeros(cbm.cbm_linear_log_probs_backward_workspace_bytes(4, 6, 50, torch.float32), dtype=torch.uint8, device="cuda")
    dX, dW = torch.ones_like(X), torch.ones_like(W)
    for bad in (lambda: cbm.cbm_linear_log_probs(X.cpu(), W, L, logp, st, ws), lambda: cbm.cbm_linear_log_probs(X, W[:5], L, logp, st, ws), lambda: cbm.cbm_linear_log_probs(X, W.half(), L, logp, st, ws),
                lambda: cbm.cbm_linear_log_probs(X, W, L[:3], logp, st, ws), lambda: cbm.cbm_linear_log_probs(X, W, L.float(), logp, st, ws),
                lambda: cbm.cbm_linear_log_probs(X, W, L, logp[:3], st, ws), lambda: cbm.cbm_linear_log_probs(X, W, L, logp, logp, ws),
                lambda: cbm.cbm_linear_log_probs_backward(X, W, L, st, logp, dX[:3], dW, wb), lambda: cbm.cbm_linear_log_probs_backward(X, W, L, st, logp, dX, dW.half(), wb),
                lambda: cbm.cbm_linear_log_probs_workspace_bytes(4, 6, 50, torch.float64)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: cbm.cbm_linear_log_probs(X, W, None, logp, st, ws), lambda: cbm.cbm_linear_log_probs(X, W, L, logp, st, None), lambda: cbm.cbm_linear_log_probs(X, W, L, logp, st, ws[:-1]),
                lambda: cbm.cbm_linear_log_probs_backward(X, W, L, st, logp, None, None, wb), lambda: cbm.cbm_linear_log_probs_backward(X, W, L, st, logp, X, dW, wb),
                lambda: cbm.cbm_linear_log_probs_backward(X, W, L, st, logp, dX, dW, wb[16:]), lambda: cbm.cbm_linear_log_probs_backward(X, W, L, None, logp, dX, dW, wb),
                lambda: cbm.cbm_linear_log_probs_backward(X, W, L, st, None, dX, dW, wb), lambda: cbm.cbm_linear_log_probs_backward(X, W, None, st, logp, dX, dW, wb)):
        with pytest.raises(cbm.CbmError) as e:
            bad()
        assert e.value.status == 1
    from paper_2409_02208_amd import binding

    lib = binding._lib()
    call = lambda n=4, d=6, c=50, t=0, ldx=6, ldw=50, bits=64, p=X.data_ptr(): lib.cbm_linear_log_probs(n, d, c, t, p, ldx, W.data_ptr(), ldw, L.data_ptr(), bits, logp.data_ptr(), None, ws.data_ptr(), ws.numel(), None)  # noqa: E731
    assert [call(n=-1), call(d=0), call(c=0), call(t=7), call(ldx=5), call(ldw=49), call(bits=16), call(p=None), call(p=X.data_ptr() + 1)] == [1] * 9
    assert [call(d=(1 << 24) + 1, ldx=1 << 25), call(c=(1 << 24) + 1, ldw=1 << 25)] == [5, 5]
    torch.cuda.synchronize()
    assert bool((logp == 1).all()) and bool((st == 1).all()) and bool((dX == 1).all()) and bool((dW == 1).all())


@pytest.mark.parametrize("name", ["bf16", "f16"])
@pytest.mark.parametrize("n,d,c", [(1, 8, 8), (130, 72, 72), (300, 64, 264), (257, 200, 1000), (4100, 72, 4104), (2304, 320, 4096)])
def test_whole_units(env, name, n, d, c):  # noqa: F811
    """Rows that are whole numbers of 16 bytes: tiles of 128 and 256 with all and with few of their rows and columns, d that ends inside a chunk of 64."""
    torch, cbm = env
    for pad in (0, 8):
        X, W, L = _inputs(torch, n, d, c, name, pad, 0)
        _check_forward(X, W, L, *_forward(torch, cbm, X, W, L))
        _check_backward(X, W, L, *_backward(torch, cbm, X, W, L, pad, 0), name)


@pytest.mark.parametrize("name", ["bf16", "f16"])
@pytest.mark.parametrize("pad,offset", [(0, 0), (1, 1), (8, 0)])
@pytest.mark.parametrize("n,d,c", [(12001, 515, 8199), (4097, 512, 24576), (1025, 1000, 50001), (300007, 258, 1061)])
def test_large_products(env, name, n, d, c, pad, offset):  # noqa: F811
    """Matrices of odd widths, strides and addresses are copied into rows of whole units, and the weights of many rows turned; the last size in several pieces, with a short last unit.  Against 64 bits on the
    GPU."""
    torch, cbm = env
    torch.manual_seed(n)
    X, W = _gpu(torch, n, d, name, pad, offset), _gpu(torch, d, c, name, pad, offset, 3 * d ** -0.5)
    L = torch.randint(-1, c + 1, (n,), device="cuda")
    need = max(cbm.cbm_linear_log_probs_workspace_bytes(n, d, c, X.dtype), cbm.cbm_linear_log_probs_backward_workspace_bytes(n, d, c, X.dtype))
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    logp, stats = torch.empty(n, device="cuda"), torch.empty((n, 2), device="cuda")
    cbm.cbm_linear_log_probs(X, W, L, logp, stats, workspace=ws)
    x, w = X.double(), W.double()
    z = x @ w
    largest, l = z.amax(dim=1), torch.logsumexp(z, dim=1)
    given = (L >= 0) & (L < c)
    want = torch.where(given, z.gather(1, L.clamp(0, c - 1)[:, None])[:, 0] - l, torch.zeros_like(l))
    # a score's sum is off by at most SUM(d) of its terms' sizes, which add up to less than 3 sqrt(d) 2 on average here and never to five times that; exponents of up to 20, c / 32 + 40 additions
    bound = SUM(d) * 30 * math.sqrt(d) + U * (6 * 20 + c / 32 + 100)
    assert float((logp - want).abs().max()) <= 3 * bound and float((stats[:, 0] - largest).abs().max()) <= bound and float((stats[:, 1] - (l - largest)).abs().max()) <= 2 * bound
    scale = 1024.0 if name == "f16" else 1.0
    dlogp = (torch.rand(n, device="cuda") + 0.5) * (-scale / n)
    dX, dW = _gpu(torch, n, d, name, pad, offset), _gpu(torch, d, c, name, pad, offset)
    cbm.cbm_linear_log_probs_backward(X, W, L, stats, dlogp, dX, dW, workspace=ws)
    a = (dlogp * given).double()[:, None]
    dz = torch.exp(z - stats.double().sum(1, keepdim=True)).neg_()
    del z
    dz[torch.arange(n, device="cuda"), L.clamp(0, c - 1)] += 1.0
    dz *= a
    # a dz is off by its rounding and by what its exponent is off by
    of = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}[name] * 1.01 + 4 * bound
    least = 2.0 ** -25 * 2.0 ** -15 * float(dlogp.abs().max()) if name == "f16" else 0.0
    t = lambda a: a.t().contiguous()  # noqa: E731
    size = dz.abs()
    off = of * size + least + 4 * bound * a.abs() * 1e-3
    _within(dX, dz @ t(w), SUM(c) * (size @ t(w.abs())) + off @ t(w.abs()), name)
    _within(dW, t(x) @ dz, SUM(n) * (t(x.abs()) @ size) + t(x.abs()) @ off, name)
