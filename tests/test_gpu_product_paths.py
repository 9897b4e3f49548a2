"""The gated layer and the log probabilities of a layer's classes at sizes that go through LDS: any matrices, whole units, copies and turned weights, shares of K (test_product_rules_host.py holds each size to its
kernels).  Captured and replayed, on two streams at once, with values that are not finite, with classes ruled out."""
import math

import numpy as np
import pytest

from oracle import train_oracle as orc
from test_gpu_gated_linear import TYPES, _gpu
from test_gpu_layer_norm import _matrix, _numbers, env  # noqa: F401

pytestmark = pytest.mark.gpu
GATED = [(9001, 17, 300), (4100, 136, 1024), (12001, 515, 4099), (4097, 512, 12288)]
CLASSES = [(9001, 17, 300), (2304, 320, 4096), (12001, 515, 8199), (4097, 512, 24576)]


def _workspace(torch, need):
    return torch.full((need,), 255, dtype=torch.uint8, device="cuda")


class Gated:
    def __init__(self, torch, cbm, n, k, m, name, act="gelu"):
        torch.manual_seed(n + m)
        self.torch, self.cbm, self.act = torch, cbm, act
        self.X, self.Wg, self.Wu = _gpu(torch, n, k, name, 0, 0), _gpu(torch, k, m, name, 0, 0, k ** -0.5), _gpu(torch, k, m, name, 0, 0, k ** -0.5)
        self.dH = _gpu(torch, n, m, name, 0, 0, 0.01)
        d = self.X.dtype
        self.need = max(cbm.cbm_gated_linear_workspace_bytes(n, k, m, d), cbm.cbm_gated_linear_backward_workspace_bytes(n, k, m, d))

    def outputs(self):
        return [self.torch.full_like(t, 7) for t in (self.dH, self.dH, self.dH, self.X, self.Wg, self.Wu)]

    def run(self, outs, ws, stream=None):
        self.cbm.cbm_gated_linear(self.X, self.Wg, self.Wu, *outs[:3], activation=self.act, workspace=ws, stream=stream)
        self.cbm.cbm_gated_linear_backward(self.dH, self.X, self.Wg, self.Wu, outs[1], outs[2], *outs[3:], activation=self.act, workspace=ws, stream=stream)


class Classes:
    def __init__(self, torch, cbm, n, d, c, name):
        torch.manual_seed(n + c)
        self.torch, self.cbm = torch, cbm
        self.X, self.W = _gpu(torch, n, d, name, 0, 0), _gpu(torch, d, c, name, 0, 0, 3 * d ** -0.5)
        self.L = torch.randint(0, c, (n,), device="cuda")
        self.dlogp = -torch.rand(n, device="cuda") - 0.1
        t = self.X.dtype
        self.need = max(cbm.cbm_linear_log_probs_workspace_bytes(n, d, c, t), cbm.cbm_linear_log_probs_backward_workspace_bytes(n, d, c, t))

    def outputs(self):
        n = len(self.X)
        return [self.torch.full((n,), 7.0, device="cuda"), self.torch.full((n, 2), 7.0, device="cuda"), self.torch.full_like(self.X, 7), self.torch.full_like(self.W, 7)]

    def run(self, outs, ws, stream=None):
        self.cbm.cbm_linear_log_probs(self.X, self.W, self.L, outs[0], outs[1], workspace=ws, stream=stream)
        self.cbm.cbm_linear_log_probs_backward(self.X, self.W, self.L, outs[1], self.dlogp, outs[2], outs[3], workspace=ws, stream=stream)


def _captured_and_on_streams(torch, step, change):
    """Replays after changes of the inputs, with eager work between, and two calls at once with a workspace each: the same bits."""
    outs, rooms = step.outputs(), [_workspace(torch, step.need) for _ in range(3)]
    step.run(outs, rooms[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step.run(outs, rooms[0])
    streams = [torch.cuda.Stream() for _ in range(2)]
    for turn in range(3):
        change(turn)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outs]
        assert all(bool(t.isfinite().all()) for t in got)
        apart = [step.outputs() for _ in range(2)]
        torch.cuda.synchronize()
        for s, o, w in zip(streams, apart, rooms[1:]):
            step.run(o, w, s)
        torch.cuda.synchronize()
        for o in apart:
            assert all(torch.equal(a, b) for a, b in zip(got, o))


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("n,k,m", GATED)
def test_gated_layer_captured_and_on_streams(env, name, n, k, m):  # noqa: F811
    torch, cbm = env
    step = Gated(torch, cbm, n, k, m, name)

    def change(turn):
        step.X.copy_(torch.randn((n, k), device="cuda") * (turn + 1))
        step.dH.copy_(torch.randn((n, m), device="cuda") * (0.01, 2.0 ** -18, 1.0)[turn])  # (fp16: slopes made once, twice, and once or twice)

    _captured_and_on_streams(torch, step, change)


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("n,d,c", CLASSES)
def test_classes_captured_and_on_streams(env, name, n, d, c):  # noqa: F811
    torch, cbm = env
    step = Classes(torch, cbm, n, d, c, name)

    def change(turn):
        step.X.copy_(torch.randn((n, d), device="cuda"))
        step.L.copy_(torch.randint(-1, c + 1, (n,), device="cuda"))
        step.dlogp.mul_(0.1)

    _captured_and_on_streams(torch, step, change)


def _other(torch, n, bad):
    keep = torch.ones(n, dtype=torch.bool, device="cuda")
    keep[bad] = False
    return keep


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("n,k,m", GATED)
def test_gated_layer_with_values_that_are_not_finite(env, name, n, k, m):  # noqa: F811
    """They reach the sums that they are part of, and leave the bits of all others."""
    torch, cbm = env
    step, ws = Gated(torch, cbm, n, k, m, name, "silu"), None
    ws = _workspace(torch, step.need)
    before = step.outputs()
    bad = [3, n // 2, n - 1]
    rows, columns, inner = _other(torch, n, bad), _other(torch, m, [1, m - 1]), _other(torch, k, [5])
    step.X[bad], step.dH[bad] = 0.0, 0.0
    step.run(before, ws)
    for value in (math.nan, math.inf, -math.inf):
        x = step.X.clone()
        step.X[bad, 5] = value
        after = step.outputs()
        step.run(after, ws)
        for a, b in zip(before[:4], after[:4]):
            assert torch.equal(a[rows], b[rows])
        for t in after[1:3]:
            assert not bool(t[~rows].isfinite().any())
        # (dH of zero times what is not finite: NaN in those rows' slopes, and so in all of the weights' gradients)
        assert not bool(after[3][~rows].isfinite().any()) and not any(bool(t.isfinite().any()) for t in after[4:])
        step.X.copy_(x)
        # as the backward pass's own input: the rows of the weights' gradients that the column of X makes
        step.X[bad, 5] = value
        grads = step.outputs()
        cbm.cbm_gated_linear_backward(step.dH, step.X, step.Wg, step.Wu, before[1], before[2], *grads[3:], activation="silu", workspace=ws)
        assert torch.equal(grads[3], before[3])
        for a, b in zip(before[4:], grads[4:]):
            assert torch.equal(a[inner], b[inner]) and not bool(b[5].isfinite().any())
        step.X.copy_(x)
        # weights: the columns that they are in
        w = step.Wu.clone()
        step.Wu[7, [1, m - 1]] = value
        after = step.outputs()
        cbm.cbm_gated_linear(step.X, step.Wg, step.Wu, *after[:3], activation="silu", workspace=ws)
        for a, b in zip(before[:3], after[:3]):
            assert torch.equal(a[:, columns], b[:, columns])
        assert torch.equal(before[1], after[1]) and not bool(after[2][:, ~columns].isfinite().any())
        step.Wu.copy_(w)


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("n,d,c", CLASSES)
def test_classes_with_values_that_are_not_finite(env, name, n, d, c):  # noqa: F811
    torch, cbm = env
    step = Classes(torch, cbm, n, d, c, name)
    ws = _workspace(torch, step.need)
    bad = [3, n // 2, n - 1]
    rows = _other(torch, n, bad)
    step.L[n // 2] = -1
    before = step.outputs()
    step.run(before, ws)
    x = step.X.clone()
    for value in (math.nan, math.inf):
        step.X[bad, 5] = value
        after = step.outputs()
        cbm.cbm_linear_log_probs(step.X, step.W, step.L, after[0], after[1], workspace=ws)
        for a, b in zip(before[:2], after[:2]):
            assert torch.equal(a[rows], b[rows])
        assert bool(after[1][~rows].isnan().all()) and bool(after[0][[3, n - 1]].isnan().all()) and float(after[0][n // 2]) == 0.0
        step.X.copy_(x)
    w = step.W.clone()
    step.W[1, c - 1] = math.nan
    after = step.outputs()
    cbm.cbm_linear_log_probs(step.X, step.W, step.L, after[0], after[1], workspace=ws)
    assert bool(after[1].isnan().all()) and bool(after[0][step.L >= 0].isnan().all())
    step.W.copy_(w)
    # a row's infinite or missing slope is its own, and that of the weights' sums
    some = []
    for value in (0.0, math.nan, math.inf):
        step.dlogp[[3, n - 1]] = value
        outs = step.outputs()
        cbm.cbm_linear_log_probs_backward(step.X, step.W, step.L, before[1], step.dlogp, outs[2], outs[3], workspace=ws)
        some.append(outs[2])
    rows = _other(torch, n, [3, n - 1])
    assert torch.equal(some[0][rows], some[1][rows]) and torch.equal(some[0][rows], some[2][rows])
    assert not bool(some[0][~rows].any()) and not bool(some[1][~rows].isfinite().any()) and not bool(some[2][~rows].isfinite().any())
    for size in (0.0, 1e-42):
        outs = step.outputs()
        cbm.cbm_linear_log_probs_backward(step.X, step.W, step.L, before[1], torch.full_like(step.dlogp, size), outs[2], outs[3], workspace=ws)
        assert all(float(t.abs().max()) <= 1e-37 for t in outs[2:])


@pytest.mark.parametrize("name", ["bf16", "f16"])
@pytest.mark.parametrize("n,d,c", [(9001, 17, 300), (2304, 320, 4096), (70001, 9, 20)])
def test_classes_ruled_out(env, name, n, d, c):  # noqa: F811
    """A last feature of one and a weight of -infinity rule a class out: it has no share and gets no gradient.  With all of them ruled out a row has no distribution, and nothing comes back from it."""
    torch, cbm = env
    rng = np.random.default_rng(n)
    x, w = rng.standard_normal((n, d)), rng.standard_normal((d, c)) / math.sqrt(d)
    x[:, -1] = 1.0
    out = rng.random(c) < 0.3
    w[-1, out] = -math.inf
    labels = rng.integers(0, c, n)
    X, W, L = _matrix(torch, x, name, 0)[0], _matrix(torch, w, name, 0)[0], torch.from_numpy(labels).cuda()
    ws = _workspace(torch, max(cbm.cbm_linear_log_probs_workspace_bytes(n, d, c, X.dtype), cbm.cbm_linear_log_probs_backward_workspace_bytes(n, d, c, X.dtype)))
    logp, stats = torch.empty(n, device="cuda"), torch.empty((n, 2), device="cuda")
    cbm.cbm_linear_log_probs(X, W, L, logp, stats, workspace=ws)
    want = orc.log_probs(_numbers(X) @ _numbers(W), labels)
    same = lambda a, b: np.all((a == b) | (np.abs(a - b) <= 1e-4))  # noqa: E731  (which classes are left, not the roundings)
    with np.errstate(invalid="ignore"):
        assert same(_numbers(logp), want[0]) and same(_numbers(stats), want[2])
    # the weights' gradients: columns of classes that are ruled out have nothing but their own rows' labels
    X0, dW = X.clone(), torch.full_like(W, 7)
    dlogp = torch.where(torch.from_numpy(out[labels]).cuda(), 0.0, -1.0)
    cbm.cbm_linear_log_probs_backward(X0, W, L, stats, dlogp, None, dW, workspace=ws)
    assert not bool(dW[:, torch.from_numpy(out).cuda()].any()) and bool(dW.isfinite().all()) and bool(dW.any())
    W[:-1], W[-1] = 0.0, -math.inf
    cbm.cbm_linear_log_probs(X, W, L, logp, stats, workspace=ws)
    assert bool((logp == -math.inf).all()) and bool((stats[:, 0] == -math.inf).all())
    dX, dW = torch.full_like(X, 7), torch.full_like(W, 7)
    cbm.cbm_linear_log_probs_backward(X, torch.zeros_like(W), L, torch.full((n, 2), -math.inf, device="cuda"), torch.ones(n, device="cuda"), dX, dW, workspace=ws)
    assert not bool(dX.any()) and not bool(dW.any())
