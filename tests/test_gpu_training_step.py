"""One training step of the example's GCN, products and operators together, against the same step in 64 bits on what was kept, and its training."""
import importlib.util
import os

import numpy as np
import pytest

import workloads as wl
from oracle import train_oracle as orc

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    import torch

    assert torch.cuda.is_available(), "this test needs the MI355X"
    spec = importlib.util.spec_from_file_location("train_gcn", os.path.join(ROOT, "examples", "train_gcn.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def _normalised(graph):
    a = np.zeros((graph.n, graph.n))
    for i in range(graph.n):
        a[i, graph.colidx[graph.rowptr[i]:graph.rowptr[i + 1]]] = 1.0
    np.fill_diagonal(a, 1.0)
    d = a.sum(axis=1) ** -0.5
    return d[:, None] * a * d[None, :]


def _close(got, want, tol, what):
    """In the 2-norm: the steps between are sums of thousands of fp32 terms, 1e-5 of the result's norm covers them as it does a product's (1e-5 a row)."""
    err = np.linalg.norm(got.double().cpu().numpy() - want) / np.linalg.norm(want)
    assert err <= tol, (what, err)


@pytest.mark.parametrize("features,hidden,classes", [(64, 64, 8), (33, 47, 3)])
def test_step_against_64_bits(example, features, hidden, classes):
    import torch

    graph = wl.tiny_graph()
    x, labels, _ = example.planted_task(graph, features, classes)
    model = example.Gcn(graph, features, hidden, classes)
    model.gamma.copy_(1 + 0.1 * torch.randn(hidden, device="cuda"))
    model.beta.copy_(0.1 * torch.randn(hidden, device="cuda"))
    model.forward(x, labels)
    a = _normalised(graph)
    num = lambda t: t.double().cpu().numpy()  # noqa: E731
    X, w0, w1, L = num(x), num(model.w0), num(model.w1), labels.cpu().numpy()
    h = np.maximum(a @ (X @ w0), 0)
    v, m, r = orc.layer_norm(h, num(model.gamma), num(model.beta), float(np.float32(1e-5)))
    out = a @ (v @ w1)
    logp, entropy, stats, _, best = orc.log_probs(out, L, 1)
    _close(model.out, out, 1e-5, "scores")
    _close(model.logp, logp, 1e-5, "log probabilities")
    _close(model.entropy, entropy, 1e-5, "entropy")
    assert np.mean(model.answer[:, 0].cpu().numpy() == best[:, 0]) > 0.999  # (scores that differ by rounding may change places)
    # the backward pass starts from what was kept, so the reference does: the 8-bit values, and the statistics and scores as the kernels left them
    kept = [orc.kept_values(c.q.cpu().numpy().astype(np.int64), c.steps.cpu().numpy().astype(np.int64) - 127) for c in (model.kept_x, model.kept_h, model.kept_v)]
    for values, exact, k in zip(kept, (X, h, v), (features, hidden, hidden)):
        blocks = np.repeat(np.stack([np.abs(exact[:, i:i + 32]).max(axis=1) for i in range(0, k, 32)], axis=1), 32, axis=1)[:, :k]
        assert np.all(np.abs(values - exact) <= blocks / 64 * 1.001)  # a step is at most a 64th of the block's largest value
    scores, mean, rstd, st = (num(t) for t in (model.out, model.mean, model.rstd, model.stats))
    g = model.backward(labels)
    count = (L >= 0).sum()
    dout = orc.log_probs_backward(scores, L, st, np.zeros(graph.n), np.full(graph.n, np.float32(-1.0) / np.float32(count)), np.zeros(graph.n))
    dz1 = a @ dout
    dv = dz1 @ w1.T
    dh, dgamma, dbeta = orc.layer_norm_backward(dv, kept[1], num(model.gamma), mean, rstd)
    dz0 = a @ np.where(kept[1] > 0, dh, 0.0)
    for name, want in (("w1", kept[2].T @ dz1), ("gamma", dgamma), ("beta", dbeta), ("w0", kept[0].T @ dz0)):
        _close(g[name], want, 1e-5, name)
    # and what 8 bits do to the gradients: the exact activations' own, to the size of a step
    dh, dgamma, dbeta = orc.layer_norm_backward(dv, h, num(model.gamma), m, r)
    for name, want in (("w1", v.T @ dz1), ("gamma", dgamma), ("w0", X.T @ (a @ np.where(h > 0, dh, 0.0)))):
        _close(g[name], want, 1 / 64, name)


def test_training_learns(example):
    losses, right = example.main(["--graph", "tiny", "--steps", "40"])
    assert losses[-1] < 0.25 * losses[0] and right > 0.9
