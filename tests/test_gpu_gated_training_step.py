"""Training steps of a gated layer under a classifier, the operators as they are used together: forward pass, loss, gradients and orthogonal updates on one stream, each call's outputs against
the definition in 64 bits on the inputs that it had, and the whole step captured and replayed."""
import math

import numpy as np
import pytest

from oracle import train_oracle as orc
from test_gpu_gated_linear import TYPES, _check_backward as _check_gated_backward, _check_forward as _check_gated, _type
from test_gpu_layer_norm import ROUNDING, _numbers, env  # noqa: F401
from test_gpu_linear_log_probs import _check_backward as _check_classes_backward, _check_forward as _check_classes
from test_gpu_orthogonalise import _error_bound

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
SIZES = [(1, 24, 40, 9), (130, 40, 72, 50), (1031, 33, 47, 129), (5000, 64, 64, 10)]
RATE = 0.02


class Step:
    """X (n x k) -> gated layer (m) -> classes (c): the mean log probability of the labels goes up along orthogonal directions."""

    def __init__(self, torch, cbm, n, k, m, c, dtype, act="silu"):
        self.torch, self.cbm, self.act = torch, cbm, act
        g = torch.Generator(device="cuda").manual_seed(n)
        new = lambda *s: torch.randn(s, device="cuda", generator=g)  # noqa: E731
        self.x = new(n, k).to(dtype)
        self.weights = [(new(*s) * s[0] ** -0.5).to(dtype) for s in ((k, m), (k, m), (m, c))]
        # a teacher's labels, some of them missing
        self.labels = (self.x.float() @ new(k, c)).argmax(dim=1)
        if n > 4:
            self.labels[::5] = -1
        given = int((self.labels >= 0).sum())
        self.h, self.g, self.u, self.dh = (torch.empty((n, m), device="cuda", dtype=dtype) for _ in range(4))
        self.grads, self.updates = ([torch.empty_like(w) for w in self.weights] for _ in range(2))
        self.logp, self.stats, self.dlogp = torch.empty(n, device="cuda"), torch.empty((n, 2), device="cuda"), torch.full((n,), -1.0 / max(given, 1), device="cuda")
        need = [cbm.cbm_gated_linear_workspace_bytes(n, k, m, dtype), cbm.cbm_gated_linear_backward_workspace_bytes(n, k, m, dtype), cbm.cbm_linear_log_probs_workspace_bytes(n, m, c, dtype),
                cbm.cbm_linear_log_probs_backward_workspace_bytes(n, m, c, dtype)] + [cbm.cbm_orthogonalise_workspace_bytes(*w.shape, dtype) for w in self.weights]
        self.workspace = torch.full((max(need),), 255, dtype=torch.uint8, device="cuda")  # one for all calls, which follow each other

    def gradients(self):
        cbm, (wg, wu, wc), (dwg, dwu, dwc) = self.cbm, self.weights, self.grads
        cbm.cbm_gated_linear(self.x, wg, wu, self.h, self.g, self.u, self.act, self.workspace)
        cbm.cbm_linear_log_probs(self.h, wc, self.labels, self.logp, self.stats, self.workspace)
        cbm.cbm_linear_log_probs_backward(self.h, wc, self.labels, self.stats, self.dlogp, self.dh, dwc, self.workspace)
        cbm.cbm_gated_linear_backward(self.dh, self.x, wg, wu, self.g, self.u, None, dwg, dwu, self.act, self.workspace)
        for grad, update in zip(self.grads, self.updates):
            cbm.cbm_orthogonalise(grad, update, scale=RATE, workspace=self.workspace)

    def run(self):
        self.gradients()
        for w, update in zip(self.weights, self.updates):
            w.sub_(update)

    def state(self):
        return [t.clone() for t in (self.h, self.g, self.u, self.logp, self.stats, self.dh, *self.grads, *self.updates)]


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("sizes", SIZES)
def test_each_call_of_a_step(env, name, sizes):  # noqa: F811
    torch, cbm = env
    act = ("silu", "gelu", "relu")[sizes[0] % 3]
    step = Step(torch, cbm, *sizes, _type(torch, name), act)
    for _ in range(3):
        step.run()
    step.gradients()
    wg, wu, wc = step.weights
    _check_gated(step.x, wg, wu, step.h, step.g, step.u, name, act)
    _check_classes(step.h, wc, step.labels, step.logp, step.stats)
    # the slopes are made with the kept maxima and sums, as they are in the definition on them
    _check_classes_backward(step.h, wc, step.labels, step.stats, step.dlogp, step.dh, step.grads[2], name)
    _check_gated_backward((step.dh, step.x, wg, wu, step.g, step.u), [torch.zeros_like(step.x), *step.grads[:2]], name, act, (False, True, True))
    for grad, update in zip(step.grads, step.updates):
        exact = _numbers(grad)
        want = orc.orthogonalise(exact, scale=RATE)
        of_z = RATE * _error_bound(exact, 5) + U * np.linalg.norm(want)
        assert np.linalg.norm(_numbers(update) - want) <= of_z + ROUNDING[name] * (np.linalg.norm(want) + of_z) + (2.0 ** -25 * math.sqrt(want.size) if name == "f16" else 0.0)


@pytest.mark.parametrize("name", TYPES)
def test_captured_steps_are_the_eager_ones(env, name):  # noqa: F811
    """Replays with eager steps of another model and synchronizations between them, each against the same step run eagerly."""
    torch, cbm = env
    sizes = (1031, 33, 47, 129)
    one, two, other = (Step(torch, cbm, *sizes, _type(torch, name)) for _ in range(3))
    start = [w.clone() for w in one.weights]
    one.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        one.run()
    for w, s in zip(one.weights, start):
        w.copy_(s)
    for _ in range(4):
        graph.replay()
        other.run()
        two.run()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(one.state() + one.weights, two.state() + two.weights))
