"""Alternatives of scores with an offset, which the probabilities do not see: distinct fp32 values close together beside their size."""
import numpy as np
import pytest

from test_gpu_layer_norm import _matrix, env  # noqa: F401
from test_gpu_log_probs import _check, _scores

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("offset", [-1e6, -300.0, 300.0, 1000.0, 30000.0, 1e6])
@pytest.mark.parametrize("c", [5, 47, 133, 200, 257, 1000, 1500, 2015, 3000, 5000, 9000, 32000, 70000])
def test_alternatives_of_scores_with_an_offset(env, c, offset):  # noqa: F811
    torch, cbm = env
    rng = np.random.default_rng(c)
    for n in (1, 7) if c > 5000 else (7, 1100):
        z = (rng.standard_normal((n, c)) * 3 + offset).astype(np.float32)
        z[0, rng.random(c) < 0.3] = -np.inf
        z[-1] = offset + np.arange(c) % 977 * float(np.spacing(np.float32(offset)))  # one unit of the last place apart, and equal
        Z, _ = _matrix(torch, z, "f32", 1)
        labels = rng.integers(-1, c, n)
        for top in (1, 8, 20, 32):
            _check(torch, Z, labels, _scores(torch, cbm, Z, labels, top), top)
