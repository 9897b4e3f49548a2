"""Log probabilities of so many rows and classes that the rows' parts go through the workspace in bands, the last one short: every row against 64 bits."""
import math

import pytest

from test_gpu_gated_linear import SUM, TYPES, _gpu
from test_gpu_layer_norm import env  # noqa: F401

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("n,d,c,bits,pad", [(66001, 8, 66002, 64, 0), (17003, 11, 600001, 32, 1)])
def test_every_row(env, name, n, d, c, bits, pad):  # noqa: F811
    torch, cbm = env
    torch.manual_seed(n)
    X, W = _gpu(torch, n, d, name, pad, pad), _gpu(torch, d, c, name, pad, pad, 3 * d ** -0.5)
    need = cbm.cbm_linear_log_probs_workspace_bytes(n, d, c, X.dtype)
    assert n * (c // 64) * 8 > need  # more than one band
    L = torch.randint(-1, c + 1, (n,), device="cuda").to(torch.int64 if bits == 64 else torch.int32)
    whole = torch.full((need + (1 << 16),), 255, dtype=torch.uint8, device="cuda")
    logp, stats = torch.full((n,), math.nan, device="cuda"), torch.full((n, 2), math.nan, device="cuda")
    cbm.cbm_linear_log_probs(X, W, L, logp, stats, workspace=whole[:need])
    assert bool((whole[need:] == 255).all())
    w, worst = W.double(), 0.0
    for r in range(0, n, 4096):
        x, label = X[r:r + 4096].double(), L[r:r + 4096].long()
        z = x @ w
        largest, l = z.amax(dim=1), torch.logsumexp(z, dim=1)
        given = (label >= 0) & (label < c)
        want = torch.where(given, z.gather(1, label.clamp(0, c - 1)[:, None])[:, 0] - l, torch.zeros_like(l))
        # a score is off by SUM(d) of its terms' sizes, |x| |w| at most; exponents of up to 60, a share of 64 classes and the joining of at most c / 64 of them over 64 lanes
        of_z = SUM(d) * x.norm(dim=1) * w.norm(dim=0).max()
        bound = of_z * 2 + U * (6 * 60 + 64 + c / 4096 + 100)
        assert bool(((stats[r:r + 4096, 0] - largest).abs() <= of_z + U * largest.abs()).all())
        assert bool(((stats[r:r + 4096, 1] - (l - largest)).abs() <= bound + 4 * U * l.abs()).all())
        assert bool(((logp[r:r + 4096] - want).abs() <= 2 * bound + 8 * U * want.abs()).all())
        worst = max(worst, float((logp[r:r + 4096] - want).abs().max()))
    assert worst > 0.0
    # the same without statistics, and without log probabilities
    again, st = torch.empty_like(logp), torch.empty_like(stats)
    cbm.cbm_linear_log_probs(X, W, L, again, None, workspace=whole[:need])
    cbm.cbm_linear_log_probs(X, W, None, None, st, workspace=whole[:need])
    assert torch.equal(again, logp) and torch.equal(st, stats)
