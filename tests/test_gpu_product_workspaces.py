"""The operators that are made of products write in the workspace that was asked for and no further: bytes on both sides of it stay as they were, at sizes whose copies, slopes, sums and shares end there."""
import math

import pytest

from test_gpu_gated_linear import SUM, TYPES, _gpu, _within
from test_gpu_layer_norm import ROUNDING, _type, env  # noqa: F401

pytestmark = pytest.mark.gpu
AROUND = 1 << 16
LEAST_F16 = 2.0 ** -25


class Room:
    """`need` bytes of NaN between bytes that have to stay."""

    def __init__(self, torch, need):
        self.whole = torch.full((AROUND + (need + 15) // 16 * 16 + AROUND,), 171, dtype=torch.uint8, device="cuda")
        self.own = self.whole[AROUND:AROUND + need]
        self.own.fill_(255)
        self.need = need

    def kept(self):
        return bool((self.whole[:AROUND] == 171).all()) and bool((self.whole[AROUND + self.need:] == 171).all())


# the first four (16 bits): copies whose last rows are zeros up to a multiple of eight, with nothing behind them
LARGE = [(8192, 1537, 2049, 0), (8147, 1734, 2285, 0), (8192, 2047, 2047, 1), (8869, 1634, 2496, 1), (1030, 1003, 25000, 0)]
SMALL = [(1, 1, 1, 0), (7, 130, 65, 1), (300, 40, 30, 3), (5000, 65, 7, 1), (9001, 17, 300, 0), (20000, 64, 72, 0), (33, 40, 8200, 1)]


@pytest.mark.parametrize("name,n,k,m,pad", [(t, *s) for t in TYPES for s in SMALL] + [(t, *s) for t in ("bf16", "f16") for s in LARGE])
def test_gated_layer(env, name, n, k, m, pad):  # noqa: F811
    torch, cbm = env
    torch.manual_seed(n)
    X, Wg, Wu = _gpu(torch, n, k, name, pad, 0), _gpu(torch, k, m, name, pad, 0, k ** -0.5), _gpu(torch, k, m, name, pad, 0, k ** -0.5)
    G, U_, H, dH = (_gpu(torch, n, m, name, pad, 0) for _ in range(4))
    room = Room(torch, cbm.cbm_gated_linear_workspace_bytes(n, k, m, X.dtype))
    cbm.cbm_gated_linear(X, Wg, Wu, H, activation="relu", workspace=room.own)
    assert room.kept()
    x, wg, wu = X.double(), Wg.double(), Wu.double()
    g, u = x @ wg, x @ wu
    of_g, of_u = SUM(k) * (x.abs() @ wg.abs()), SUM(k) * (x.abs() @ wu.abs())
    _within(H, g.clamp_min(0) * u, of_g * (u.abs() + of_u) + g.abs() * of_u, name)
    del g, u, of_g, of_u
    outs = [_gpu(torch, *s, name, pad, 0) for s in ((n, k), (k, m), (k, m))]
    room = Room(torch, cbm.cbm_gated_linear_backward_workspace_bytes(n, k, m, X.dtype))
    cbm.cbm_gated_linear_backward(dH, X, Wg, Wu, G, U_, *outs, activation="relu", workspace=room.own)
    assert room.kept()
    dh, g, u = dH.double(), G.double(), U_.double()
    du, dg = dh * g.clamp_min(0), dh * u * (g > 0)
    t = lambda a: a.t().contiguous()  # noqa: E731
    one = torch.ones((n, m), dtype=torch.float64, device="cuda")
    # dG and dU: two products in fp32 and the type's rounding, fp16's smallest values among them; then a sum of terms
    half, least = 1.01 * ROUNDING[name] + 4 * 2.0 ** -24, LEAST_F16 if name == "f16" else 0.0
    for got, want, terms, off in ((outs[0], dg @ t(wg) + du @ t(wu), dg.abs() @ t(wg.abs()) + du.abs() @ t(wu.abs()), one @ t(wg.abs()) + one @ t(wu.abs())),
                                  (outs[1], t(x) @ dg, t(x.abs()) @ dg.abs(), t(x.abs()) @ one), (outs[2], t(x) @ du, t(x.abs()) @ du.abs(), t(x.abs()) @ one)):
        _within(got, want, (half + SUM(max(n, 2 * m + 128))) * terms + least * off, name)


@pytest.mark.parametrize("name,n,d,c,pad", [(t, *s) for t in TYPES for s in SMALL + [(262147, 4, 1100, 0)]] + [(t, n, d, 2 * c, pad) for t in ("bf16", "f16") for n, d, c, pad in LARGE])
def test_classes(env, name, n, d, c, pad):  # noqa: F811
    torch, cbm = env
    torch.manual_seed(n)
    X, W = _gpu(torch, n, d, name, pad, 0), _gpu(torch, d, c, name, pad, 0, 3 * d ** -0.5)
    L = torch.randint(-1, c + 1, (n,), device="cuda")
    logp, stats, dlogp = torch.empty(n, device="cuda"), torch.empty((n, 2), device="cuda"), torch.full((n,), -1.0, device="cuda")
    dX, dW = _gpu(torch, n, d, name, pad, 0), _gpu(torch, d, c, name, pad, 0)
    room = Room(torch, cbm.cbm_linear_log_probs_workspace_bytes(n, d, c, X.dtype))
    cbm.cbm_linear_log_probs(X, W, L, logp, stats, workspace=room.own)
    assert room.kept()
    room = Room(torch, cbm.cbm_linear_log_probs_backward_workspace_bytes(n, d, c, X.dtype))
    cbm.cbm_linear_log_probs_backward(X, W, L, stats, dlogp, dX, dW, workspace=room.own)
    assert room.kept()
    z = X.double() @ W.double()
    lse = torch.logsumexp(z, dim=1)
    given = (L >= 0) & (L < c)
    want = torch.where(given, z.gather(1, L.clamp(0, c - 1)[:, None])[:, 0] - lse, torch.zeros_like(lse))
    # (how near the values come is measured elsewhere: a score's sum, exponents of up to 30, additions)
    assert float((logp - want).abs().max()) <= 3 * SUM(d) * 30 * math.sqrt(d) + 2.0 ** -24 * (6 * 30 + c / 32 + 100)
    dz = torch.exp(z.sub_(lse[:, None])).neg_()
    dz[torch.arange(n, device="cuda"), L.clamp(0, c - 1)] += 1.0
    dz *= -given.double()[:, None]
    # in the 2-norm, where terms of either sign add up: the type's rounding of each dz and of the results, and scores that are off in fp32
    tol = {"f32": 1e-5, "bf16": 2.0 ** -7, "f16": 2.0 ** -10}[name]
    for got, want in ((dX, dz @ W.double().t().contiguous()), (dW, X.double().t().contiguous() @ dz)):
        assert float((got.double() - want).norm()) <= tol * float(want.norm()) + (LEAST_F16 * math.sqrt(want.numel()) if name == "f16" else 0.0) + 1e-30


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("m,n", [(1, 1), (64, 64), (65, 129), (500, 129), (513, 1537), (1025, 1031)])
def test_update(env, name, m, n):  # noqa: F811
    torch, cbm = env
    X, Y = _gpu(torch, m, n, name, 1, 0), _gpu(torch, m, n, name, 1, 0)
    room = Room(torch, cbm.cbm_orthogonalise_workspace_bytes(m, n, _type(torch, name)))
    cbm.cbm_orthogonalise(X, Y, workspace=room.own)
    assert room.kept() and bool(Y.isfinite().all())
