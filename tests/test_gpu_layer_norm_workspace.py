"""Sums of the layer norm's weights' gradients in the workspace that was asked for, and no further."""
import pytest

from test_gpu_layer_norm import U, env  # noqa: F401

pytestmark = pytest.mark.gpu
BEHIND = 1 << 16


@pytest.mark.parametrize("name", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("n,k", [(700, 1536), (700, 1540), (2500, 3072), (600, 3080), (600, 12289), (500, 16384), (500, 16392), (300, 40001), (20, 300000), (5, 1 << 20)])
def test_sums_stay_within_the_workspace(env, n, k, name):  # noqa: F811
    torch, cbm = env
    gen = torch.Generator(device="cuda").manual_seed(k)
    X, dY = (torch.randn((n, k), device="cuda", generator=gen).to(getattr(torch, name)) for _ in range(2))
    mean, rstd = torch.randn(n, device="cuda", generator=gen), torch.rand(n, device="cuda", generator=gen) + 0.5
    need = cbm.cbm_layer_norm_workspace_bytes(n, k)
    room = torch.full((need + BEHIND,), 255, dtype=torch.uint8, device="cuda")  # (NaN all over)
    dgamma, dbeta = torch.empty(k, device="cuda"), torch.empty(k, device="cuda")
    cbm.cbm_layer_norm_backward(dY, X, None, mean, rstd, torch.empty_like(X), dgamma, dbeta, room[:need])
    assert bool((room[need:] == 255).all())
    h, dy = (X.double() - mean.double()[:, None]) * rstd.double()[:, None], dY.double()
    depth = n + 10  # additions on the way into a sum
    for got, terms in ((dgamma, dy * h), (dbeta, dy)):
        assert bool(((got.double() - terms.sum(dim=0)).abs() <= depth * U * terms.abs().sum(dim=0)).all())
