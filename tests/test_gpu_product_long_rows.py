"""The gated layer with rows of millions of values: 256 rows of a tile lie further apart than 32 bits reach.  Whole numbers, whose sums are exact in fp32."""
import pytest

from test_gpu_layer_norm import env  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("k,pad", [((1 << 23) + 35 * 2048, 1), ((1 << 23) + 35 * 2048, 0), ((1 << 22) - 8, 1)])
def test_every_row_is_its_own(env, k, pad):  # noqa: F811
    torch, cbm = env
    n, m = 1024, 128
    torch.manual_seed(0)
    whole = torch.empty((n, k + pad), dtype=torch.float16, device="cuda")
    X = whole[:, :k]
    for r in range(0, n, 64):
        X[r:r + 64] = torch.randint(-1, 2, (64, k), dtype=torch.int8, device="cuda")
    Wg, Wu = (torch.randint(0, 2, (k, m), dtype=torch.int8, device="cuda").half() for _ in range(2))
    want = [torch.zeros((n, m), dtype=torch.float64, device="cuda") for _ in range(2)]
    for a in range(0, k, 1 << 19):
        x = X[:, a:a + (1 << 19)].double()
        for sums, w in zip(want, (Wg, Wu)):
            sums.addmm_(x, w[a:a + (1 << 19)].double())
    assert max(float(w.abs().max()) for w in want) < 2 ** 24
    H, G, U = (torch.empty((n, m), dtype=torch.float16, device="cuda") for _ in range(3))
    ws = torch.empty(cbm.cbm_gated_linear_workspace_bytes(n, k, m, X.dtype), dtype=torch.uint8, device="cuda")
    cbm.cbm_gated_linear(X, Wg, Wu, H, G, U, activation="relu", workspace=ws)
    for got, exact in zip((G, U), want):
        assert torch.equal(got, exact.half())
