"""The orthogonal update at sizes that go through each of its tiles, of 32 to 256 a side (test_product_rules_host.py holds the sizes to them), against the iteration in 64 bits on the device: all tiles of an output
checked apart, wide and tall, in place, odd strides; captured, and on two streams at once."""
import math

import pytest

from test_gpu_gated_linear import TYPES, _gpu
from test_gpu_layer_norm import ROUNDING, env  # noqa: F401

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
USUAL = (3.4445, -4.7750, 2.0315)
FLAT = (1.875, -1.25, 0.375)  # (slopes of up to 1.9: after two steps the bound is a quarter of a tile of 32 x 32 of the largest output; the usual one's is as large as one)
SIZES = [(513, 1537), (1025, 1031), (2049, 2051), (3001, 3003), (3073, 4001), (4097, 4099), (4353, 4361)]


def _largest(torch, gram):
    """A bound of the root of the largest eigenvalue: the trace of the 32nd power is at least its 32nd power."""
    size = float(gram.norm())
    power = gram / size
    for _ in range(5):
        power = power @ power
    return math.sqrt(size * float(power.trace()) ** (1 / 32))


def _iteration(torch, x, steps, abc, eps=1e-7):
    """Z after `steps`, and by how much products in fp32 may be off in the Frobenius norm: a sum of K terms by (K + 16) 2^-24 |P| |Q|; a step carries an earlier error on by at most the largest slope of
    a s + b s^3 + c s^5 up to the largest singular value."""
    a, b, c = abc
    z = x / (x.norm() + eps)
    s, l = z.shape
    error = 4 * U
    for _ in range(steps):
        gram = z @ z.t().contiguous()
        top = _largest(torch, gram) + error
        slope = max(abs(a + 3 * b * y + 5 * c * y * y) for y in ((top * i / 2000) ** 2 for i in range(2001)))
        size, of_gram = float(z.norm()), (l + 16) * U * float(z.norm()) ** 2
        p = b * gram + c * gram @ gram
        of_p = (abs(b) + 2 * abs(c) * top * top) * of_gram + (s + 20) * U * (abs(c) * float(gram.norm()) ** 2 + abs(b) * float(gram.norm()))
        error = slope * error + of_p * top + (s + 20) * U * (float(p.norm()) + abs(a)) * size
        z = a * z + p @ z
    return z, error


def _near(torch, got, want, of_z, name):
    """The whole, and every band of 32 rows and of 32 columns: a tile in the wrong place, or a row left out, is most of a band."""
    off = got.double() - want
    least = 2.0 ** -25 if name == "f16" else 0.0
    for of, size in ((off, want), (off.t(), want.t())):
        for r in range(0, of.shape[0], 32):
            band = size[r:r + 32]
            bound = of_z + ROUNDING[name] * (float(band.norm()) + of_z) + least * math.sqrt(band.numel())
            assert float(of[r:r + 32].norm()) <= bound, (r, float(of[r:r + 32].norm()), bound)


def _gradient(torch, m, n, name, pad, offset):
    """A few strong directions and noise: every entry of Z Z^T counts."""
    X = _gpu(torch, m, n, name, pad, offset)
    X.add_((torch.randn((m, 3), device="cuda") @ torch.randn((3, n), device="cuda")).to(X.dtype))
    return X


@pytest.mark.parametrize("name,steps,abc,pad,offset,in_place", [("f32", 2, FLAT, 0, 0, False), ("f32", 1, USUAL, 1, 3, False), ("bf16", 2, FLAT, 3, 1, True), ("f16", 1, USUAL, 8, 8, False), ("f32", 3, FLAT, 1, 1, True),
                                                               ("f32", 5, USUAL, 0, 0, True)])
@pytest.mark.parametrize("tall", [False, True])
@pytest.mark.parametrize("s,l", SIZES)
def test_against_64_bits(env, s, l, tall, name, steps, abc, pad, offset, in_place):  # noqa: F811
    torch, cbm = env
    torch.manual_seed(s + steps)
    m, n = (l, s) if tall else (s, l)
    X = _gradient(torch, m, n, name, pad, offset)
    whole = X._base if X._base is not None else X
    around = whole.clone()
    x = X.double()
    Y = X if in_place else _gpu(torch, m, n, name, pad, offset)
    need = cbm.cbm_orthogonalise_workspace_bytes(m, n, X.dtype)
    ws = torch.full((need + 4096,), 255, dtype=torch.uint8, device="cuda")
    cbm.cbm_orthogonalise(X, Y, steps=steps, coefficients=abc, workspace=ws[:need])
    assert bool((ws[need:] == 255).all())
    want, of_z = _iteration(torch, x.t().contiguous() if tall else x, steps, abc)
    _near(torch, Y, want.t() if tall else want, of_z, name)
    X.copy_(x.to(X.dtype))  # nothing beside the columns has changed, nor X where it is not the output
    assert torch.equal(whole.nan_to_num(5.0), around.nan_to_num(5.0))


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("s,l", [(513, 1537), (1031, 1025), (2049, 2051), (4097, 4099)])
def test_captured_and_on_streams(env, s, l, name):  # noqa: F811
    torch, cbm = env
    X = _gradient(torch, s, l, name, 0, 0)
    need = cbm.cbm_orthogonalise_workspace_bytes(s, l, X.dtype)
    outs, rooms = [torch.empty_like(X) for _ in range(3)], [torch.full((need,), 255, dtype=torch.uint8, device="cuda") for _ in range(3)]
    step = lambda i, stream=None: cbm.cbm_orthogonalise(X, outs[i], workspace=rooms[i], stream=stream)  # noqa: E731
    step(0)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(0)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for turn in range(3):
        X.copy_(torch.randn((s, l), device="cuda") * (turn + 1))
        graph.replay()
        torch.cuda.synchronize()
        for i in (1, 2):
            step(i, streams[i - 1])
        torch.cuda.synchronize()
        assert bool(outs[0].isfinite().all()) and torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


@pytest.mark.parametrize("s,l", SIZES)
def test_values_that_are_not_finite_and_zeros(env, s, l):  # noqa: F811
    torch, cbm = env
    ws = torch.empty(cbm.cbm_orthogonalise_workspace_bytes(s, l, torch.bfloat16), dtype=torch.uint8, device="cuda")
    X, Y = torch.zeros((s, l), dtype=torch.bfloat16, device="cuda"), torch.ones((s, l), dtype=torch.bfloat16, device="cuda")
    cbm.cbm_orthogonalise(X, Y, workspace=ws)
    assert not bool(Y.any())
    for value in (math.nan, math.inf):
        X[s - 1, l // 2] = value
        cbm.cbm_orthogonalise(X, Y, workspace=ws)
        assert bool(Y.isnan().all())
