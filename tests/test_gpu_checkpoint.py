"""Activations in 8 bits and their use in the backward pass, through the C ABI against the definition in 64 bits: what is kept and restored bit for bit, the weights'
gradient exactly on whole numbers and within a derived bound on others."""
import math

import numpy as np
import pytest

from oracle import train_oracle as orc
from test_gpu_layer_norm import _matrix, _numbers, _type, _untouched, env  # noqa: F401

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
WIDTHS = [1, 2, 3, 4, 5, 7, 8, 9, 31, 32, 33, 39, 47, 63, 64, 65, 100, 127, 128, 129, 255, 256, 257, 500, 1000, 1025, 4100, 16399]


def _room(torch, n, k, pad):
    """Buffers for Q and E with `pad` bytes of 77 beside each row."""
    q = torch.full((n, k + pad), 77, dtype=torch.int8, device="cuda")
    e = torch.full((n, -(-k // 32) + pad), 77, dtype=torch.uint8, device="cuda")
    return q[:, :k], e[:, :-(-k // 32)], q, e


def _kept(Q, E):
    return Q.cpu().numpy().astype(np.int64), E.cpu().numpy().astype(np.int64) - 127


def _activations(rng, n, k):
    """Values of all sizes: rows from 2^-140 to 2^120, zeros, halves of steps, a block of zeros."""
    x = rng.standard_normal((n, k)) * np.exp2(rng.integers(-20, 10, (n, 1)))
    x[rng.random((n, k)) < 0.3] = 0.0
    if n > 4:
        x[1] *= 2.0 ** -120
        x[2] *= 2.0 ** 100
        x[3, ::2] = (rng.integers(0, 255, x[3, ::2].shape) - 127) / 2.0
        x[4, :32] = 0.0
    return x


@pytest.mark.parametrize("name", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("k", WIDTHS)
def test_kept_and_restored_bit_for_bit(env, name, k):  # noqa: F811
    torch, cbm = env
    rng = np.random.default_rng(k)
    for n, pad, offset in ((1, 0, 0), (7, 3, 1), (67, 0, 0)) + (((3000, 4, 4),) if k <= 500 else ()):
        x = _activations(rng, n, k)
        if name == "f16":
            x = np.clip(x, -65504, 65504)
        X, _ = _matrix(torch, x, name, pad, offset)
        Q, E, wq, we = _room(torch, n, k, pad)
        cbm.cbm_checkpoint_save(X, Q, E)
        q, e = orc.keep(_numbers(X))
        got_q, got_e = _kept(Q, E)
        assert np.array_equal(got_q, q) and np.array_equal(got_e, e), (n, pad)
        assert bool((wq[:, k:] == 77).all()) and bool((we[:, E.shape[1]:] == 77).all()), "wrote outside the columns"
        for out in ("f32", "bf16", "f16"):
            B, whole = _matrix(torch, np.zeros((n, k)), out, pad, offset)
            cbm.cbm_checkpoint_restore(Q, E, B)
            want = torch.from_numpy(orc.kept_values(q, e)).to(_type(torch, out))  # (64 bits to 16 directly: the values are bf16 values)
            assert torch.equal(B.cpu(), want) and (out == "f16" or np.array_equal(_numbers(B), orc.kept_values(q, e))), (n, pad, out)
            _untouched(torch, B, whole, offset)
            dY, _ = _matrix(torch, rng.standard_normal((n, k)), out, pad + 1, offset)
            dX, whole = _matrix(torch, np.zeros((n, k)), out, pad, offset)
            cbm.cbm_checkpoint_relu_backward(Q, E, dY, dX)
            assert np.array_equal(_numbers(dX), orc.relu_backward(q, e, _numbers(dY))), (n, pad, out)
            _untouched(torch, dX, whole, offset)
            cbm.cbm_checkpoint_relu_backward(Q, E, dY, dY)  # in place
            assert torch.equal(dY, dX)


def test_extreme_values(env):  # noqa: F811
    torch, cbm = env
    big = float(np.finfo(np.float32).max)
    rows = [[big, -big, 1.0, 0.0], [2.0 ** -149, -(2.0 ** -149), 0.0, -0.0], [2.0 ** -126, 2.0 ** -127, 2.0 ** -133, 0], [127.5, 126.5, 0.5, 1.5], [1.0, 1e-30, -1e-38, 2.0 ** -149]]
    X = torch.zeros((len(rows), 40), device="cuda")
    X[:, :4] = torch.tensor(rows, device="cuda")
    X[:, 36:] = torch.tensor(rows, device="cuda")
    Q, E, _, _ = _room(torch, len(rows), 40, 0)
    cbm.cbm_checkpoint_save(X, Q, E)
    q, e = orc.keep(_numbers(X))
    assert np.array_equal(_kept(Q, E)[0], q) and np.array_equal(_kept(Q, E)[1], e)
    B = torch.empty_like(X)
    cbm.cbm_checkpoint_restore(Q, E, B)
    assert bool(B.isfinite().all()) and torch.equal(torch.sign(B), torch.sign(X))
    H, _ = _matrix(torch, np.full((1, 5), 65504.0), "f16", 0)
    Q, E, _, _ = _room(torch, 1, 5, 0)
    cbm.cbm_checkpoint_save(H, Q, E)
    cbm.cbm_checkpoint_restore(Q, E, H)
    assert bool(H.isfinite().all()) and bool((H == 127 * 512).all())


@pytest.mark.parametrize("name", ["f32", "bf16", "f16"])
def test_values_that_are_not_finite_take_their_block_only(env, name):  # noqa: F811
    torch, cbm = env
    X, _ = _matrix(torch, np.random.default_rng(0).standard_normal((6, 100)), name, 0)
    X[0, 0], X[1, 99], X[2, 40] = math.nan, math.inf, -math.inf
    Q, E, _, _ = _room(torch, 6, 100, 0)
    cbm.cbm_checkpoint_save(X, Q, E)
    q, e = orc.keep(_numbers(X))
    assert np.array_equal(_kept(Q, E)[0], q) and np.array_equal(_kept(Q, E)[1], e)
    B, G = torch.empty_like(X), torch.empty_like(X)
    cbm.cbm_checkpoint_restore(Q, E, B)
    cbm.cbm_checkpoint_relu_backward(Q, E, torch.ones_like(X), G)
    bad = torch.zeros((6, 100), dtype=torch.bool, device="cuda")
    bad[0, :32] = bad[1, 96:] = bad[2, 32:64] = True
    assert torch.equal(B.isnan(), bad) and torch.equal(G.isnan(), bad)
    dW, ws = torch.empty((100, 3), device="cuda"), torch.empty(cbm.cbm_checkpoint_workspace_bytes(6, 100, 3), dtype=torch.uint8, device="cuda")
    cbm.cbm_checkpoint_weight_grad(Q, E, torch.ones((6, 3), device="cuda"), dW, ws)
    assert torch.equal(dW.isnan().any(dim=1), bad.any(dim=0))


def _grad(torch, cbm, Q, E, dY, c, pad=0):
    k = Q.shape[1]
    whole = torch.full((k, c + pad), math.nan, device="cuda")
    ws = torch.full((cbm.cbm_checkpoint_workspace_bytes(Q.shape[0], k, c),), 255, dtype=torch.uint8, device="cuda")
    cbm.cbm_checkpoint_weight_grad(Q, E, dY, whole[:, :c], ws)
    assert bool(whole[:, c:].isnan().all()), "wrote outside the columns"
    return _numbers(whole[:, :c])


# both operands on both sides of their tiles (128 and 64 columns, 16 rows), of what a wave and a workgroup take, and of the byte-wise loads
@pytest.mark.parametrize("name", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("k", [1, 2, 3, 4, 5, 31, 32, 33, 47, 64, 68, 100, 127, 128, 129, 132, 256, 300, 1000])
def test_weight_gradient_of_whole_numbers_is_exact(env, name, k):  # noqa: F811
    torch, cbm = env
    rng = np.random.default_rng(k)
    for c in (1, 2, 3, 16, 32, 33, 47, 63, 64, 65, 66, 128, 130, 200):
        for n, pad in ((1, 0), (15, 1), (17, 3), (64, 0), (65, 4), (333, 0)) + (((5001, 1), (40000, 0)) if c in (2, 47, 64) and k in (4, 47, 100, 128, 300) else ()):
            q, e = rng.integers(-9, 10, (n, k)), rng.integers(-1, 2, (n, -(-k // 32)))  # products are multiples of 1/2, sums below 2^23
            Q, E, wq, we = _room(torch, n, k, pad)
            Q.copy_(torch.from_numpy(q))
            E.copy_(torch.from_numpy(e + 127))
            dY, _ = _matrix(torch, rng.integers(-8, 9, (n, c)).astype(np.float64), name, pad)
            assert np.array_equal(_grad(torch, cbm, Q, E, dY, c, pad), orc.weight_grad(q, e, _numbers(dY))), (n, c, pad)


@pytest.mark.parametrize("name", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,k,c", [(1, 64, 16), (200, 100, 47), (5000, 128, 64), (30000, 36, 130)])
def test_weight_gradient_within_the_bound(env, name, n, k, c):  # noqa: F811
    """Exact products of parts; a sum takes at most three parts x n additions of fp32, of which a wave has n / shares, a few waves and shares the rest: 3 n / 64 + 100
    roundings of a partial sum, each at most 2^-24 of the sum of sizes (and twice that: the cores need not round to nearest)."""
    torch, cbm = env
    rng = np.random.default_rng(n)
    q, e = rng.integers(-127, 128, (n, k)), rng.integers(-12, 3, (n, -(-k // 32)))
    Q, E, _, _ = _room(torch, n, k, 0)
    Q.copy_(torch.from_numpy(q))
    E.copy_(torch.from_numpy(e + 127))
    dY, _ = _matrix(torch, rng.standard_normal((n, c)) * np.exp2(rng.integers(-8, 1, (n, 1))), name, 0)
    dy = _numbers(dY)
    ref, size = orc.weight_grad(q, e, dy), np.abs(orc.kept_values(q, e)).T @ np.abs(dy)
    got = _grad(torch, cbm, Q, E, dY, c)
    assert np.all(np.abs(got - ref) <= 2 * (3 * n / 64 + 100) * U * size)
    assert np.linalg.norm(got - ref) <= 1e-6 * np.linalg.norm(ref)
    assert np.array_equal(got, _grad(torch, cbm, Q, E, dY, c)), "the same call gave other bits"


@pytest.mark.parametrize("name", ["f32", "bf16", "f16"])
def test_weight_gradient_keeps_infinities_and_large_values(env, name):  # noqa: F811
    torch, cbm = env
    rng = np.random.default_rng(7)
    n, k, c = 100, 40, 6
    q, e = rng.integers(-100, 101, (n, k)), np.full((n, 2), -20)
    q[50] = np.where(q[50] == 0, 1, q[50])
    q[50, 3] = 0
    Q, E, _, _ = _room(torch, n, k, 0)
    Q.copy_(torch.from_numpy(q))
    E.copy_(torch.from_numpy(e + 127))
    dY, _ = _matrix(torch, rng.standard_normal((n, c)), name, 0)
    dY[50, 0], dY[50, 1], dY[20, 2] = math.inf, -math.inf, math.nan
    dY[10, 3] = torch.finfo(dY.dtype).max
    got, ref = _grad(torch, cbm, Q, E, dY, c), orc.weight_grad(q, e, _numbers(dY))
    assert np.array_equal(np.isnan(got), np.isnan(ref)) and np.array_equal(np.isposinf(got), np.isposinf(ref)) and np.array_equal(np.isneginf(got), np.isneginf(ref))
    assert np.isinf(ref[:, 0]).sum() == k - 1 and np.isnan(ref[3, 0]) and np.isnan(ref[:, 2]).all()
    fine = np.isfinite(ref)
    size = np.abs(orc.kept_values(q, e)).T @ np.where(np.isfinite(_numbers(dY)), np.abs(_numbers(dY)), 0.0)
    assert np.all(np.abs(got - ref)[fine] <= 300 * U * size[fine])


def test_no_rows_and_offsets_beyond_32_bits(env):  # noqa: F811
    torch, cbm = env
    Q, E, _, _ = _room(torch, 0, 40, 0)
    X = torch.empty((0, 40), device="cuda")
    cbm.cbm_checkpoint_save(X, Q, E)
    cbm.cbm_checkpoint_restore(Q, E, X)
    cbm.cbm_checkpoint_relu_backward(Q, E, X, X)
    assert not _grad(torch, cbm, Q, E, torch.empty((0, 3), device="cuda"), 3).any()
    n, k, last = 1 << 21, 1056, 200
    X = torch.zeros((n, k), dtype=torch.float16, device="cuda")
    X[-last:] = torch.randn((last, k), device="cuda")
    Q, E, _, _ = _room(torch, n, k, 0)
    small_q, small_e, _, _ = _room(torch, last, k, 0)
    cbm.cbm_checkpoint_save(X, Q, E)
    cbm.cbm_checkpoint_save(X[-last:].clone(), small_q, small_e)
    assert torch.equal(Q[-last:], small_q) and torch.equal(E[-last:], small_e)
    B, G = torch.empty_like(X), torch.empty_like(X)
    cbm.cbm_checkpoint_restore(Q, E, B)
    cbm.cbm_checkpoint_relu_backward(Q, E, X, G)
    b, g = torch.empty_like(X[-last:]), torch.empty_like(X[-last:])
    cbm.cbm_checkpoint_restore(small_q, small_e, b)
    cbm.cbm_checkpoint_relu_backward(small_q, small_e, X[-last:].clone(), g)
    assert torch.equal(B[-last:], b) and torch.equal(G[-last:], g)
    dY = torch.randint(-4, 5, (n, 2), device="cuda").float()
    Q[-last:] = torch.randint(-5, 6, (last, k), device="cuda")
    E.fill_(127)
    assert np.array_equal(_grad(torch, cbm, Q, E, dY, 2), _numbers(Q[-last:].float()).T @ _numbers(dY[-last:]))


def test_graph_capture_replays(env):  # noqa: F811
    torch, cbm = env
    n, k, c = 3000, 100, 47
    X, dY = torch.randn((n, k), device="cuda"), torch.randn((n, c), device="cuda")
    Q, E, _, _ = _room(torch, n, k, 0)
    B, dW = torch.empty_like(X), torch.empty((k, c), device="cuda")
    ws = torch.empty(cbm.cbm_checkpoint_workspace_bytes(n, k, c), dtype=torch.uint8, device="cuda")

    def step():
        cbm.cbm_checkpoint_save(X, Q, E)
        cbm.cbm_checkpoint_restore(Q, E, B)
        cbm.cbm_checkpoint_weight_grad(Q, E, dY, dW, ws)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in range(3):
        X.copy_(torch.randn((n, k), device="cuda") + seed)
        graph.replay()
        torch.cuda.synchronize()
        got = [B.clone(), dW.clone()]
        B.fill_(math.nan)
        dW.fill_(math.nan)
        step()
        torch.cuda.synchronize()
        assert torch.equal(got[0], B) and torch.equal(got[1], dW)


def test_refusals(env):  # noqa: F811
    torch, cbm = env
    X, Y = torch.zeros((4, 40), device="cuda"), torch.zeros((4, 40), device="cuda")
    Q, E, _, _ = _room(torch, 4, 40, 0)
    dW = torch.zeros((40, 8), device="cuda")
    dY = torch.zeros((100, 8), device="cuda")
    Q2, E2, _, _ = _room(torch, 100, 40, 0)
    ws = torch.zeros(cbm.cbm_checkpoint_workspace_bytes(100, 40, 8), dtype=torch.uint8, device="cuda")
    assert ws.numel() > 0
    for bad in (lambda: cbm.cbm_checkpoint_save(X.cpu(), Q, E), lambda: cbm.cbm_checkpoint_save(X.double(), Q, E), lambda: cbm.cbm_checkpoint_save(X, Q.int(), E),
                lambda: cbm.cbm_checkpoint_save(X, Q, E.char()), lambda: cbm.cbm_checkpoint_save(X, Q, E[:, :1]), lambda: cbm.cbm_checkpoint_save(X[:, :39], Q, E),
                lambda: cbm.cbm_checkpoint_restore(Q, E, X[:2]), lambda: cbm.cbm_checkpoint_relu_backward(Q, E, X, Y.half()), lambda: cbm.cbm_checkpoint_relu_backward(Q, E, X[:, :8], Y[:, :8]),
                lambda: cbm.cbm_checkpoint_weight_grad(Q2, E2, dY[:50], dW, ws), lambda: cbm.cbm_checkpoint_weight_grad(Q2, E2, dY, dW[:, :4], ws),
                lambda: cbm.cbm_checkpoint_weight_grad(Q2, E2, dY, dW.half(), ws)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: cbm.cbm_checkpoint_weight_grad(Q2, E2, dY, dW, None), lambda: cbm.cbm_checkpoint_weight_grad(Q2, E2, dY, dW, ws[:-1]),
                lambda: cbm.cbm_checkpoint_weight_grad(Q2, E2, dY, dY[:40], ws), lambda: cbm.cbm_checkpoint_weight_grad(Q2, E2, dY, dW, ws[1:]),
                lambda: cbm.cbm_checkpoint_save(X, X.view(torch.int8)[:, :40], E), lambda: cbm.cbm_checkpoint_restore(X.view(torch.int8)[:, :40], E, X),
                lambda: cbm.cbm_checkpoint_relu_backward(Q, E, Y[:, :40], Y.as_strided((4, 40), (30, 1)))):
        with pytest.raises(cbm.CbmError) as e:
            bad()
        assert e.value.status == 1
    from paper_2409_02208_amd import binding

    lib, p, q, s = binding._lib(), X.data_ptr(), Q.data_ptr(), E.data_ptr()
    call = lambda n, k, t, ldx, ldq, lde, x=p: lib.cbm_checkpoint_save(n, k, t, x, ldx, q, ldq, s, lde, None)  # noqa: E731
    assert [call(4, 40, 7, 40, 40, 2), call(-1, 40, 0, 40, 40, 2), call(4, 0, 0, 40, 40, 2), call(4, 40, 0, 39, 40, 2), call(4, 40, 0, 40, 39, 2), call(4, 40, 0, 40, 40, 1),
            call(4, 40, 0, 40, 40, 2, None), call(4, 40, 0, 40, 40, 2, p + 2)] == [1] * 8
    assert call(4, (1 << 24) + 1, 0, 1 << 25, 1 << 25, 1 << 25) == 5
    assert lib.cbm_checkpoint_weight_grad(4, 1 << 20, 1 << 20, q, 1 << 20, s, 1 << 20, 0, p, 1 << 20, p, 1 << 20, None, 0, None) == 5
    assert not bool(X.any()) and not bool(dW.any())
