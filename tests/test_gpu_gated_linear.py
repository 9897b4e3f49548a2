"""The gated layer, forward and backward, through the C ABI against the definition in 64 bits: sizes around every tile and chunk, types, strides, empty and single rows, values that are
not finite, refusals."""
import math

import numpy as np
import pytest

from oracle import train_oracle as orc
from test_gpu_layer_norm import ROUNDING, _matrix, _numbers, _type, _untouched, env  # noqa: F401

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TYPES = ["f32", "bf16", "f16"]
LEAST = {"f32": 2.0 ** -126, "bf16": 2.0 ** -126, "f16": 2.0 ** -25}  # what rounding to the type may lose beside its relative part
# Sums of k exact products (fp32: six products of parts; what is left out is 2^-24 of a term) in fp32: k additions at most on the way of a term, a few shares joined.
SUM = lambda k: (k + 16) * U  # noqa: E731

SIZES = [(1, 1, 1), (2, 3, 2), (5, 7, 3), (3, 8, 4), (31, 9, 5), (33, 31, 7), (32, 32, 8), (127, 33, 9), (128, 63, 31), (129, 64, 32), (65, 65, 33), (64, 100, 47), (1, 128, 64),
         (7, 130, 65), (300, 129, 100), (16, 500, 130), (1, 1000, 333), (257, 40, 257), (1000, 24, 12), (2, 2049, 66)]


def _rounded(value, bound, name):
    return bound + ROUNDING[name] * (np.abs(value) + bound) + LEAST[name]


def _function(name, g):
    """Of the activation and of its slope, relative to |g| + 1: exp's argument is off by |g| 2^-24 of it, erfc's by g^2 2^-23, a few operations each."""
    return (np.abs(g) + (np.minimum(g * g, 64.0) if name == "gelu" else 0.0) + 16) * U * 2


def _near(got, want, bound):
    got = _numbers(got)
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), (np.argwhere(bad)[:4].tolist(), got[bad][:4], want[bad][:4], bound[bad][:4])


def _forward(torch, cbm, n, k, m, name, act, pad, offset, keep=True, scale=1.0):
    rng = np.random.default_rng(n + 7 * k + 31 * m)
    X, _ = _matrix(torch, scale * rng.standard_normal((n, k)), name, pad, offset)
    Wg, Wu = (_matrix(torch, rng.standard_normal((k, m)) / math.sqrt(k), name, pad, offset)[0] for _ in range(2))
    outs = [_matrix(torch, np.zeros((n, m)), name, pad, offset) for _ in range(3)]
    ws = torch.full((cbm.cbm_gated_linear_workspace_bytes(n, k, m, _type(torch, name)),), 255, dtype=torch.uint8, device="cuda")
    H, G, U_ = (t for t, _ in outs)
    cbm.cbm_gated_linear(X, Wg, Wu, H, *((G, U_) if keep else (None, None)), activation=act, workspace=ws)
    for t, whole in outs:
        if t.numel():
            _untouched(torch, t, whole, offset)
    return X, Wg, Wu, H, G, U_


def _check_forward(X, Wg, Wu, H, G, U_, name, act, keep=True):
    x, wg, wu = (_numbers(t) for t in (X, Wg, Wu))
    h, g, u = orc.gated_linear(x, wg, wu, act)
    of_g, of_u = (SUM(x.shape[1]) * (np.abs(x) @ np.abs(w)) for w in (wg, wu))
    value = np.abs(orc.activation(act, g)[0])
    of_value = 1.13 * of_g + _function(act, g) * (np.abs(g) + 1)  # (no slope is above 1.13)
    _near(H, h, _rounded(h, of_value * (np.abs(u) + of_u) + value * of_u, name))
    if keep:
        _near(G, g, _rounded(g, of_g, name))
        _near(U_, u, _rounded(u, of_u, name))


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("n,k,m", SIZES)
def test_forward(env, name, n, k, m):  # noqa: F811
    torch, cbm = env
    for i, (pad, offset) in enumerate(((0, 0), (3, 1), (8, 8))):
        act = ("silu", "gelu", "relu")[(i + n + k) % 3]
        _check_forward(*_forward(torch, cbm, n, k, m, name, act, pad, offset, keep=i != 1), name, act, keep=i != 1)


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("act", ["silu", "gelu", "relu"])
def test_activations_far_from_zero(env, name, act):  # noqa: F811
    torch, cbm = env
    _check_forward(*_forward(torch, cbm, 50, 16, 40, name, act, 0, 0, scale=12.0), name, act)


def _backward(torch, cbm, n, k, m, name, act, pad, offset, size=1.0, outputs=(True, True, True)):
    rng = np.random.default_rng(3 * n + 5 * k + m)
    X, _ = _matrix(torch, rng.standard_normal((n, k)), name, pad, offset)
    Wg, Wu = (_matrix(torch, rng.standard_normal((k, m)) / math.sqrt(k), name, pad, offset)[0] for _ in range(2))
    G, U_ = (_matrix(torch, 2 * rng.standard_normal((n, m)), name, pad, offset)[0] for _ in range(2))
    dH, _ = _matrix(torch, size * rng.standard_normal((n, m)), name, pad, offset)
    outs = [_matrix(torch, np.zeros(s), name, pad, offset) for s in ((n, k), (k, m), (k, m))]
    ws = torch.full((cbm.cbm_gated_linear_backward_workspace_bytes(n, k, m, _type(torch, name)),), 255, dtype=torch.uint8, device="cuda")
    cbm.cbm_gated_linear_backward(dH, X, Wg, Wu, G, U_, *(t if on else None for (t, _), on in zip(outs, outputs)), activation=act, workspace=ws)
    for t, whole in outs:
        if t.numel():
            _untouched(torch, t, whole, offset)
    return (dH, X, Wg, Wu, G, U_), [t for t, _ in outs]


def _check_backward(args, outs, name, act, outputs=(True, True, True)):
    dh, x, wg, wu, g, u = (_numbers(t) for t in args)
    dx, dwg, dwu, dg, du = orc.gated_linear_backward(dh, x, wg, wu, g, u, act)
    of = _function(act, g) * (np.abs(g) + 1)
    of_du, of_dg = (_rounded(v, b, name) for v, b in ((du, np.abs(dh) * of + 2 * U * np.abs(du)), (dg, np.abs(dh * u) * of + 3 * U * np.abs(dg))))
    for on, got, want, terms in zip(outputs, outs, (dx, dwg, dwu), (((dg, of_dg, wg.T), (du, of_du, wu.T)), ((x.T, None, dg, of_dg),), ((x.T, None, du, of_du),))):
        if not on:
            assert not bool(got.any())
            continue
        bound = 0.0
        for t in terms:
            if len(t) == 3:
                bound = bound + SUM(2 * t[0].shape[1] + 128) * ((np.abs(t[0]) + t[1]) @ np.abs(t[2])) + t[1] @ np.abs(t[2])
            else:
                bound = bound + SUM(t[0].shape[1]) * (np.abs(t[0]) @ (np.abs(t[2]) + t[3])) + np.abs(t[0]) @ t[3]
        _near(got, want, _rounded(want, bound, name))


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("n,k,m", SIZES + [(3000, 20, 24), (5000, 65, 7)])
def test_backward(env, name, n, k, m):  # noqa: F811
    torch, cbm = env
    for i, (pad, offset) in enumerate(((0, 0), (5, 1), (8, 8))):
        act = ("silu", "gelu", "relu")[(i + n + k) % 3]
        on = ((True, True, True), (True, False, True), (False, True, False))[i] if n % 2 else (True, True, True)
        _check_backward(*_backward(torch, cbm, n, k, m, name, act, pad, offset, outputs=on), name, act, on)


MANY_ROWS = [(40001, 31, 8), (20003, 65, 47), (9001, 17, 300), (5001, 63, 130), (33, 40, 8200)]  # tiles through LDS, where the rest above is small


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("n,k,m", MANY_ROWS)
def test_many_rows_or_columns(env, name, n, k, m):  # noqa: F811
    torch, cbm = env
    for i, (pad, offset) in enumerate(((0, 0), (3, 1), (8, 8))):
        act = ("silu", "gelu", "relu")[(i + n + k) % 3]
        _check_forward(*_forward(torch, cbm, n, k, m, name, act, pad, offset, keep=i != 1), name, act, keep=i != 1)
        on = ((True, True, True), (True, False, True), (False, True, False))[i]
        _check_backward(*_backward(torch, cbm, n, k, m, name, act, pad, offset, outputs=on), name, act, on)


def test_small_gradients_in_fp16_are_not_lost(env):  # noqa: F811
    """Gradients below fp16's smallest normal value, 2^-14: rounded to multiples of 2^-24, and counted."""
    torch, cbm = env
    _check_backward(*_backward(torch, cbm, 200, 40, 30, "f16", "silu", 0, 0, size=2e-5), "f16", "silu")


@pytest.mark.parametrize("act", ["silu", "gelu", "relu"])
def test_backward_against_differences(env, act):  # noqa: F811
    """The gradients of sum(H o R) by central differences of the 64-bit forward pass."""
    torch, cbm = env
    args, outs = _backward(torch, cbm, 6, 5, 7, "f32", act, 0, 0)
    dh, x, wg, wu = (_numbers(t) for t in args[:4])
    _, g, u = orc.gated_linear(x, wg, wu, act)
    for t, v in zip(args[4:], (g, u)):
        t.copy_(torch.from_numpy(v))
    cbm.cbm_gated_linear_backward(*args, *outs, activation=act, workspace=torch.empty(cbm.cbm_gated_linear_backward_workspace_bytes(6, 5, 7, torch.float32), dtype=torch.uint8, device="cuda"))
    loss = lambda *p: (orc.gated_linear(*p, act)[0] * dh).sum()  # noqa: E731
    step = 1e-5
    for i, got in enumerate(outs):
        want = np.zeros(got.shape)
        for at in np.ndindex(*got.shape):
            both = []
            for s in (step, -step):
                p = [x.copy(), wg.copy(), wu.copy()]
                p[i][at] += s
                both.append(loss(*p))
            want[at] = (both[0] - both[1]) / (2 * step)
        # differences are off by step^2 of third derivatives of size 10, roundings by 2^-53 / step of losses of size 100
        assert np.abs(_numbers(got) - want).max() <= 1e-5 * max(1.0, np.abs(want).max())


@pytest.mark.parametrize("name", TYPES)
def test_no_rows(env, name):  # noqa: F811
    torch, cbm = env
    args, outs = _backward(torch, cbm, 0, 12, 9, name, "silu", 0, 0)
    assert not any(bool(t.any()) for t in outs)
    for t in outs[1:]:
        t.fill_(3)
    cbm.cbm_gated_linear_backward(*args, None, *outs[1:], workspace=torch.empty(cbm.cbm_gated_linear_backward_workspace_bytes(0, 12, 9, _type(torch, name)), dtype=torch.uint8, device="cuda"))
    assert not any(bool(t.any()) for t in outs[1:])
    _forward(torch, cbm, 0, 12, 9, name, "silu", 0, 0)


@pytest.mark.parametrize("name", TYPES)
def test_values_that_are_not_finite_stay_in_their_rows(env, name):  # noqa: F811
    torch, cbm = env
    rng = np.random.default_rng(1)
    x = rng.standard_normal((140, 70))
    X, _ = _matrix(torch, x, name, 0)
    Wg, Wu = (_matrix(torch, rng.standard_normal((70, 90)), name, 0)[0] for _ in range(2))
    H, G, U_ = (torch.zeros((140, 90), dtype=X.dtype, device="cuda") for _ in range(3))
    cbm.cbm_gated_linear(X, Wg, Wu, H, G, U_)
    X[3, 5], X[130, 69], X[131, 0] = math.nan, math.inf, -math.inf
    odd = [t.clone() for t in (H, G, U_)]
    cbm.cbm_gated_linear(X, Wg, Wu, *odd)
    rows = torch.ones(140, dtype=torch.bool, device="cuda")
    rows[[3, 130, 131]] = False
    for before, after in zip((H, G, U_), odd):
        assert torch.equal(before[rows], after[rows])
    for after in odd[1:]:
        assert not bool(after[~rows].isfinite().any())
    assert bool(odd[0][3].isnan().all())


def test_captured_and_on_streams(env):  # noqa: F811
    torch, cbm = env
    n, k, m = 700, 65, 80
    g = torch.Generator(device="cuda").manual_seed(0)
    new = lambda *s: torch.randn(s, device="cuda", generator=g).bfloat16()  # noqa: E731
    X, Wg, Wu, dH = new(n, k), new(k, m), new(k, m), new(n, m)
    outs = [new(n, m), new(n, m), new(n, m), new(n, k), new(k, m), new(k, m)]
    need = max(cbm.cbm_gated_linear_workspace_bytes(n, k, m, torch.bfloat16), cbm.cbm_gated_linear_backward_workspace_bytes(n, k, m, torch.bfloat16))
    ws = [torch.empty(need, dtype=torch.uint8, device="cuda") for _ in range(3)]

    def step(outs, ws, stream=None):
        cbm.cbm_gated_linear(X, Wg, Wu, *outs[:3], activation="gelu", workspace=ws, stream=stream)
        cbm.cbm_gated_linear_backward(dH, X, Wg, Wu, outs[1], outs[2], *outs[3:], activation="gelu", workspace=ws, stream=stream)

    step(outs, ws[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(outs, ws[0])
    streams = [torch.cuda.Stream() for _ in range(2)]
    for seed in range(3):
        X.copy_(torch.randn((n, k), device="cuda") * (seed + 1))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outs]
        apart = [[torch.full_like(t, 7) for t in outs] for _ in range(2)]
        torch.cuda.synchronize()
        for s, o, w in zip(streams, apart, ws[1:]):  # two calls at once, a workspace each
            step(o, w, s)
        torch.cuda.synchronize()
        for o in apart:
            assert all(torch.equal(a, b) for a, b in zip(got, o))


def test_refusals(env):  # noqa: F811
    torch, cbm = env
    X, Wg, Wu, H = torch.zeros((4, 6), device="cuda"), torch.zeros((6, 5), device="cuda"), torch.zeros((6, 5), device="cuda"), torch.ones((4, 5), device="cuda")
    for bad in (lambda: cbm.cbm_gated_linear(X.cpu(), Wg, Wu, H), lambda: cbm.cbm_gated_linear(X, Wg, Wu[:, :4], H), lambda: cbm.cbm_gated_linear(X, Wg[:5], Wu[:5], H),
                lambda: cbm.cbm_gated_linear(X, Wg, Wu, H[:3]), lambda: cbm.cbm_gated_linear(X, Wg, Wu, H.half()), lambda: cbm.cbm_gated_linear(X, Wg.half(), Wu.half(), H),
                lambda: cbm.cbm_gated_linear(X, Wg, Wu, H, H[:, :4]), lambda: cbm.cbm_gated_linear(X, Wg, Wu, H, activation="tanh"), lambda: cbm.cbm_gated_linear(X, Wg, Wu, H, activation=[]),
                lambda: cbm.cbm_gated_linear(X.t(), Wg, Wu, H)):
        with pytest.raises(ValueError):
            bad()
    dX, dWg, dWu = torch.ones_like(X), torch.ones_like(Wg), torch.ones_like(Wu)
    ws = torch.zeros(cbm.cbm_gated_linear_backward_workspace_bytes(4, 6, 5, torch.float32), dtype=torch.uint8, device="cuda")
    G, U_, dH = (torch.zeros_like(H) for _ in range(3))
    for bad in (lambda: cbm.cbm_gated_linear(X, Wg, Wu, H, H), lambda: cbm.cbm_gated_linear(X, X[:, :5].new_zeros((6, 5)), Wu, Wu[:4]),
                lambda: cbm.cbm_gated_linear_backward(dH, X, Wg, Wu, G, U_, None, None, None, workspace=ws), lambda: cbm.cbm_gated_linear_backward(dH, X, Wg, Wu, G, U_, dX, dWg, dWu),
                lambda: cbm.cbm_gated_linear_backward(dH, X, Wg, Wu, G, U_, dX, dWg, dWg, workspace=ws), lambda: cbm.cbm_gated_linear_backward(dH, X, Wg, Wu, G, U_, dX, dWg, dWu, workspace=ws[:-1]),
                lambda: cbm.cbm_gated_linear_backward(dH, X, Wg, Wu, G, U_, X, dWg, dWu, workspace=ws)):
        with pytest.raises(cbm.CbmError) as e:
            bad()
        assert e.value.status == 1
    from paper_2409_02208_amd import binding

    lib = binding._lib()
    x, w, h = X.data_ptr(), Wg.data_ptr(), H.data_ptr()
    call = lambda n=4, k=6, m=5, t=0, a=0, ldx=6, ldw=5, p=x: lib.cbm_gated_linear(n, k, m, t, a, p, ldx, w, ldw, Wu.data_ptr(), 5, h, 5, None, 5, None, 5, None, 0, None)  # noqa: E731
    assert [call(n=-1), call(k=0), call(m=0), call(t=3), call(a=3), call(a=-1), call(ldx=5), call(ldw=4), call(p=None), call(p=x + 2)] == [1] * 10
    assert [call(k=(1 << 24) + 1, ldx=1 << 25), call(n=(1 << 31) + 1)] == [5, 5]
    torch.cuda.synchronize()
    assert bool((H == 1).all()) and bool((dX == 1).all())


# rows that are whole numbers of 16 bytes, which 16-bit types go through LDS as they are: tiles of 128 and 256 with all and with few of their rows and columns, K that ends inside a chunk of 64
UNITS = [(1, 8, 8), (130, 72, 72), (300, 64, 264), (257, 200, 136), (1100, 136, 520), (4100, 72, 2056), (2304, 320, 2048)]


@pytest.mark.parametrize("name", ["bf16", "f16"])
@pytest.mark.parametrize("n,k,m", UNITS)
def test_whole_units(env, name, n, k, m):  # noqa: F811
    torch, cbm = env
    for pad in (0, 8):
        act = "silu" if pad else "gelu"
        _check_forward(*_forward(torch, cbm, n, k, m, name, act, pad, 0, keep=pad == 0), name, act, keep=pad == 0)
        _check_backward(*_backward(torch, cbm, n, k, m, name, act, pad, 0), name, act)


@pytest.mark.parametrize("n,k,m", [(8, 2048, 8), (20000, 64, 72), (9000, 520, 24)])
def test_backward_with_shares_of_k(env, n, k, m):  # noqa: F811
    torch, cbm = env
    for name in ("f32", "bf16"):
        _check_backward(*_backward(torch, cbm, n, k, m, name, "silu", 0, 0), name, "silu")


def _gpu(torch, n, k, name, pad, offset, scale=1.0):
    t, whole = _matrix(torch, np.zeros((0, k)), name, 0)
    whole = torch.full((offset + n * (k + pad),), math.nan, dtype=_type(torch, name), device="cuda")
    t = whole[offset:].view(n, k + pad)[:, :k]
    t.copy_(torch.randn((n, k), device="cuda") * scale)
    return t


def _within(got, want, bound, name):
    bound = bound + ROUNDING[name] * (want.abs() + bound) + LEAST[name]
    assert bool(((got.double() - want).abs() <= bound).all())


@pytest.mark.parametrize("name", ["bf16", "f16"])
@pytest.mark.parametrize("pad,offset", [(0, 0), (1, 1), (8, 0)])
@pytest.mark.parametrize("n,k,m", [(12001, 515, 4099), (4097, 512, 12288), (1025, 1000, 25000)])
def test_large_products(env, name, n, k, m, pad, offset):  # noqa: F811
    """Matrices of odd widths, strides and addresses are copied into rows of whole units, and the weights of many rows turned.  Against 64 bits on the GPU."""
    torch, cbm = env
    torch.manual_seed(n)
    X, Wg, Wu = _gpu(torch, n, k, name, pad, offset), _gpu(torch, k, m, name, pad, offset, k ** -0.5), _gpu(torch, k, m, name, pad, offset, k ** -0.5)
    H, G, U_, dX, dWg, dWu = (_gpu(torch, *s, name, pad, offset) for s in ((n, m), (n, m), (n, m), (n, k), (k, m), (k, m)))
    need = max(cbm.cbm_gated_linear_workspace_bytes(n, k, m, X.dtype), cbm.cbm_gated_linear_backward_workspace_bytes(n, k, m, X.dtype))
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    cbm.cbm_gated_linear(X, Wg, Wu, H, G, U_, activation="relu", workspace=ws)
    x, wg, wu = X.double(), Wg.double(), Wu.double()
    g, u = x @ wg, x @ wu
    of_g, of_u = SUM(k) * (x.abs() @ wg.abs()), SUM(k) * (x.abs() @ wu.abs())
    _within(G, g, of_g, name)
    _within(U_, u, of_u, name)
    _within(H, g.clamp_min(0) * u, of_g * (u.abs() + of_u) + g.abs() * of_u, name)
    del g, u, of_g, of_u
    dH = _gpu(torch, n, m, name, pad, offset)
    cbm.cbm_gated_linear_backward(dH, X, Wg, Wu, G, U_, dX, dWg, dWu, activation="relu", workspace=ws)
    dh, g, u = dH.double(), G.double(), U_.double()
    du, dg = dh * g.clamp_min(0), dh * u * (g > 0)
    del dh, g, u
    half = 1.01 * ROUNDING[name]  # of dG and dU, and fp16's smallest values
    t = lambda a: a.t().contiguous()  # noqa: E731
    for got, want, terms in ((dX, dg @ t(wg) + du @ t(wu), dg.abs() @ t(wg.abs()) + du.abs() @ t(wu.abs())), (dWg, t(x) @ dg, t(x.abs()) @ dg.abs()), (dWu, t(x) @ du, t(x.abs()) @ du.abs())):
        # (fp16's smallest dG and dU: 2^-25 each, of at most 40,000 terms of size below 6)
        _within(got, want, (half + SUM(max(n, 2 * m))) * terms + (0.01 if name == "f16" else 0.0), name)
