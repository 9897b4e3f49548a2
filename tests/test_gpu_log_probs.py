"""Log probabilities, entropy, top alternatives and their gradient through the C ABI against the definition in 64 bits: every width at which a kernel's shape changes, one
row to many, ties, masks that leave little or nothing, values that are not finite, refusals."""
import math

import numpy as np
import pytest

from oracle import train_oracle as orc
from test_gpu_layer_norm import ROUNDING, _matrix, _numbers, _type, _untouched, env  # noqa: F401

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
WIDTHS = [1, 2, 3, 4, 5, 7, 8, 9, 16, 17, 31, 32, 33, 47, 63, 64, 65, 127, 128, 129, 255, 256, 257, 511, 512, 513, 1000, 1023, 1024, 1025, 2047, 2048, 2049, 2056, 4100, 8192, 8193, 20000,
          50001, 131073, 300007]


def _scores(torch, cbm, Z, labels, top, label_type=None):
    n, c = Z.shape
    nan = lambda *shape: torch.full(shape, math.nan, device="cuda")  # noqa: E731
    L = torch.from_numpy(np.asarray(labels)).to(label_type or torch.int64).cuda()
    logp, entropy, stats, values = nan(n), nan(n), nan(n, 2), nan(n, top)
    columns = torch.full((n, top), -7, dtype=torch.int32, device="cuda")
    ws = torch.full((cbm.cbm_log_probs_workspace_bytes(n, c, top),), 255, dtype=torch.uint8, device="cuda")
    cbm.cbm_log_probs(Z, L, logp, entropy, stats, values if top else None, columns if top else None, ws)
    return L, logp, entropy, stats, values, columns


def _bounds(z, ref):
    """Of l, log p at a score z_j, and H.  e = exp(z - m) is off by (3 |d| + 2) 2^-24 of itself (its argument's two roundings, the hardware's unit in the last place), as much
    again where a larger maximum was met later; 150 additions on the way into a row's sum, 40 more (32 in a lane, a rescaling) for each 8,192 columns."""
    logp, entropy, stats, _, _ = ref
    m, l = stats[:, 0], stats[:, 1]  # noqa: E741
    with np.errstate(invalid="ignore"):
        d = np.where(z > -np.inf, z - m[:, None], 0.0)
        p = np.where(z > -np.inf, np.exp(d - l[:, None]), 0.0)
    first, second = (np.abs(d) * p).sum(axis=1), (d * d * p).sum(axis=1)
    depth = 150 + 40 * z.shape[1] / 8192
    of_sum = U * (6 * first + depth)
    of_l = of_sum + 3 * U * np.abs(l) + U
    of_entropy = of_l + first * of_sum + U * (6 * second + (depth + 10) * first) + 2 * U * (np.abs(l) + np.abs(entropy))
    of_log = lambda away: of_l + 3 * U * (np.abs(away) + np.abs(l))  # noqa: E731
    return of_l, of_entropy, of_log


def _check(torch, Z, labels, got, top):
    _, logp, entropy, stats, values, columns = got
    z = _numbers(Z)
    ref = orc.log_probs(z, labels, top)
    of_l, of_entropy, of_log = _bounds(z, ref)
    fine = np.isfinite(ref[2][:, 0])

    def near(a, b, bound):
        a = _numbers(a)
        same = (a == b) | (np.isnan(a) & np.isnan(b))
        with np.errstate(invalid="ignore"):
            assert np.all(same | (np.isfinite(b) & (np.abs(a - b) <= bound))), np.argwhere(~(same | (np.abs(a - b) <= bound)))[:5]

    assert np.array_equal(_numbers(stats)[:, 0], ref[2][:, 0], equal_nan=True)
    near(stats[:, 1], ref[2][:, 1], of_l)
    near(entropy, ref[1], of_entropy)
    away = np.where(fine, ref[0] + np.where(fine, ref[2][:, 1], 0.0), 0.0)
    with np.errstate(invalid="ignore"):
        near(logp, ref[0], of_log(np.where(np.isfinite(away), away, 0.0)))
        if top:
            assert np.array_equal(columns.cpu().numpy(), ref[4])
            near(values, ref[3], (of_l[:, None] + 3 * U * (np.abs(np.where(np.isfinite(ref[3]), ref[3], 0.0)) + 2 * np.abs(ref[2][:, 1:]))))
    return z, ref


@pytest.mark.parametrize("name", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("c", WIDTHS)
def test_forward(env, name, c):  # noqa: F811
    torch, cbm = env
    rng = np.random.default_rng(c)
    for i, (n, pad, offset) in enumerate(((1, 0, 0), (5, 3, 1), (70 if c < 60000 else 9, 0, 0)) + (((3000, 4, 4),) if c <= 600 else ())):
        Z, _ = _matrix(torch, 3 * rng.standard_normal((n, c)), name, pad, offset)
        labels = rng.integers(-1, c + 1, n)
        for top in ((0, 1, 5, 32) if n > 1 else (20,)):
            _check(torch, Z, labels, _scores(torch, cbm, Z, labels, top, torch.int32 if top == 5 else None), top)


@pytest.mark.parametrize("name", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("c", [2, 8, 47, 100, 300, 1000, 1500, 9000, 40000])
def test_ties_and_orders(env, name, c):  # noqa: F811
    """Few different scores, all equal, rising, falling, the largest in one lane's columns, both zeros."""
    torch, cbm = env
    rng = np.random.default_rng(c + 1)
    z = np.zeros((8, c))
    z[0] = rng.integers(-2, 3, c)
    z[1] = 7.0
    z[2] = np.arange(c) / 8.0 % 2048
    z[3] = -np.arange(c) / 8.0 % 2048
    z[4, :32] = 10 + np.arange(min(c, 32)) / 4
    z[5] = np.where(rng.random(c) < 0.5, 0.0, -0.0)
    z[6] = np.where(np.arange(c) % 256 < 4, 5.0, rng.standard_normal(c))
    z[7] = torch.finfo(_type(torch, name)).min  # a mask of the type's lowest value all over: equal scores
    Z, _ = _matrix(torch, z, name, 0)
    labels = rng.integers(0, c, 8)
    for rows in (slice(0, 8), slice(1, 2), slice(2, 3), slice(4, 5)):
        for top in (1, 7, 32):
            part = Z[rows]
            _check(torch, part, labels[rows], _scores(torch, cbm, part, labels[rows], top), top)


@pytest.mark.parametrize("name", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("c", [1, 3, 8, 47, 200, 1000, 1500, 9000, 70000])
def test_masks_and_values_that_are_not_finite(env, name, c):  # noqa: F811
    torch, cbm = env
    rng = np.random.default_rng(c + 2)
    z = rng.standard_normal((9, c))
    z[0, rng.random(c) < 0.7] = -math.inf
    z[1] = -math.inf                          # nothing is left
    z[2] = -math.inf
    z[2, c // 2] = 1.0                        # one class is
    z[3] = torch.finfo(_type(torch, name)).min
    z[3, c - 1] = 0.0
    z[4, c - 1] = math.nan
    z[5, 0] = math.inf
    z[6] = math.nan
    z[7] = -math.inf
    z[7, 0] = math.nan
    Z, _ = _matrix(torch, z, name, 0)
    labels = rng.integers(0, c, 9)
    for rows in (slice(0, 9),) + tuple(slice(i, i + 1) for i in range(8)):
        part, want = Z[rows], labels[rows]
        got = _scores(torch, cbm, part, want, 6)
        zn, ref = _check(torch, part, want, got, 6)
        dlogp, dentropy = torch.ones(len(want), device="cuda"), torch.full((len(want),), 0.5, device="cuda")
        dZ = torch.full_like(part, 3.0)
        cbm.cbm_log_probs_backward(part, got[0], got[3], got[2], dlogp, dentropy, dZ)
        bad, empty = np.isnan(ref[2][:, 0]), np.isneginf(ref[2][:, 0])
        d = _numbers(dZ)
        assert np.isnan(d[bad]).all() and (d[empty] == 0).all() and np.isfinite(d[~bad]).all()
        off = np.isneginf(zn) & ~bad[:, None]
        off[np.arange(len(want)), want] = False
        assert (d[off] == 0).all()


@pytest.mark.parametrize("name", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("c", WIDTHS)
def test_backward(env, name, c):  # noqa: F811
    torch, cbm = env
    rng = np.random.default_rng(c + 3)
    for n, pad, offset in ((1, 0, 0), (5, 3, 1), (70 if c < 60000 else 9, 0, 0)) + (((3000, 4, 4),) if c <= 600 else ()):
        Z, _ = _matrix(torch, 3 * rng.standard_normal((n, c)), name, pad, offset)
        dZ, whole = _matrix(torch, np.zeros((n, c)), name, pad, offset)
        labels = rng.integers(-1, c + 1, n)
        L, _, entropy, stats, _, _ = _scores(torch, cbm, Z, labels, 0)
        a, b = (torch.from_numpy(rng.standard_normal(n).astype(np.float32)).cuda() for _ in range(2))
        for da, db in ((a, b), (a, None), (None, b)):
            cbm.cbm_log_probs_backward(Z, None if da is None else L, stats, None if db is None else entropy, da, db, dZ)
            z, st, H = _numbers(Z), _numbers(stats), _numbers(entropy)
            an, bn = (np.zeros(n) if t is None else _numbers(t) for t in (da, db))
            ref = orc.log_probs_backward(z, labels, st, H, an, bn)
            logs = z - st[:, :1] - st[:, 1:]
            p, given = np.exp(logs), (labels >= 0) & (labels < c)
            away, size = np.abs(z - st[:, :1]), np.abs(an * given)[:, None] + np.abs(bn)[:, None] * (np.abs(logs) + np.abs(H)[:, None])
            bound = p * U * (size * (2 * away + 6 * np.abs(logs) + 10) + np.abs(bn)[:, None] * (2 * away + 4 * np.abs(logs) + 2 * np.abs(H)[:, None])) + 2 * U * np.abs(ref) + 1e-37
            assert np.all(np.abs(_numbers(dZ) - ref) <= bound + ROUNDING[name] * (np.abs(ref) + bound) + (2.0 ** -25 if name == "f16" else 0.0)), (n, pad)
            _untouched(torch, dZ, whole, offset)
        last = dZ.clone()
        cbm.cbm_log_probs_backward(Z, None, stats, entropy, None, b, Z)  # in place
        assert torch.equal(Z, last)


def test_gradient_is_the_slope_of_the_forward_pass(env):  # noqa: F811
    torch, cbm = env
    rng = np.random.default_rng(3)
    n, c, h = 30, 47, 1e-5
    z, v = rng.standard_normal((n, c)).astype(np.float32), rng.standard_normal((n, c))
    labels, a, b = rng.integers(0, c, n), rng.standard_normal(n).astype(np.float32), rng.standard_normal(n).astype(np.float32)
    Z = torch.from_numpy(z).cuda()
    L, _, entropy, stats, _, _ = _scores(torch, cbm, Z, labels, 0)
    dZ = torch.empty_like(Z)
    cbm.cbm_log_probs_backward(Z, L, stats, entropy, torch.from_numpy(a).cuda(), torch.from_numpy(b).cuda(), dZ)
    loss = lambda t: (orc.log_probs(t, labels)[0] * a + orc.log_probs(t, labels)[1] * b).sum()  # noqa: E731
    # 1,400 terms below 10 with 200 roundings each at most
    assert (_numbers(dZ) * v).sum() == pytest.approx((loss(z + h * v) - loss(z - h * v)) / (2 * h), abs=1400 * 10 * 200 * U)


def test_no_rows_and_outputs_left_out(env):  # noqa: F811
    torch, cbm = env
    _scores(torch, cbm, torch.empty((0, 9), device="cuda"), np.zeros(0, dtype=np.int64), 3)
    none = torch.empty(0, device="cuda")
    cbm.cbm_log_probs_backward(torch.empty((0, 9), device="cuda"), torch.empty(0, dtype=torch.int64, device="cuda"), torch.empty((0, 2), device="cuda"), none, none, none,
                               torch.empty((0, 9), device="cuda"))
    for n, c in ((4, 40), (2, 5000), (600, 3000)):
        Z = torch.randn((n, c), device="cuda")
        L, logp, entropy, stats, _, _ = _scores(torch, cbm, Z, np.zeros(n, dtype=np.int64), 0)
        ws = torch.empty(cbm.cbm_log_probs_workspace_bytes(n, c, 4), dtype=torch.uint8, device="cuda")
        one = torch.zeros(n, device="cuda")
        cbm.cbm_log_probs(Z, L, one, workspace=ws)
        assert torch.equal(one, logp)
        cbm.cbm_log_probs(Z, None, None, one, workspace=ws)
        assert torch.equal(one, entropy)
        values, columns = torch.empty((n, 4), device="cuda"), torch.empty((n, 4), dtype=torch.int32, device="cuda")
        cbm.cbm_log_probs(Z, None, None, None, None, values, columns, ws)
        assert torch.equal(columns.long(), torch.topk(Z, 4).indices)


def test_more_than_2_to_the_31_values(env):  # noqa: F811
    torch, cbm = env
    n, c, last = 1 << 21, 1056, 100
    Z = torch.zeros((n, c), dtype=torch.float16, device="cuda")
    Z[-last:] = torch.randn((last, c), device="cuda")
    labels = np.arange(n) % c
    L, logp, entropy, stats, values, columns = _scores(torch, cbm, Z, labels, 3)
    # (a row of its own takes the same shape of workgroup where it is not shared: 600 rows)
    tail = _scores(torch, cbm, Z[-600:].clone(), labels[-600:], 3)
    assert all(torch.equal(a[-600:], b) for a, b in zip((logp, entropy, stats, values, columns), tail[1:]))
    dZ, small = torch.empty_like(Z), torch.empty_like(Z[-last:])
    one = torch.ones(n, device="cuda")
    cbm.cbm_log_probs_backward(Z, L, stats, entropy, one, one, dZ)
    cbm.cbm_log_probs_backward(Z[-last:].clone(), L[-last:].clone(), stats[-last:].clone(), entropy[-last:].clone(), one[:last], one[:last], small)
    assert torch.equal(dZ[-last:], small)


def test_graph_capture_replays(env):  # noqa: F811
    torch, cbm = env
    for n, c, top in ((3000, 47, 5), (3, 20000, 9)):
        Z, L = torch.randn((n, c), device="cuda"), torch.randint(0, c, (n,), device="cuda")
        outs = [torch.empty(n, device="cuda"), torch.empty(n, device="cuda"), torch.empty((n, 2), device="cuda"), torch.empty((n, top), device="cuda"),
                torch.empty((n, top), dtype=torch.int32, device="cuda"), torch.empty((n, c), device="cuda")]
        ws = torch.empty(cbm.cbm_log_probs_workspace_bytes(n, c, top), dtype=torch.uint8, device="cuda")
        one = torch.ones(n, device="cuda")

        def step():
            cbm.cbm_log_probs(Z, L, *outs[:5], ws)
            cbm.cbm_log_probs_backward(Z, L, outs[2], outs[1], one, one, outs[5])

        step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        for seed in range(3):
            Z.copy_(torch.randn((n, c), device="cuda") * (seed + 1))
            graph.replay()
            torch.cuda.synchronize()
            got = [t.clone() for t in outs]
            for t in outs:
                t.fill_(-5)
            step()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, outs))


def test_refusals(env):  # noqa: F811
    torch, cbm = env
    Z, dZ = torch.zeros((4, 5000), device="cuda"), torch.ones((4, 5000), device="cuda")
    L, s, st = torch.zeros(4, dtype=torch.int64, device="cuda"), torch.ones(4, device="cuda"), torch.ones((4, 2), device="cuda")
    v, col = torch.ones((4, 3), device="cuda"), torch.ones((4, 3), dtype=torch.int32, device="cuda")
    ws = torch.zeros(cbm.cbm_log_probs_workspace_bytes(4, 5000, 3), dtype=torch.uint8, device="cuda")
    assert ws.numel() > 0
    for bad in (lambda: cbm.cbm_log_probs(Z.cpu(), L, s, workspace=ws), lambda: cbm.cbm_log_probs(Z.double(), L, s, workspace=ws), lambda: cbm.cbm_log_probs(Z, L[:2], s, workspace=ws),
                lambda: cbm.cbm_log_probs(Z, L.float(), s, workspace=ws), lambda: cbm.cbm_log_probs(Z, L, s[:1], workspace=ws), lambda: cbm.cbm_log_probs(Z, L, s, None, s, workspace=ws),
                lambda: cbm.cbm_log_probs(Z, L, s, None, None, v, col[:, :2], ws), lambda: cbm.cbm_log_probs(Z, L, s, None, None, v, col.long(), ws),
                lambda: cbm.cbm_log_probs_backward(Z, L, st, s, s, s, dZ[:2]), lambda: cbm.cbm_log_probs_backward(Z, L, s, s, s, s, dZ), lambda: cbm.cbm_log_probs_backward(Z, L, st, s, s, s, dZ.half())):
        with pytest.raises(ValueError):
            bad()
    other = s.clone()
    for bad in (lambda: cbm.cbm_log_probs(Z, None, s, workspace=ws), lambda: cbm.cbm_log_probs(Z, L, s, workspace=None), lambda: cbm.cbm_log_probs(Z, L, s, None, None, v, col, ws[:-1]),
                lambda: cbm.cbm_log_probs(Z, L, s, s, None, workspace=ws), lambda: cbm.cbm_log_probs(Z, L, s, None, None, v, None, ws),
                lambda: cbm.cbm_log_probs(Z, L, s, None, None, torch.ones((4, 33), device="cuda"), torch.ones((4, 33), dtype=torch.int32, device="cuda"), ws),
                lambda: cbm.cbm_log_probs_backward(Z, None, st, s, other, None, dZ), lambda: cbm.cbm_log_probs_backward(Z, L, st, None, None, other, dZ),
                lambda: cbm.cbm_log_probs_backward(Z, L, None, s, other, None, dZ), lambda: cbm.cbm_log_probs_backward(Z, L, st, s, None, None, dZ),
                lambda: cbm.cbm_log_probs_backward(Z[:3], L[:3], st[:3], s[:3], other[:3], None, Z[1:])):
        with pytest.raises(cbm.CbmError) as e:
            bad()
        assert e.value.status == 1
    from paper_2409_02208_amd import binding

    lib, p, q, r = binding._lib(), Z.data_ptr(), L.data_ptr(), s.data_ptr()
    call = lambda n, c, t, ldz, bits, z=p: lib.cbm_log_probs(n, c, t, z, ldz, q, bits, r, None, None, 0, None, None, None, 0, None)  # noqa: E731
    assert [call(4, 40, 4, 40, 64), call(-1, 40, 0, 40, 64), call(4, 0, 0, 40, 64), call(4, 40, 0, 39, 64), call(4, 40, 0, 40, 16), call(4, 40, 0, 40, 64, None),
            call(4, 40, 0, 40, 64, p + 2)] == [1] * 7
    assert call(4, (1 << 24) + 1, 0, 1 << 25, 64) == 5
    assert not bool(Z.any()) and bool((dZ == 1).all()) and bool((v == 1).all()) and bool((s == 1).all())


@pytest.mark.parametrize("name", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,c", [(1, 49152), (1, 49153), (1, 70001), (7, 60000), (300, 50000)])
def test_ties_and_orders_in_the_longest_rows(env, name, n, c):  # noqa: F811
    """On both sides of the length from which workgroups share a row: all equal, rising, few different scores, the largest in a few lanes' columns."""
    torch, cbm = env
    rng = np.random.default_rng(c + n)
    kinds = [np.full(c, -2.0), np.arange(c) / 64.0 % 1024, rng.integers(-2, 3, c).astype(np.float64), np.where(np.arange(c) % 2048 < 8, 5.0, rng.standard_normal(c)),
             np.where(np.arange(c) < c - 40, -math.inf, 1.0)]
    for first in range(len(kinds)) if n == 1 else (0,):
        z = np.stack([kinds[(first + i) % len(kinds)] for i in range(n)])
        Z, _ = _matrix(torch, z, name, 0)
        labels = rng.integers(0, c, n)
        for top in (1, 8, 32):
            _check(torch, Z, labels, _scores(torch, cbm, Z, labels, top), top)
