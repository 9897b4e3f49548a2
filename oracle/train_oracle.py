"""The operators between the products of a training step, from their definitions in 64 bits (numpy): what the kernels are checked against."""
from __future__ import annotations

import numpy as np

BLOCK = 32  # columns of a row that share a step in the 8-bit form


def layer_norm(x, gamma=None, beta=None, eps=1e-5):
    """(y, mean, rstd) of each row."""
    x = np.asarray(x, dtype=np.float64)
    m = x.mean(axis=1)
    c = x - m[:, None]
    with np.errstate(divide="ignore", invalid="ignore"):
        r = 1.0 / np.sqrt((c * c).mean(axis=1) + eps)
        y = c * r[:, None]
    if gamma is not None:
        y = y * np.asarray(gamma, dtype=np.float64)
    if beta is not None:
        y = y + np.asarray(beta, dtype=np.float64)
    return y, m, r


def layer_norm_backward(dy, x, gamma, mean, rstd):
    """(dx, dgamma, dbeta) with the row statistics as given."""
    dy, x = np.asarray(dy, dtype=np.float64), np.asarray(x, dtype=np.float64)
    r = np.asarray(rstd, dtype=np.float64)[:, None]
    h = (x - np.asarray(mean, dtype=np.float64)[:, None]) * r
    u = dy if gamma is None else dy * np.asarray(gamma, dtype=np.float64)
    dx = r * (u - u.mean(axis=1, keepdims=True) - h * (u * h).mean(axis=1, keepdims=True))
    return dx, (dy * h).sum(axis=0), dy.sum(axis=0)


def keep(x):
    """(q, e): whole numbers of steps 2^e, one step for each 32 columns of a row; e = 128 for a block that is not finite."""
    x = np.asarray(x, dtype=np.float64)
    n, k = x.shape
    q, e = np.zeros((n, k), dtype=np.int64), np.zeros((n, -(-k // BLOCK)), dtype=np.int64)
    for b in range(e.shape[1]):
        part = x[:, b * BLOCK:(b + 1) * BLOCK]
        with np.errstate(invalid="ignore"):
            finite = np.isfinite(part).all(axis=1)
        part = np.where(finite[:, None], part, 0.0)
        largest = np.abs(part).max(axis=1)
        exponent = np.frexp(largest)[1].astype(np.int64) - 1  # largest = f 2^exponent, 1 <= f < 2
        step = np.maximum(np.where(largest > 0, exponent - 6, -126), -126)
        size = np.clip(np.rint(np.ldexp(np.abs(part), -step[:, None])), 1, 127)
        q[:, b * BLOCK:(b + 1) * BLOCK] = np.where(part == 0, 0, np.sign(part) * size)
        e[:, b] = np.where(finite, step, 128)
    return q, e


def kept_values(q, e):
    step = np.repeat(np.where(e == 128, np.nan, np.ldexp(1.0, np.where(e == 128, 0, e))), BLOCK, axis=1)[:, :q.shape[1]]
    return q * step


def relu_backward(q, e, dy):
    bad = np.repeat(e == 128, BLOCK, axis=1)[:, :q.shape[1]]
    return np.where(bad, np.nan, np.where(q > 0, dy, 0.0))


def weight_grad(q, e, dy):
    with np.errstate(invalid="ignore"):
        return kept_values(q, e).T @ np.asarray(dy, dtype=np.float64)


def log_probs(z, labels, top=0):
    """(log p[label], entropy, (m, l), values, columns): see the C ABI's header for rows without a distribution."""
    z = np.asarray(z, dtype=np.float64)
    n, c = z.shape
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        m = z.max(axis=1)
        bad, empty = ~(m < np.inf), m == -np.inf  # (NaN passes through max)
        d = z - np.where(empty, 0.0, m)[:, None]
        e = np.exp(d)
        s = e.sum(axis=1)
        l = np.log(s)  # noqa: E741
        entropy = np.where(empty, 0.0, l - np.where(e > 0, d * e, 0.0).sum(axis=1) / np.where(empty, 1.0, s))
        logs = np.where(empty[:, None], -np.inf, d - np.where(empty, 0.0, l)[:, None])
    labels = np.asarray(labels)
    given = (labels >= 0) & (labels < c)
    logp = np.where(given, logs[np.arange(n), np.where(given, labels, 0)], 0.0)
    m, l, entropy = (np.where(bad, np.nan, a) for a in (m, l, entropy))  # noqa: E741
    logp = np.where(bad & given, np.nan, logp)
    values, columns = np.full((n, top), -np.inf), np.full((n, top), -1, dtype=np.int64)
    if top:
        order = np.argsort(-np.where(np.isnan(z), -np.inf, z), axis=1, kind="stable")[:, :top]  # (equal scores: the lower column first)
        some = order.shape[1]
        there = np.take_along_axis(z, order, axis=1) > -np.inf
        columns[:, :some] = np.where(there & ~bad[:, None], order, -1)
        values[:, :some] = np.where(there, np.take_along_axis(logs, order, axis=1), -np.inf)
        values[bad] = np.nan
    return logp, entropy, np.stack([m, l], axis=1), values, columns


def log_probs_backward(z, labels, stats, entropy, dlogp, dentropy):
    z, stats = np.asarray(z, dtype=np.float64), np.asarray(stats, dtype=np.float64)
    n, c = z.shape
    labels = np.asarray(labels)
    given = (labels >= 0) & (labels < c)
    empty = stats[:, 0] == -np.inf
    with np.errstate(invalid="ignore"):
        logs = np.where(empty[:, None], -np.inf, z - stats[:, :1] - stats[:, 1:])
    p = np.exp(logs)
    a = np.where(given & ~empty, dlogp, 0.0)[:, None]
    hot = np.zeros_like(z)
    hot[np.arange(n), np.where(given, labels, 0)] = 1.0
    slope = np.where(logs == -np.inf, 0.0, p * (np.where(logs == -np.inf, 0.0, logs) + np.asarray(entropy, dtype=np.float64)[:, None]))
    return a * (hot - p) - np.asarray(dentropy, dtype=np.float64)[:, None] * slope


def activation(name, g):
    """(a(g), a'(g))."""
    from scipy.special import erfc, expit

    g = np.asarray(g, dtype=np.float64)
    if name == "relu":
        return np.where(g <= 0, 0.0, g), (g > 0).astype(np.float64)
    with np.errstate(over="ignore", invalid="ignore"):
        if name == "silu":
            s = expit(g)
            return g * s, s * (1 + g * expit(-g))
        below = 0.5 * erfc(-g / np.sqrt(2.0))
        return g * below, below + g * np.exp(-0.5 * g * g) / np.sqrt(2 * np.pi)


def gated_linear(x, wg, wu, name):
    """(h, g, u)."""
    x, wg, wu = (np.asarray(a, dtype=np.float64) for a in (x, wg, wu))
    g, u = x @ wg, x @ wu
    return activation(name, g)[0] * u, g, u


def gated_linear_backward(dh, x, wg, wu, g, u, name):
    """(dx, dwg, dwu), and dg and du that they are made of."""
    dh, x, wg, wu, g, u = (np.asarray(a, dtype=np.float64) for a in (dh, x, wg, wu, g, u))
    value, slope = activation(name, g)
    du, dg = dh * value, dh * u * slope
    return dg @ wg.T + du @ wu.T, x.T @ dg, x.T @ du, dg, du


def linear_log_probs_backward(x, w, labels, stats, dlogp):
    """(dx, dw), and dz that they are made of."""
    x, w = np.asarray(x, dtype=np.float64), np.asarray(w, dtype=np.float64)
    zero = np.zeros(len(x))
    dz = log_probs_backward(x @ w, labels, stats, zero, np.where((np.asarray(labels) >= 0) & (np.asarray(labels) < w.shape[1]), dlogp, 0.0), zero)
    return dz @ w.T, x.T @ dz, dz


def orthogonalise(x, steps=5, coefficients=(3.4445, -4.7750, 2.0315), eps=1e-7, scale=1.0):
    z = np.asarray(x, dtype=np.float64)
    a, b, c = coefficients
    with np.errstate(divide="ignore", invalid="ignore"):
        z = z / (np.sqrt((z * z).sum()) + eps)
    for _ in range(steps):
        gram = z @ z.T if z.shape[0] <= z.shape[1] else z.T @ z
        p = a * np.eye(len(gram)) + b * gram + c * gram @ gram
        z = p @ z if z.shape[0] <= z.shape[1] else z @ p
    return scale * z
