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
