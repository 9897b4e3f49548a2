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
