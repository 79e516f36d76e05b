"""Plain CPU oracle of layer norm and its gradients, by their definitions (numpy, float64)."""

from __future__ import annotations

import numpy as np


def layernorm(x, gamma=None, beta=None, eps: float = 1e-5):
    """(y, mean, rstd) of the rows of x [M, N]."""
    x = np.asarray(x, np.float64)
    with np.errstate(invalid="ignore", divide="ignore"):
        mean = x.mean(axis=1)
        c = x - mean[:, None]
        rstd = 1.0 / np.sqrt((c * c).mean(axis=1) + eps)
        y = c * rstd[:, None]
        if gamma is not None:
            y = y * np.asarray(gamma, np.float64)
        if beta is not None:
            y = y + np.asarray(beta, np.float64)
    return y, mean, rstd


def layernorm_grad(dy, x, gamma, mean, rstd):
    """(dx, dgamma, dbeta, xh, u) for the gradient dy of y, with the given mean and rstd."""
    dy, x = np.asarray(dy, np.float64), np.asarray(x, np.float64)
    mean, rstd = np.asarray(mean, np.float64)[:, None], np.asarray(rstd, np.float64)[:, None]
    with np.errstate(invalid="ignore"):
        xh = (x - mean) * rstd
        u = dy if gamma is None else dy * np.asarray(gamma, np.float64)
        dx = rstd * (u - u.mean(axis=1, keepdims=True) - xh * (u * xh).mean(axis=1, keepdims=True))
        return dx, (dy * xh).sum(axis=0), dy.sum(axis=0), xh, u
