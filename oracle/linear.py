"""Plain CPU oracle of the linear-layer operators, by their definitions (numpy, float64; integers where they are exact)."""

from __future__ import annotations

import numpy as np


def quantize_i8(x: np.ndarray):
    """(q [M, ceil(K / 16) * 16] int8, scale [M] float32) of x [M, K].

    scale = max |x| / 127 rounded to float32; q = the integer nearest to x / scale, halves to even.  The quotient is taken in
    float64: x and scale have at most 24 bits, so a quotient that is not a half differs from it by at least 2^-26 relative, far
    above float64's rounding.  A row with a value that is not finite gets scale NaN and q = 0."""
    x = np.asarray(x, dtype=np.float64)
    M, K = x.shape
    kp = (K + 15) // 16 * 16
    q = np.zeros((M, kp), dtype=np.int8)
    fine = np.isfinite(x).all(axis=1)
    scale = np.full(M, np.nan, dtype=np.float32)
    scale[fine] = (np.abs(x[fine]).max(axis=1) / 127.0).astype(np.float32)
    for m in np.nonzero(fine & (scale > 0))[0]:
        q[m, :K] = np.clip(np.rint(x[m] / np.float64(scale[m])), -127, 127).astype(np.int8)
    return q, scale


def gemm_i8(A, a_scale, B, b_scale) -> np.ndarray:
    """float32 of a_scale * b_scale * (A . B^T): exact integer sums, then one float32 rounding per step."""
    acc = np.asarray(A, dtype=np.float64) @ np.asarray(B, dtype=np.float64).T   # |sum| < 2^31: exact
    with np.errstate(invalid="ignore"):
        return (acc.astype(np.float32) * np.asarray(a_scale, np.float32)[:, None]) * np.asarray(b_scale, np.float32)[None, :]


def linear_ce(h, W, target, reduction: str, ignore_index: int = -100):
    """(loss, lse, each, kept) in float64; loss is a vector for "none", else one number."""
    z = np.asarray(h, np.float64) @ np.asarray(W, np.float64).T
    top = z.max(axis=1)
    lse = top + np.log(np.exp(z - top[:, None]).sum(axis=1))
    kept = target != ignore_index
    each = np.zeros(len(lse))
    each[kept] = lse[kept] - z[np.nonzero(kept)[0], target[kept]]
    if reduction == "none":
        loss = each
    else:
        with np.errstate(invalid="ignore"):
            loss = each.sum() / (np.float64(kept.sum()) if reduction == "mean" else 1.0)
    return loss, lse, each, kept


def linear_ce_grad(h, W, target, grad, reduction: str, ignore_index: int = -100):
    """(dh, dW, g, p, c) in float64: g = c (p - onehot), c = 0 for ignored tokens."""
    h, W = np.asarray(h, np.float64), np.asarray(W, np.float64)
    z = h @ W.T
    p = np.exp(z - z.max(axis=1, keepdims=True))
    p /= p.sum(axis=1, keepdims=True)
    kept = target != ignore_index
    c = np.zeros(len(target))
    if kept.any():
        c[kept] = (np.broadcast_to(np.asarray(grad, np.float64), target.shape) / (kept.sum() if reduction == "mean" else 1.0))[kept]
    g = p.copy()
    g[np.nonzero(kept)[0], target[kept]] -= 1.0
    g *= c[:, None]
    return g @ W, g.T @ h, g, p, c
