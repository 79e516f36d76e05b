"""Plain CPU oracle of distillation from a teacher's top logits, by its definition (numpy, float64): every word of the vocabulary has its own q and p."""

from __future__ import annotations

import numpy as np


def teacher(top_index, top_logit, V: int, temperature: float):
    """(q [T, V], kept [T]): the softmax of the used logits / temperature, added up by word."""
    T, K = top_index.shape
    q, kept = np.zeros((T, V)), np.zeros(T, dtype=bool)
    for t in range(T):
        used = [j for j in range(K) if top_index[t, j] >= 0 and top_logit[t, j] != -np.inf]
        if not used:
            continue
        kept[t] = True
        x = np.asarray([np.float64(top_logit[t, j]) / temperature for j in used])
        e = np.exp(x - x.max())
        for j, m in zip(used, e / e.sum()):
            q[t, top_index[t, j]] += m
    return q, kept


def linear_distill(h, W, top_index, top_logit, temperature: float, reduction: str):
    """(loss, lse, diff, each, kept, p, q); loss is a vector for "none", else one number."""
    z = np.asarray(h, np.float64) @ np.asarray(W, np.float64).T / temperature
    top = z.max(axis=1, keepdims=True)
    lse = (top + np.log(np.exp(z - top).sum(axis=1, keepdims=True)))[:, 0]
    logp = z - lse[:, None]
    q, kept = teacher(top_index, top_logit, z.shape[1], temperature)
    with np.errstate(divide="ignore", invalid="ignore"):
        each = temperature ** 2 * np.where(q > 0, q * (np.log(q) - logp), 0.0).sum(axis=1)
    p = np.exp(logp)
    diff = np.where(top_index >= 0, np.take_along_axis(p - q, np.maximum(top_index, 0), axis=1), 0.0)
    each[~kept], diff[~kept], lse[~kept] = 0.0, 0.0, np.inf
    if reduction == "none":
        loss = each
    else:
        with np.errstate(invalid="ignore"):
            loss = each.sum() / (np.float64(kept.sum()) if reduction == "mean" else 1.0)
    return loss, lse, diff, each, kept, p, q


def linear_distill_grad(h, W, top_index, top_logit, grad, temperature: float, reduction: str):
    """(dh, dW) in float64."""
    _, _, _, _, kept, p, q = linear_distill(h, W, top_index, top_logit, temperature, reduction)
    c = np.where(kept, np.broadcast_to(np.asarray(grad, np.float64), kept.shape), 0.0) / (max(kept.sum(), 1) if reduction == "mean" else 1.0)
    g = (c * temperature)[:, None] * (p - q)
    return g @ np.asarray(W, np.float64), g.T @ np.asarray(h, np.float64)
