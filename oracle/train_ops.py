"""Plain 64-bit forms of layer norm, the embedding, their gradients, and gradient clipping: what the HIP kernels are checked against.

    norm           mean, rstd = 1 / sqrt(variance + eps) of every row;  y = (x - mean) * rstd * gamma + beta
    norm backward  h = (x - mean) * rstd,  g = dy * gamma;  dx = rstd * (g - mean(g) - h * mean(g * h)) + residual;  dgamma = column sums of dy * h,  dbeta of dy
    embedding      y[i] = scale * table[token[i]];  padding: zeros;  other tokens outside the table: NaN
    its gradient   dtable[v] = scale * the sum of dy[i] over token[i] = v
    clipping       norm of everything;  grad * max_norm / norm if norm is finite and above max_norm
"""
from __future__ import annotations

import numpy as np


def layer_norm(x, gamma=None, beta=None, eps=1e-5):
    """Returns (y, mean, rstd)."""
    x = np.asarray(x, np.float64)
    mean = x.mean(1)
    rstd = 1 / np.sqrt(((x - mean[:, None]) ** 2).mean(1) + float(np.float32(eps)))
    y = (x - mean[:, None]) * rstd[:, None]
    if gamma is not None:
        y = y * np.asarray(gamma, np.float64)
    return (y if beta is None else y + np.asarray(beta, np.float64)), mean, rstd


def layer_norm_bwd(dy, x, mean, rstd, gamma=None, residual=None):
    """mean, rstd: as the forward pass stored them.  Returns (dx, dgamma, dbeta)."""
    dy, x = np.asarray(dy, np.float64), np.asarray(x, np.float64)
    r = np.asarray(rstd, np.float64)[:, None]
    h = (x - np.asarray(mean, np.float64)[:, None]) * r
    g = dy if gamma is None else dy * np.asarray(gamma, np.float64)
    dx = r * (g - g.mean(1, keepdims=True) - h * (g * h).mean(1, keepdims=True))
    return (dx if residual is None else dx + np.asarray(residual, np.float64)), (dy * h).sum(0), dy.sum(0)


def embedding(tokens, table, scale=1.0, pad=-1):
    tokens, table = np.asarray(tokens).reshape(-1), np.asarray(table, np.float64)
    y = np.full((tokens.size, table.shape[1]), np.nan)
    for i, t in enumerate(tokens.tolist()):
        if t == pad:
            y[i] = 0
        elif 0 <= t < table.shape[0]:
            y[i] = float(np.float32(scale)) * table[t]
    return y


def embedding_bwd(dy, tokens, vocab, scale=1.0, pad=-1, start=None):
    dy, out = np.asarray(dy, np.float64), np.zeros((vocab, np.shape(dy)[1]))
    for i, t in enumerate(np.asarray(tokens).reshape(-1).tolist()):
        if t != pad and 0 <= t < vocab:
            out[t] += dy[i]
    out *= float(np.float32(scale))
    return out if start is None else out + np.asarray(start, np.float64)


def grad_clip(grads, max_norm):
    """Returns (norm, factor, clipped)."""
    with np.errstate(over="ignore"):
        norm = float(np.sqrt(sum((np.asarray(g, np.float64) ** 2).sum() for g in grads)))
        n32 = float(np.float32(norm))
    factor = float(np.float32(max_norm)) / norm if np.isfinite(n32) and n32 > float(np.float32(max_norm)) else 1.0
    return norm, factor, [np.asarray(g, np.float64) * factor for g in grads]
