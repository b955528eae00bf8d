"""Plain 64-bit forms of the linear layer with its epilogue, of its gradients, and of dropout: what the HIP kernels are checked against.

    forward   y = dropout(act(z)) + residual,  z = x W^T + bias
    backward  dz = act'(z) * dropout(dy);  dx = dz W,  dW = dz^T x,  db = column sums of dz
"""
from __future__ import annotations

import numpy as np
from scipy.special import ndtr

ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")     # in the order of sol_act


def philox4x32(counter, key):
    """Philox4x32-10 on an array [..., 4] of counters (Salmon, Moraes, Dror, Shaw, SC 2011)."""
    c = [np.asarray(counter)[..., i].astype(np.uint64) for i in range(4)]
    k = [int(key[0]), int(key[1])]
    low = np.uint64(0xFFFFFFFF)
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), b & low, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), a & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return np.stack(c, -1).astype(np.uint32)


def dropout_threshold(p):
    return int(np.rint(float(np.float32(p)) * 65536))


def dropout_kept(rows, cols, p, seed, call=0, step=0):
    """Truth array [rows][cols] of the elements that are kept."""
    groups = (cols + 7) // 8
    ctr = np.empty((rows, groups, 4), np.uint32)
    ctr[..., 0], ctr[..., 1] = np.arange(groups)[None, :], np.arange(rows)[:, None]
    ctr[..., 2], ctr[..., 3] = call, step
    w = philox4x32(ctr, (seed & 0xFFFFFFFF, seed >> 32 & 0xFFFFFFFF))
    halves = np.stack([w & 0xFFFF, w >> 16], -1).reshape(rows, groups * 8)[:, :cols]
    return halves >= dropout_threshold(p)


def dropout(v, p, seed, call=0, step=0):
    v = np.asarray(v, np.float64)
    t = dropout_threshold(p)
    if t == 65536:
        return np.zeros_like(v)
    return np.where(dropout_kept(*v.shape, p, seed, call, step), v * (65536 / (65536 - t)), 0.0)


def act(name, z):
    if name == "relu":
        return np.maximum(z, 0.0)
    if name == "gelu":
        return z * ndtr(z)
    if name == "gelu_tanh":
        return 0.5 * z * (1 + np.tanh(np.sqrt(2 / np.pi) * (z + 0.044715 * z**3)))
    return z / (1 + np.exp(-z)) if name == "silu" else z


def slope(name, z):
    if name == "relu":
        return (z > 0).astype(np.float64)
    if name == "gelu":
        return ndtr(z) + z * np.exp(-z * z / 2) / np.sqrt(2 * np.pi)
    if name == "gelu_tanh":
        t = np.tanh(np.sqrt(2 / np.pi) * (z + 0.044715 * z**3))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * np.sqrt(2 / np.pi) * (1 + 3 * 0.044715 * z * z)
    if name == "silu":
        s = 1 / (1 + np.exp(-z))
        return s * (1 + z * (1 - s))
    return np.ones_like(z)


def linear_fused(x, w, bias=None, act_name="none", drop=None, residual=None):
    """drop: None or (p, seed, call, step).  Returns (y, z)."""
    z = np.asarray(x, np.float64) @ np.asarray(w, np.float64).T
    if bias is not None:
        z = z + np.asarray(bias, np.float64)
    y = act(act_name, z)
    if drop is not None:
        y = dropout(y, *drop)
    return (y if residual is None else y + np.asarray(residual, np.float64)), z


def linear_dz(dy, z, act_name="none", drop=None):
    g = np.asarray(dy, np.float64)
    if drop is not None:
        g = dropout(g, *drop)
    return g if act_name == "none" else g * slope(act_name, np.asarray(z, np.float64))


def linear_fused_bwd(dy, x, w, z, act_name="none", drop=None):
    """Returns (dx, dW, db, dz)."""
    dz = linear_dz(dy, z, act_name, drop)
    return dz @ np.asarray(w, np.float64), dz.T @ np.asarray(x, np.float64), dz.sum(0), dz
