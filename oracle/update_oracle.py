"""Plain float64 definitions of the end of a policy update and of linear layers in 8-bit integers (numpy)."""
from __future__ import annotations

import numpy as np


def quantize_rows(x):
    """x [rows][cols] -> (integers, scales). The scale is an fp32 number by definition; the quotient is rounded exactly, ties to
    even: 64 bits separate the quotient of two fp32 numbers from any half that it does not equal."""
    x = np.asarray(x, np.float64)
    top = np.abs(x).max(axis=1, initial=0.0)
    bad = ~np.isfinite(x).all(axis=1)
    scale = np.maximum((np.where(bad, 0.0, top) / 127).astype(np.float32), np.float32(2.0 ** -126)).astype(np.float64)
    q = np.rint(np.where(bad[:, None], 0.0, x) / scale[:, None])
    return q.astype(np.int64), np.where(bad, np.nan, scale)


def gelu_tanh(z):
    return 0.5 * z * (1 + np.tanh(np.sqrt(2 / np.pi) * (z + 0.044715 * z ** 3)))


def int8_matmul(xq, xs, wq, ws, bias=None, gelu=False):
    """-> (y, the integer sums). The sums are below 2^53: exact in float64."""
    total = xq.astype(np.float64) @ wq.astype(np.float64).T
    y = total * xs[:, None] * ws[None, :]
    if bias is not None:
        y = y + bias
    return (gelu_tanh(y) if gelu else y), total


def grad_norm(grads, max_norm):
    """-> (norm, scale); the scale of a norm that is not finite is NaN."""
    norm = np.sqrt(sum(float((np.asarray(g, np.float64) ** 2).sum()) for g in grads))
    return norm, (min(1.0, max_norm / (norm + 1e-6)) if np.isfinite(norm) else np.nan)


def adamw(p, g, m, v, lr, beta1, beta2, eps, decay, t, scale=1.0):
    """-> (p, m, v)"""
    if np.isnan(scale):
        return p, m, v
    g = scale * g
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    return p - lr * (m / (1 - beta1 ** t) / (np.sqrt(v / (1 - beta2 ** t)) + eps) + decay * p), m, v
