"""Plain float64 definitions of the policy-update operators (numpy, one sequence and head at a time)."""
from __future__ import annotations

import math

import numpy as np


def visible(m, n, causal):
    """[m][n] truth values: query i sees key j where j <= i + n - m (causal), or every key."""
    if not causal:
        return np.ones((m, n), bool)
    return np.arange(n)[None, :] <= np.arange(m)[:, None] + (n - m)


def attention(q, k, v, scale, causal):
    """q [m][d], k, v [n][d] of one head -> (o, lse, p). Rows that see no key: o = 0, lse = -inf."""
    see = visible(len(q), len(k), causal)
    s = np.where(see, scale * (q @ k.T), -np.inf)
    some = see.any(1)
    top = np.where(some, np.max(s, axis=1, initial=-np.inf), 0.0)
    e = np.exp(s - top[:, None])
    total = e.sum(1)
    p = e / np.where(some, total, 1.0)[:, None]
    lse = np.where(some, top + np.log(np.where(some, total, 1.0)), -np.inf)
    return p @ v, lse, p


def attention_gradients(q, k, v, o, lse, do, scale, causal):
    """-> (dq, dk, dv, p, ds) with p from the given lse, ds without the factor scale."""
    see = visible(len(q), len(k), causal) & (lse > -np.inf)[:, None]
    p = np.where(see, np.exp(np.where(see, scale * (q @ k.T) - np.where(lse > -np.inf, lse, 0.0)[:, None], 0.0)), 0.0)
    ds = p * (do @ v.T - (do * o).sum(1)[:, None])
    return scale * ds @ k, scale * ds.T @ q, p.T @ do, p, ds


def norm(kind, x, eps):
    """Rows normalised, and their reciprocal deviations."""
    if kind == "none":
        return x, np.ones((len(x), 1))
    c = x - x.mean(1, keepdims=True) if kind == "layer" else x
    r = 1.0 / np.sqrt((c * c).mean(1, keepdims=True) + eps)
    return c * r, r


def norm_gradient(kind, xhat, r, g):
    if kind == "none":
        return g
    out = g - xhat * (g * xhat).mean(1, keepdims=True)
    if kind == "layer":
        out = out - g.mean(1, keepdims=True)
    return out * r


def gated_norm(x, y, gate, scale, shift, post_w, pre_w, post, pre, eps, alpha):
    """One sequence: x, y [rows][D] (y may be None), vectors [D]. -> (x_out, h)"""
    x_out = alpha * x
    if y is not None:
        x_out = x_out + gate * (norm(post, y, eps)[0] * post_w)
    return x_out, norm(pre, x_out, eps)[0] * pre_w * (1.0 + scale) + shift


def gated_norm_gradients(x_out, y, gate, scale, post_w, pre_w, dx_out, dh, post, pre, eps, alpha):
    """One sequence -> dict of dx, dy and the vectors' gradients."""
    xh, r = norm(pre, x_out, eps)
    t = dx_out + norm_gradient(pre, xh, r, dh * (1.0 + scale) * pre_w)
    out = {"dx": alpha * t, "dshift": dh.sum(0), "dscale": (dh * xh * pre_w).sum(0),
           "dpre_w": (dh * (1.0 + scale) * xh).sum(0)}
    if y is not None:
        yh, ry = norm(post, y, eps)
        out.update(dy=norm_gradient(post, yh, ry, t * gate * post_w), dgate=(t * yh * post_w).sum(0),
                   dpost_w=(t * gate * yh).sum(0))
    return out


def step_mean(x, v, t, t_next, a):
    """Mean and variance of the SDE step's transition."""
    h, sigma = t_next - t, a * math.sqrt(t / (1.0 - t))
    return x + h * (v + sigma * sigma / (2.0 * t) * (x + (1.0 - t) * v)), sigma * sigma * -h


def policy_loss(x, v, x_next, logp_old, adv, t, t_next, a, logp_scale, clip_low, clip_high, v_ref=None, kl_weight=0.0):
    """x, v, x_next, v_ref [B][n] -> dict of loss, logp, ratio, dv."""
    B, n = x.shape
    mean, var = step_mean(x, v, t, t_next, a)
    dmean = (step_mean(x, v + 1.0, t, t_next, a)[0] - mean).flat[0]      # the mean is linear in v
    e = x_next - mean
    logp = -(e * e).sum(1) / (2.0 * var) - 0.5 * n * math.log(2.0 * math.pi * var)
    with np.errstate(over="ignore", invalid="ignore"):
        ratio = np.exp(logp_scale * (logp - logp_old))
        free = np.where(adv == 0.0, 0.0, ratio * adv)
        clipped = np.clip(ratio, 1.0 - clip_low, 1.0 + clip_high) * adv
        loss = -np.minimum(free, clipped)
        slope = np.where(free <= clipped, -free * logp_scale, 0.0) / B
    dv = np.where(slope[:, None] == 0.0, 0.0, slope[:, None] * dmean / var * e)
    if v_ref is not None:
        apart = mean - step_mean(x, v_ref, t, t_next, a)[0]
        loss = loss + kl_weight * logp_scale * (apart * apart).sum(1) / (2.0 * var)
        dv = dv + kl_weight * logp_scale / B * dmean / var * apart
    return {"loss": loss.mean(), "logp": logp, "ratio": ratio, "dv": dv}
