"""The policy-update oracle's gradients against central differences of its own forward definitions, and what the
definitions give where a mask leaves nothing, a ratio is clipped or an advantage is zero."""
import numpy as np
import pytest

from oracle import policy_oracle as P

STEP = 1e-5          # differences of O(1) functions: error ~ STEP^2 + 1e-16 / STEP, below 1e-9 relative to O(1) sums
TOL = 2e-8


def differences(f, x):
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        keep = x[i]
        x[i] = keep + STEP
        up = f()
        x[i] = keep - STEP
        down = f()
        x[i] = keep
        g[i] = (up - down) / (2 * STEP)
    return g


@pytest.mark.parametrize("m,n,causal", [(4, 4, True), (3, 6, True), (5, 3, True), (3, 5, False), (1, 1, True)])
def test_attention_gradients(rng, m, n, causal):
    q, k, v, do = rng.standard_normal((m, 6)), rng.standard_normal((n, 6)), rng.standard_normal((n, 6)), rng.standard_normal((m, 6))
    o, lse, p = P.attention(q, k, v, 0.4, causal)
    got = P.attention_gradients(q, k, v, o, lse, do, 0.4, causal)[:3]
    for g, x in zip(got, (q, k, v)):
        want = differences(lambda: float((P.attention(q, k, v, 0.4, causal)[0] * do).sum()), x)
        np.testing.assert_allclose(g, want, atol=TOL)


def test_attention_rows_without_keys():
    rng = np.random.default_rng(0)
    q, k = rng.standard_normal((5, 4)), rng.standard_normal((2, 4))
    o, lse, p = P.attention(q, k, k, 1.0, True)       # queries 0..2 stand before the first key
    assert np.all(o[:3] == 0) and np.all(lse[:3] == -np.inf) and np.all(np.isfinite(lse[3:]))
    np.testing.assert_allclose(p[3:].sum(1), 1.0)
    dq, dk, dv, *_ = P.attention_gradients(q, k, k, o, lse, np.ones((5, 4)), 1.0, True)
    assert np.all(dq[:3] == 0) and np.all(np.isfinite(dk)) and np.all(np.isfinite(dv))


@pytest.mark.parametrize("post", ["none", "layer", "rms"])
@pytest.mark.parametrize("pre", ["none", "layer", "rms"])
def test_gated_norm_gradients(rng, post, pre):
    R, D, eps, alpha = 3, 7, 1e-3, 0.7
    a = {n: rng.standard_normal((R, D)) for n in ("x", "y")}
    a.update({n: rng.standard_normal(D) for n in ("gate", "scale", "shift", "post_w", "pre_w")})
    cx, ch = rng.standard_normal((R, D)), rng.standard_normal((R, D))

    def f():
        xo, h = P.gated_norm(a["x"], a["y"], a["gate"], a["scale"], a["shift"], a["post_w"], a["pre_w"], post, pre, eps, alpha)
        return float((xo * cx).sum() + (h * ch).sum())

    xo, _ = P.gated_norm(a["x"], a["y"], a["gate"], a["scale"], a["shift"], a["post_w"], a["pre_w"], post, pre, eps, alpha)
    got = P.gated_norm_gradients(xo, a["y"], a["gate"], a["scale"], a["post_w"], a["pre_w"], cx, ch, post, pre, eps, alpha)
    for n in a:
        np.testing.assert_allclose(got["d" + n], differences(f, a[n]), atol=50 * TOL, err_msg=n)


@pytest.mark.parametrize("reference", [False, True])
def test_policy_loss_gradient(rng, reference):
    B, n, t, tn, lvl = 4, 5, 0.6, 0.5, 0.7
    x, v, eps = (rng.standard_normal((B, n)) for _ in range(3))
    mean, var = P.step_mean(x, v + 0.1, t, tn, lvl)
    xn = mean + np.sqrt(var) * eps
    old = P.policy_loss(x, v + 0.1, xn, np.zeros(B), np.zeros(B), t, tn, lvl, 1.0, 0.2, 0.2)["logp"]
    adv = np.array([1.0, -1.0, 2.0, 0.0])
    ref = v + 0.3 * rng.standard_normal((B, n)) if reference else None

    def f():
        return float(P.policy_loss(x, v, xn, old, adv, t, tn, lvl, 1.0 / n, 0.2, 0.3, ref, 0.1)["loss"])

    got = P.policy_loss(x, v, xn, old, adv, t, tn, lvl, 1.0 / n, 0.2, 0.3, ref, 0.1)
    np.testing.assert_allclose(got["dv"], differences(f, v), atol=TOL)


def test_policy_loss_clips_and_ignores_a_zero_advantage():
    x = np.zeros((4, 2))
    v = np.zeros((4, 2))
    xn, _ = P.step_mean(x, v, 0.5, 0.4, 0.7)
    logp = P.policy_loss(x, v, xn, np.zeros(4), np.zeros(4), 0.5, 0.4, 0.7, 1.0, 0.2, 0.2)["logp"]
    old = logp - np.array([1.0, 1.0, -1.0, 1e4])      # ratios e, e, 1/e and inf
    got = P.policy_loss(x, v, xn + 0.01, old, np.array([1.0, -1.0, -1.0, 0.0]), 0.5, 0.4, 0.7, 1.0, 0.2, 0.2)
    r = got["ratio"]
    np.testing.assert_allclose(got["loss"], (-1.2 + r[1] + 0.8 + 0.0) / 4)
    assert np.all(got["dv"][0] == 0) and np.any(got["dv"][1] != 0) and np.all(got["dv"][2:] == 0)
