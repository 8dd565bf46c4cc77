"""packed_attention at values where a softmax goes wrong first: a NaN in a used row, and scores so large that what is left of a
difference of two of them has to be exact.

The scores of the second kind are products of powers of two, so they are exact in every kernel and the bounds hold no error of
theirs: o is off by U |o| + (P + (n + 8) 2^-24) sum p |v| (U, P: tests/policy_util.py), lse by 2^-21 of its size."""
import numpy as np
import pytest
import torch

from oracle import policy_oracle as P
from tests.gpu_util import host64
from tests.policy_util import F32, UNIT, attention_reference, check, stored, to_dev
from tests.test_gpu_packed_attention import Problem

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def d():
    from paper_2606_19004_amd import ditstep
    return ditstep


# H, G, q lengths, k lengths (None: the same), causal: few rows whole and in parts, wide tiles whole and in parts, many tiles
FORMS = {"few": (8, 2, [1, 1], [150, 60], True), "few in parts": (8, 2, [1, 1], [2000, 900], True),
         "wide": (4, 2, [70, 33], [100, 33], True), "wide in parts": (2, 1, [40], [3000], True),
         "many": (16, 16, [40, 9, 64] * 14, None, True)}


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("form", FORMS)
def test_a_nan_query_gives_a_nan_row(d, form, dtype, hd):
    """However the keys are shared out, and no other row changes."""
    H, G, ql, kl, causal = FORMS[form]
    p = Problem(d, dtype, hd, H, G, ql, kl, causal, lead=1, tail=1, seed=hd + len(ql))
    assert (d.packed_attention_workspace_bytes(p.cfg) > 0) == ("parts" in form)
    ref = p.reference()
    row, head = int(p.q_off[0]), 1
    p.tq[row, head] = float("nan")
    o, lse = p.forward()
    assert np.isnan(o[row, head]).all() and np.isnan(lse[row, head])
    ref["o"][row, head] = ref["lse"][row, head] = np.nan
    check(o, ref["o"], ref["o_tol"], "o")
    check(lse, ref["lse"], ref["lse_tol"], "lse")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("form", FORMS)
def test_a_nan_key_reaches_the_rows_that_see_it(d, form, dtype):
    """The first key of the first sequence, one key/value head: the rows of its query heads, and none of the others."""
    H, G, ql, kl, causal = FORMS[form]
    p = Problem(d, dtype, 64, H, G, ql, kl, causal, seed=3)
    ref = p.reference()
    p.tk[int(p.k_off[0]), 0] = float("nan")
    o, lse = p.forward()
    rows, heads = slice(0, ql[0]), slice(0, H // G)
    assert np.isnan(o[rows, heads]).all() and np.isnan(lse[rows, heads]).all()
    ref["o"][rows, heads] = ref["lse"][rows, heads] = np.nan
    check(o, ref["o"], ref["o_tol"], "o")
    check(lse, ref["lse"], ref["lse_tol"], "lse")


def exact_case(d, dtype, hd, H, G, m, n, causal, q0, k0, v, scale):
    """One sequence whose queries and keys have their first element alone: q0 [m], k0 [n], the same in every head; v [n][hd]."""
    q, k, vv = np.zeros((m, H, hd)), np.zeros((n, G, hd)), np.repeat(v[:, None], G, 1)
    q[:, :, 0], k[:, :, 0] = np.asarray(q0)[:, None], np.asarray(k0)[:, None]
    assert np.array_equal(q, stored(q, dtype)) and np.array_equal(k, stored(k, dtype)) and np.array_equal(vv, stored(vv, dtype))
    tq, tk, tv = (to_dev(x, dtype) for x in (q, k, vv))
    o, lse = torch.zeros_like(tq), torch.zeros((m, H), device="cuda")
    cfg = d.packed_config(tq, tk, tv, o, 1, causal, scale, max_q=m)
    ws = d.workspace(d.packed_attention_workspace_bytes(cfg)).fill_(255)
    d.packed_attention(cfg, tq, tk, tv, o, lse=lse, ws=ws)
    torch.cuda.synchronize()
    ref = attention_reference(q, k, vv, [0, m], [0, n], [n], scale, causal, dtype)
    Pr = UNIT["bf16"] if dtype == "bf16" else 0.0
    top = np.abs(vv).max()
    tol = UNIT[dtype] * np.abs(ref["o"]) + (Pr + (n + 8) * F32) * top
    check(host64(o), ref["o"], tol, "o")
    check(lse.double().cpu().numpy(), ref["lse"], 2.0 ** -21 * (np.abs(np.where(np.isfinite(ref["lse"]), ref["lse"], 0.0)) + 8), "lse")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("H,G,m,n", [(8, 2, 1, 2100), (2, 1, 40, 3000), (8, 2, 1, 300)])
def test_parts_keep_their_weights_at_large_scores(d, H, G, m, n, hd, dtype):
    """Equal scores of 2^18, whose lse is known to 2^-6 only: o is the mean of v, whose parts have unlike means."""
    v = stored(np.repeat((np.arange(n) / n)[:, None], hd, 1), dtype)
    exact_case(d, dtype, hd, H, G, m, n, False, np.full(m, 2.0 ** 9), np.full(n, 2.0 ** 9), v, 1.0)


LARGE = [2.0 ** 17, -2.0 ** 17, 2.0 ** 22, -2.0 ** 22, 2.0 ** 33, -2.0 ** 33, 2.0 ** 80, -2.0 ** 80, 2.0 ** 123, -2.0 ** 123, 2.0 ** 125,
         -2.0 ** 125]
# H, G, queries, keys, causal: few rows and wide tiles, one key, whole and in parts, rows that see nothing, enough tiles for 64 fp32 rows
PLACES = [(8, 2, 1, 1, False), (8, 2, 1, 150, False), (8, 2, 1, 2000, False), (2, 1, 40, 1, False), (2, 1, 40, 77, True), (2, 1, 40, 20, True),
          (2, 1, 40, 3000, False), (16, 16, 2112, 3, False)]


@pytest.mark.parametrize("dtype,hd", [("bf16", 64), ("bf16", 128), ("f32", 64), ("f32", 128)])
@pytest.mark.parametrize("H,G,m,n,causal", PLACES)
def test_large_scores_have_the_softmax_of_their_differences(d, H, G, m, n, causal, dtype, hd):
    """Equal scores weigh the same; one that is 2^-7 of their size above the others is all that counts."""
    v = stored(np.random.default_rng(n).standard_normal((n, hd)), dtype)
    for s in LARGE:
        q0 = np.full(m, np.copysign(2.0 ** 60, s))
        k0 = np.full(n, abs(s) * 2.0 ** -59)
        exact_case(d, dtype, hd, H, G, m, n, causal, q0, k0, v, 0.5)
        for at in {0, n // 2, n - 1}:
            k1 = k0.copy()
            if s > 0:
                k1[at] *= 1 + 2.0 ** -7
            else:
                k1 *= 1 + 2.0 ** -7
                k1[at] = k0[at]
            exact_case(d, dtype, hd, H, G, m, n, causal, q0, k1, v, 0.5)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,G,m,n", [(8, 2, 1, 2000), (2, 1, 40, 600), (2, 1, 40, 3000)])
def test_scores_that_grow_along_the_keys(d, H, G, m, n, dtype):
    """From ordinary ones to 2^40, and rows of ordinary scores beside rows of large ones."""
    v = stored(np.random.default_rng(n).standard_normal((n, 64)), dtype)
    k0 = 2.0 ** (np.arange(n) * 40 // n)
    for k in (k0, -k0, k0[::-1], -k0[::-1]):
        exact_case(d, dtype, 64, H, G, m, n, False, np.ones(m), k, v, 1.0)
        exact_case(d, dtype, 64, H, G, m, n, True, np.where(np.arange(m) % 3, 2.0 ** -40, 1.0), k, v, 1.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,G,m,n", [(8, 2, 1, 300), (2, 1, 40, 300), (2, 1, 40, 3000)])
def test_neighbouring_large_scores_keep_their_ratio(d, H, G, m, n, dtype):
    """Scores of a whole number near 726817 (2^20 in log2 units) and of one more: weights of e^-1 and 1, to the bound."""
    q, k = np.zeros((m, H, 64)), np.zeros((n, G, 64))
    q[:, :, :3] = 1.0
    k[:, :, 0], k[:, :, 1] = 704 * 1024, 5888
    k[:, :, 2] = 33 + (np.arange(n)[:, None] >= n // 2)
    v = stored(np.random.default_rng(n).standard_normal((n, G, 64)), dtype)
    tq, tk, tv = (to_dev(x, dtype) for x in (q, k, v))
    o, lse = torch.zeros_like(tq), torch.zeros((m, H), device="cuda")
    cfg = d.packed_config(tq, tk, tv, o, 1, False, 1.0, max_q=m)
    ws = d.workspace(d.packed_attention_workspace_bytes(cfg)).fill_(255)
    d.packed_attention(cfg, tq, tk, tv, o, lse=lse, ws=ws)
    ref = attention_reference(q, k, v, [0, m], [0, n], [n], 1.0, False, dtype)
    tol = UNIT[dtype] * np.abs(ref["o"]) + ((UNIT["bf16"] if dtype == "bf16" else 0.0) + (n + 8) * F32) * np.abs(v).max()
    check(host64(o), ref["o"], tol, "o")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,G,m,n", [(8, 2, 1, 150), (8, 2, 1, 2000), (2, 1, 40, 70), (2, 1, 40, 3000)])
def test_scores_of_minus_infinity_are_not_an_empty_row(d, H, G, m, n, dtype):
    """A row whose scores all overflow has no softmax: NaN, not the zeros of a row that sees no key."""
    q, k = np.full((m, H, 64), 2.0 ** 100), np.full((n, G, 64), -2.0 ** 100)
    tq, tk = to_dev(q, dtype), to_dev(k, dtype)
    o, lse = torch.zeros_like(tq), torch.zeros((m, H), device="cuda")
    cfg = d.packed_config(tq, tk, tk, o, 1, False, 1.0, max_q=m)
    ws = d.workspace(d.packed_attention_workspace_bytes(cfg)).fill_(255)
    d.packed_attention(cfg, tq, tk, tk, o, lse=lse, ws=ws)
    assert torch.isnan(o).all() and torch.isneginf(lse).all()


@pytest.mark.parametrize("H,G,hd,m", [(4, 2, 64, 70), (2, 1, 128, 33), (16, 16, 64, 2112), (8, 8, 128, 2112)])
def test_fp32_gradients_take_the_difference_from_lse_first(d, H, G, hd, m):
    """Whole scores from 4096 on, exact in every kernel, in tiles of 16 and of 64. With e the given lse, p = exp(s - e) is off by 2^-20:
    s - e is exact (within a factor of two of each other), |s - e| < 10 goes to the base 2 with 2^-24 of itself, twice, and the
    exponential by 2^-23. The rest is tests/policy_util.py's."""
    rng = np.random.default_rng(m)
    scale, n = 0.125, m
    q, k = np.zeros((m, hd)), np.zeros((n, hd))
    q[:, 0], k[:, 0] = 256.0, 128 + rng.integers(0, 6, n) / 32
    v, do = (stored(rng.standard_normal((m, h, hd)), "f32") for h in (G, H))
    o, lse = np.zeros((m, H, hd)), np.zeros((m, H))
    for j in range(H):
        o[:, j], lse[:, j], _ = P.attention(q, k, v[:, j // (H // G)], scale, True)
    o, lse = stored(o, "f32"), stored(lse, "f32")
    tq, tk = (to_dev(np.repeat(x[:, None], h, 1), "f32") for x, h in ((q, H), (k, G)))
    tv, to, tdo = (to_dev(x, "f32") for x in (v, o, do))
    dq, dk, dv = (torch.zeros_like(t) for t in (tq, tk, tv))
    cfg = d.packed_config(tq, tk, tv, to, 1, True, scale, max_q=m)
    ws = d.workspace(d.packed_attention_backward_workspace_bytes(cfg)).fill_(255)
    d.packed_attention_backward(cfg, tq, tk, tv, to, torch.from_numpy(lse).float().cuda(), tdo, dq, dk, dv, ws=ws)
    gq, gk, gv = (host64(t) for t in (dq, dk, dv))
    e_p = 2.0 ** -20
    wk, wv, tk_, tv_ = (np.zeros((n, G, hd)) for _ in range(4))
    for j in range(H):
        g = j // (H // G)
        wq, k1, v1, p, ds = P.attention_gradients(q, k, v[:, g], o[:, j], lse[:, j], do[:, j], scale, True)
        e_dp = (hd + 8) * F32 * (np.abs(do[:, j]) @ np.abs(v[:, g]).T + (np.abs(do[:, j]) * np.abs(o[:, j])).sum(1)[:, None])
        b = (e_p + F32 * 8) * np.abs(ds) + p * e_dp
        check(gq[:, j], wq, F32 * np.abs(wq) + scale * (b + n * F32 * np.abs(ds)) @ np.abs(k), "dq")
        wk[:, g] += k1
        wv[:, g] += v1
        tk_[:, g] += scale * (b + m * F32 * np.abs(ds)).T @ np.abs(q)
        tv_[:, g] += ((e_p + m * F32) * p).T @ np.abs(do[:, j])
    check(gk, wk, tk_ + F32 * np.abs(wk), "dk")
    check(gv, wv, tv_ + F32 * np.abs(wv), "dv")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kw", [dict(H=2, G=1, q_len=[100, 70], causal=True), dict(H=4, G=4, q_len=[33, 5], k_len=[60, 90])])
def test_gradients_of_large_scores(d, dtype, kw):
    """The bounds of tests/policy_util.py, and what underflow adds to them: a probability below 2^-126, the least number the exponential
    gives, is 0, and so is such a ds = p (dp - delta). That is off by at most t = 2^-126 (1 + |dp| + |delta|), which the products carry
    into at most rows t scale |q| of dk, keys t scale |k| of dq and rows 2^-126 |do| of dv."""
    p = Problem(d, dtype, 64, seed=7, q_gain=40.0, **kw)
    grads = p.backward()
    ref = attention_reference(p.q, p.k, p.v, p.q_off, p.k_off, p.k_len, p.scale, p.causal, dtype, p.do, p.o64, p.lse64)
    t = 2.0 ** -126 * (1 + np.nanmax(np.abs(p.do).sum(2)) * (np.nanmax(np.abs(p.v)) + np.nanmax(np.abs(p.o64))))
    rows = max(p.q_len) * p.q.shape[1] // p.k.shape[1]
    tiny = {"dq": max(p.k_len) * t * p.scale * np.nanmax(np.abs(p.k)), "dk": rows * t * p.scale * np.nanmax(np.abs(p.q)),
            "dv": rows * 2.0 ** -126 * np.nanmax(np.abs(p.do))}
    for n, g in zip(("dq", "dk", "dv"), grads):
        check(host64(g.contiguous()), ref[n], ref[n + "_tol"] + tiny[n], n)


@pytest.mark.parametrize("dtype,hd", [("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("count", [60, 130, 600])
def test_few_long_caches_among_many_short_ones(d, count, dtype, hd):
    """The partial results of the long ones lie together, whatever is before and between them; new tokens of none, one and two."""
    rng = np.random.default_rng(count)
    keys = rng.integers(0, 90, count)
    keys[[0, 3, count // 2, count - 3, count - 2]] = [4000, 5100, 2500, 8111, 3000]
    new = rng.integers(0, 3, count)
    new[[0, 3, count // 2, count - 3, count - 2]] = [1, 0, 2, 1, 2]
    p = Problem(d, dtype, hd, 8, 2, new, keys, True, slack=1, lead=2, tail=1, seed=count)
    assert d.packed_attention_workspace_bytes(p.cfg) > 0
    p.check_forward()


@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
@pytest.mark.parametrize("dtype,hd", [("bf16", 64), ("bf16", 128), ("f32", 64), ("f32", 128)])
@pytest.mark.parametrize("H,G,m,n", [(2, 1, 8, 5), (2, 1, 120, 70), (2, 1, 3050, 3000), (16, 16, 2112, 40)])
def test_rows_that_see_no_key_are_empty_whatever_the_keys_hold(d, H, G, m, n, dtype, hd, bad):
    """The first m - n of m causal queries: o = 0, lse = -inf and dq = 0, beside queries that see keys and values of no number."""
    p = Problem(d, dtype, hd, H, G, [m], [n], True, layout="plain", seed=m)
    p.tk[0], p.tv[0] = bad, bad
    o, lse = p.forward()
    assert np.all(o[:m - n] == 0.0) and np.all(np.isneginf(lse[:m - n]))
    assert np.isnan(o[m - n:]).all()
    dq = p.backward()[0]
    assert bool((dq[:m - n] == 0.0).all())
