"""packed_attention at values where a softmax goes wrong first: a NaN in a used row, and scores so large that what is left of a
difference of two of them has to be exact.

The scores of the second kind are products of powers of two, so they are exact in every kernel and the bounds hold no error of
theirs: o is off by U |o| + (P + (n + 8) 2^-24) sum p |v| (U, P: tests/policy_util.py), lse by 2^-21 of its size."""
import numpy as np
import pytest
import torch

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
