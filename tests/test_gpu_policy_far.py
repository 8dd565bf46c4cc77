"""Rows so far apart that their offsets pass 32 bits, at the largest row stride that attention takes, in every kind of kernel."""
import numpy as np
import pytest
import torch

from oracle import policy_oracle as P
from tests.gpu_util import host64
from tests.policy_util import F32, UNIT, attention_reference, check, stored, to_dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def d():
    from paper_2606_19004_amd import ditstep
    return ditstep


def far(rows, heads, hd, row, dtype, x=None, at=0, store=None):
    """[rows][heads][hd] at row stride `row`, `at` elements into a store; only those elements are ever touched."""
    if store is None:
        store = torch.empty(rows * row + 8192, dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, device="cuda")
    t = store.as_strided((rows, heads, hd), (row, hd, 1), at)
    if x is not None:
        t.copy_(to_dev(x, dtype))
    return t, store


# H, G, queries: a few rows, and wide tiles
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,G,m", [(4, 2, 3), (4, 2, 150)])
def test_attention(d, H, G, m, dtype):
    n, hd, row = 150, 128, (1 << 24) - 8           # 150 rows of 32 or 64 MiB
    rng = np.random.default_rng(m)
    q, k, v, do = (stored(rng.standard_normal((r, h, hd)), dtype) for r, h in ((m, H), (n, G), (n, G), (m, H)))
    tk, store = far(n, G, hd, row, dtype, k)
    tv, _ = far(n, G, hd, row, dtype, v, 2048, store)
    tq, _ = far(m, H, hd, row, dtype, q, 4096, store)
    o, _ = far(m, H, hd, row, dtype)
    lse = torch.zeros((m, H), device="cuda")
    cfg = d.packed_config(tq, tk, tv, o, 1, True, 0.125, max_q=m)
    ws = d.workspace(d.packed_attention_workspace_bytes(cfg))
    d.packed_attention(cfg, tq, tk, tv, o, lse=lse, ws=ws)
    ref = attention_reference(q, k, v, [0, m], [0, n], [n], 0.125, True, dtype)
    check(host64(o.contiguous()), ref["o"], ref["o_tol"], "o")
    check(lse.double().cpu().numpy(), ref["lse"], ref["lse_tol"], "lse")
    o64, lse64 = stored(ref["o"], dtype), stored(ref["lse"], "f32")
    o.copy_(to_dev(o64, dtype))
    tdo, _ = far(m, H, hd, row, dtype, do)
    dk, gs = far(n, G, hd, row, dtype)
    dv, _ = far(n, G, hd, row, dtype, None, 2048, gs)
    dq, _ = far(m, H, hd, row, dtype, None, 4096, gs)
    ws = d.workspace(d.packed_attention_backward_workspace_bytes(cfg))
    d.packed_attention_backward(cfg, tq, tk, tv, o, to_dev(lse64, "f32"), tdo, dq, dk, dv, ws=ws)
    ref = attention_reference(q, k, v, [0, m], [0, n], [n], 0.125, True, dtype, do, o64, lse64)
    for name, t in (("dq", dq), ("dk", dk), ("dv", dv)):
        check(host64(t.contiguous()), ref[name], ref[name + "_tol"], name)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 520])
def test_gated_norm(d, D, dtype):
    """Bounds as in tests/test_gpu_gated_norm.py, without a branch: x_out = x, h its normalised row."""
    rows, row, eps = 300, 1 << 23, 1e-5
    rng = np.random.default_rng(D)
    x, dh = (stored(rng.standard_normal((rows, 1, D)), dtype) for _ in range(2))
    tx, store = far(rows, 1, D, row, dtype, x)
    th, _ = far(rows, 1, D, row, dtype, None, 2048, store)
    tdh, gstore = far(rows, 1, D, row, dtype, dh)
    tdx, _ = far(rows, 1, D, row, dtype, None, 2048, gstore)
    tx, th, tdh, tdx = (t[:, 0] for t in (tx, th, tdh, tdx))
    cfg = d.gated_norm_config(tx, 3, "none", "rms", eps)
    d.gated_norm(cfg, tx, None, None, th)
    K = (D / 64 + 16) * F32
    hat, r = P.norm("rms", x[:, 0], eps)
    e = 4 * K * (np.abs(hat) + 1)
    check(host64(th.contiguous()), hat, UNIT[dtype] * np.abs(hat) + e + 8 * F32 * np.abs(hat), "h")
    d.gated_norm_backward(cfg, tx, None, None, tdh, tdx, None, ws=d.workspace(d.gated_norm_backward_workspace_bytes(cfg)))
    want = P.norm_gradient("rms", hat, r, dh[:, 0])
    g = np.abs(dh[:, 0])
    size = g + np.abs(hat) * (g * np.abs(hat)).mean(1, keepdims=True)
    e = e * (g * np.abs(hat)).mean(1, keepdims=True) + np.abs(hat) * (g * e).mean(1, keepdims=True)
    check(host64(tdx.contiguous()), want, UNIT[dtype] * np.abs(want) + r * (e + 8 * K * 2 * size), "dx")
