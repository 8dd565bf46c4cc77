"""A product of more than 2^34 results, which runs in the tiles that its form has."""
import numpy as np
import pytest
import torch

from oracle import update_oracle as U
from tests.gpu_util import host64
from tests.test_gpu_int8_matmul import bound

pytestmark = pytest.mark.gpu


def test_more_than_2_34_results():
    from paper_2606_19004_amd import ditstep as d
    M, K, N = 1_500_001, 20, 12291
    g = torch.Generator(device="cuda").manual_seed(4)
    x, w = d.int8_rows(M, K), d.int8_rows(N, K)
    for t in (x, w):
        t.copy_(torch.randint(-127, 128, t.shape, generator=g, device="cuda", dtype=torch.int8))
    xs, ws = (torch.rand(n, generator=g, device="cuda") / 100 + 0.005 for n in (M, N))
    y = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
    cfg = d.int8_config(x, w, y)
    d.int8_matmul(cfg, x, xs, w, ws, y, ws=d.workspace(d.int8_matmul_workspace_bytes(cfg)))
    for rows in (slice(0, 300), slice(349_500, 349_700), slice(M // 2, M // 2 + 300), slice(M - 300, M)):   # (row 349 525: past 2^32 elements)
        a, b = host64(xs[rows]), host64(ws)
        want, total = U.int8_matmul(x[rows].cpu().numpy(), a, w.cpu().numpy(), b)
        assert (np.abs(host64(y[rows]) - want) <= bound(total, a, b, None, want, False, "bf16")).all()


def test_two_rows_of_more_features_than_dot_products_take():
    """2^28 features and some: tiles take them, also where int8_linear would round short rows in the product's launch."""
    from paper_2606_19004_amd import ditstep as d
    M, K, N = 2, 10, (1 << 28) + 37
    g = torch.Generator(device="cuda").manual_seed(5)
    w = d.int8_rows(N, K)
    w.copy_(torch.arange(N * K, device="cuda").remainder_(251).sub_(125).view(N, K))
    x, ws = torch.randn(M, K, generator=g, device="cuda").bfloat16(), torch.rand(N, generator=g, device="cuda") / 100 + 0.005
    q, xs = d.int8_rows(M, K), torch.empty(M, device="cuda")
    d.quantize_rows(x, q, xs)
    y, again = (torch.empty(M, N, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    cfg = d.int8_config(q, w, y)
    d.int8_matmul(cfg, q, xs, w, ws, y, ws=d.workspace(d.int8_matmul_workspace_bytes(cfg)))
    cfg = d.int8_config(x, w, again)
    d.int8_linear(cfg, x, w, ws, again, ws=d.workspace(d.int8_linear_workspace_bytes(cfg)))
    assert torch.equal(y, again)
    a, iq = host64(xs), q.cpu().numpy()
    for cols in (slice(0, 5000), slice(N // 2, N // 2 + 5000), slice(N - 5000, N)):
        b = host64(ws[cols])
        want, total = U.int8_matmul(iq, a, w[cols].cpu().numpy(), b)
        assert (np.abs(host64(y[:, cols]) - want) <= bound(total, a, b, None, want, False, "bf16")).all()
