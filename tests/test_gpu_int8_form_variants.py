"""Every form of the 8-bit product with and without gelu and bias, in both types, at one k-tile, two, three, four and more where the rule picks it there;
and int8_linear's two launches into each form. The bounds are those of test_gpu_int8_matmul."""
import numpy as np
import pytest
import torch

from oracle import update_oracle as U
from tests.gpu_util import host64
from tests.int8_util import int8_form
from tests.test_gpu_int8_matmul import TYPES, Problem, bound
from tests.test_gpu_policy_guards import Guarded

pytestmark = pytest.mark.gpu
SIZES = [("few rows", 1, 300, 70), ("few rows", 2, 5000, 130), ("32, shared k", 65, 2, 8197), ("32, shared k", 40, 1300, 70), ("64, shared k", 4, 19, 16),
         ("64, shared k", 4, 135, 16), ("64, shared k", 33, 884, 8746), ("64", 5758, 36, 129), ("64", 8506, 170, 65), ("64", 67, 265, 8206), ("64", 8851, 414, 65),
         ("64", 66, 580, 8371), ("128", 195, 5, 8135), ("128", 199, 146, 9419), ("128", 334, 268, 6932), ("128", 9068, 389, 269), ("128", 7854, 538, 322),
         ("128", 321, 819, 8308), ("256 x 192", 642, 2, 9846), ("256 x 192", 5442, 175, 1283), ("256 x 192", 1238, 261, 5975), ("256 x 192", 4554, 395, 1695),
         ("256 x 192", 3258, 644, 2574), ("256 x 256", 1029, 6, 9892), ("256 x 256", 1306, 162, 8148), ("256 x 256", 9244, 264, 1191), ("256 x 256", 1157, 387, 9864),
         ("256 x 256", 6469, 669, 1731), ("256 x 256", 1369, 773, 8192)]


@pytest.fixture(scope="module")
def d():
    from paper_2606_19004_amd import ditstep
    return ditstep


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("gelu", [False, True])
@pytest.mark.parametrize("form,M,K,N", SIZES)
def test_products(d, form, M, K, N, gelu, dtype):
    assert int8_form(M, K, N) == form
    Problem(d, M, K, N, dtype, gelu=gelu, bias=(M + K + gelu) % 2 == 0, ypad=N % 2).check()


LINEAR = [("few rows", 2, 9000, 40), ("32, shared k", 65, 2, 8197), ("32, shared k", 40, 1300, 70), ("64, shared k", 33, 884, 8746), ("64", 8506, 170, 65),
          ("64", 66, 580, 8371), ("128", 9068, 389, 269), ("128", 321, 819, 8308), ("256 x 192", 5442, 175, 1283), ("256 x 192", 3258, 644, 2574),
          ("256 x 256", 1306, 162, 8148), ("256 x 256", 1369, 773, 8192)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("act", ["none", "gelu"])
@pytest.mark.parametrize("form,M,K,N", LINEAR)
def test_linear_in_two_launches(d, form, M, K, N, act, dtype):
    """Against the oracle's integers and their product, and the bits of int8_matmul of the rounded rows."""
    assert int8_form(M, K, N) == form
    m, rng = Guarded(), np.random.default_rng(M + K + N)
    x = torch.randn(M, K + 3, device="cuda").to(TYPES[dtype])[:, :K]
    x[0] = 0.0
    w = d.int8_rows(N, K).copy_(torch.from_numpy(rng.integers(-127, 128, (N, K)).astype(np.int8)))
    ws = torch.from_numpy(np.exp(rng.normal(size=N)).astype(np.float32) / np.float32(60 * np.sqrt(K))).cuda()
    bias = torch.randn(N, device="cuda").to(x.dtype)
    y, again = m.empty(M, N, dtype=x.dtype), torch.empty(M, N, dtype=x.dtype, device="cuda")
    cfg = d.int8_config(x, w, y, act=act)
    need = d.int8_linear_workspace_bytes(cfg)
    assert need > 0   # two launches
    d.int8_linear(cfg, x, w, ws, y, bias=bias, ws=m.empty(need, dtype=torch.uint8))
    m.check()
    q, xs = U.quantize_rows(host64(x))
    want, total = U.int8_matmul(q, xs, w.cpu().numpy(), host64(ws), host64(bias), act == "gelu")
    assert (np.abs(host64(y) - want) <= bound(total, xs, host64(ws), host64(bias), want, act == "gelu", dtype)).all()
    qd, sd = d.int8_rows(M, K), torch.empty(M, device="cuda")
    d.quantize_rows(x, qd, sd)
    cfg = d.int8_config(qd, w, again, act=act)
    d.int8_matmul(cfg, qd, sd, w, ws, again, bias=bias, ws=d.workspace(d.int8_matmul_workspace_bytes(cfg)))
    assert torch.equal(y.view(torch.int8), again.view(torch.int8))
