"""int8_matmul and int8_linear against the oracle.

The sum is exact. It is rounded to fp32, multiplied twice and added to the bias: four roundings of 2^-24 of the product (and of
the bias once), then one to y's type. gelu_tanh is z sigmoid(2u) with 2u = z (c + d z^2) in fp32: its argument is off by at most
5 roundings of |2u| (absolute in the exponent, so relative in the exponential), the exponential, sum, reciprocal and product
by at most 2, 1, 2 and 1 more units; what z is off by counts by the slope, at most 1.13."""
import numpy as np
import pytest
import torch

from oracle import update_oracle as U
from tests.gpu_util import host64
from tests.policy_util import F32, UNIT
from tests.test_gpu_policy_guards import Guarded

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def d():
    from paper_2606_19004_amd import ditstep
    return ditstep


def bound(total, xs, ws, bias, y, gelu, dtype):
    z = total * xs[:, None] * ws[None, :]
    e = 4 * F32 * np.abs(z) + (F32 * np.abs(z + bias) if bias is not None else 0.0)
    if gelu:
        z = z if bias is None else z + bias
        u2 = 2 * np.sqrt(2 / np.pi) * np.abs(z + 0.044715 * z ** 3)
        e = 1.13 * e + np.abs(y) * (5 * u2 + 12) * F32
    return e + UNIT[dtype] * (np.abs(y) + e) + 2.0 ** -125


def int8_tensor(m, rows, cols, pad, rng, low=-127):
    """Rows at a stride of `pad` bytes more than they need, with other numbers in what lies between them."""
    row = -(-cols // 16) * 16 + pad
    t = m.empty(rows, row, dtype=torch.int8)
    t.copy_(torch.from_numpy(rng.integers(-128, 128, (rows, row)).astype(np.int8)))
    t[:, :cols] = torch.from_numpy(rng.integers(low, 128, (rows, cols)).astype(np.int8)).cuda()
    return t[:, :cols]


class Problem:
    def __init__(self, d, M, K, N, dtype, gelu=False, bias=True, pad=0, ypad=0, low=-127):
        self.d, self.m, self.dtype, self.gelu = d, Guarded(), dtype, gelu
        rng = np.random.default_rng(M * 7 + K * 3 + N)
        m, t = self.m, TYPES[dtype]
        self.x, self.w = int8_tensor(m, M, K, pad, rng, low), int8_tensor(m, N, K, 2 * pad, rng, low)
        self.xs = torch.from_numpy(np.exp(rng.normal(size=M)).astype(np.float32) / np.float32(100 * np.sqrt(K))).cuda()
        self.ws = torch.from_numpy(np.exp(rng.normal(size=N)).astype(np.float32) / np.float32(60)).cuda()
        self.bias = torch.from_numpy(rng.normal(size=N).astype(np.float32)).cuda().to(t) if bias else None
        self.full = m.empty(M, N + ypad, dtype=t)
        self.y = self.full[:, :N]
        self.cfg = d.int8_config(self.x, self.w, self.y, act="gelu" if gelu else "none")
        self.ws_bytes = m.empty(max(d.int8_matmul_workspace_bytes(self.cfg), 1), dtype=torch.uint8)

    def run(self):
        self.d.int8_matmul(self.cfg, self.x, self.xs, self.w, self.ws, self.y, bias=self.bias, ws=self.ws_bytes)

    def check(self):
        hole = self.full[:, self.y.shape[1]:].clone()
        self.run()
        self.m.check()
        assert torch.equal(self.full[:, self.y.shape[1]:].view(torch.int8), hole.view(torch.int8))
        b = None if self.bias is None else host64(self.bias)
        xs, ws = host64(self.xs), host64(self.ws)
        want, total = U.int8_matmul(self.x.cpu().numpy(), xs, self.w.cpu().numpy(), ws, b, self.gelu)
        off = np.abs(host64(self.y) - want) - bound(total, xs, ws, b, want, self.gelu, self.dtype)
        assert off.max() <= 0, off.max()


SIZES = [(1, 1, 1), (1, 16, 16), (1, 5000, 9000), (2, 1024, 4200), (2, 1025, 77), (4, 3000, 8200), (6, 4097, 40), (8, 2048, 8300), (8, 7680, 21), (8, 7681, 21), (9, 640, 50), (1, 100, 3), (2, 17, 5), (1, 3072, 640), (3, 128, 64), (5, 129, 65), (16, 1000, 100), (17, 64, 33), (31, 255, 127),
         (33, 333, 129), (64, 512, 64), (65, 127, 257), (100, 2050, 48), (127, 384, 130), (128, 256, 128), (129, 640, 513), (255, 1001, 515),
         (256, 768, 256), (300, 4096, 320), (520, 300, 1030), (1000, 160, 72), (1300, 90, 700)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,K,N", SIZES)
def test_sizes(d, M, K, N, dtype):
    Problem(d, M, K, N, dtype, gelu=(M + N) % 2 == 0, bias=M % 3 != 0).check()


# every form at sizes that do not fill its tiles: one k-tile, two, three, and more than its stages, rows of w that end inside 16 bytes
FORMS = [("few rows", 1, 61440, 50), ("few rows", 2, 30720, 9), ("few rows", 2, 2049, 8210), ("32, shared k", 1, 61441, 50), ("32, shared k", 3, 700, 9000),
         ("32, shared k", 190, 3001, 2100), ("64, shared k", 250, 12001, 3001), ("64", 300, 2001, 4000), ("64", 513, 260, 11665), ("64", 4100, 130, 4100),
         ("128", 333, 3001, 9215), ("128", 1427, 1120, 2271), ("128", 1959, 72, 1734), ("128", 2478, 131, 1471), ("128", 2642, 365, 1396),
         ("128", 942, 505, 3198), ("128", 527, 566, 5683), ("128", 1477, 732, 2335), ("256 x 192", 7000, 131, 8001), ("256 x 192", 1401, 315, 6787),
         ("256 x 192", 2807, 2847, 8364), ("256 x 256", 9003, 90, 3001), ("256 x 256", 5000, 200, 2500), ("256 x 256", 4000, 333, 8009), ("256 x 256", 7901, 639, 6935)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("form,M,K,N", FORMS)
def test_every_form(d, form, M, K, N, dtype):
    from tests.int8_util import int8_form
    assert int8_form(M, K, N) == form
    Problem(d, M, K, N, dtype, gelu=K % 2 == 0, bias=M % 2 == 1, pad=16 * (N % 2), ypad=3 * (M % 2)).check()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,K,N", [(1, 200, 30), (7, 47, 19), (40, 1100, 70), (200, 130, 300), (700, 333, 260)])
def test_strides_and_what_lies_between_rows(d, M, K, N, dtype):
    Problem(d, M, K, N, dtype, pad=48, ypad=5).check()
    Problem(d, M, K, N, dtype, pad=16, ypad=8, gelu=True).check()


@pytest.mark.parametrize("M", [1, 30, 200])
def test_longest_rows_of_the_largest_numbers(d, M):
    """in_features 131071 with nothing but -128: a sum of 2^31 - 2^14."""
    p = Problem(d, M, 131071, 33, "f32", bias=False, pad=16)
    p.x.fill_(-128)
    p.w.fill_(-128)
    p.check()
    p.w[1].fill_(127)
    p.w[2, ::2] = 127
    p.check()


@pytest.mark.parametrize("M", [1, 9, 150])
def test_scales_that_are_not_finite(d, M):
    p = Problem(d, M, 96, 40, "bf16")
    p.check()
    want = p.y.clone()
    p.xs[M // 2], p.ws[7] = float("nan"), float("nan")
    p.run()
    hit = torch.zeros(M, 40, dtype=torch.bool, device="cuda")
    hit[M // 2], hit[:, 7] = True, True
    assert torch.isnan(p.y[hit].float()).all() and torch.equal(p.y[~hit], want[~hit])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,K,N,act", [(1, 3072, 384, "none"), (1, 16384, 40, "none"), (1, 16385, 40, "gelu"), (1, 3000, 9000, "gelu"), (2, 8191, 8300, "none"), (2, 8192, 50, "none"), (2, 8193, 50, "none"), (1, 5, 3, "none"), (2, 8, 2, "none"),
                                       (33, 512, 70, "gelu"), (500, 511, 1000, "none"), (64, 9, 40, "none"), (3, 130, 16384, "gelu"), (3, 130, 16416, "none"),
                                       (100, 256, 100, "none"), (47, 257, 33, "gelu"), (5, 128, 31, "none"), (300, 1, 20, "none"), (2, 8192, 33, "gelu"), (3, 4096, 8200, "none"),
                                       (3, 5461, 9, "gelu"), (4, 4096, 20, "none"), (8, 2048, 8210, "gelu"), (7, 1033, 50, "none"), (8, 2049, 30, "none"), (1, 77, 9, "gelu"), (4, 1000, 100, "gelu"), (20, 513, 70, "none"), (130, 2049, 257, "gelu"),
                                       (300, 20000, 33, "none"), (600, 256, 512, "gelu")])
def test_linear_is_the_product_of_rounded_rows(d, M, K, N, act, dtype):
    """Bit for bit, with x at a row stride of its own."""
    m = Guarded()
    x = torch.randn(M, K + 3, device="cuda").to(TYPES[dtype])[:, :K]
    if M > 2:
        x[1, K // 2], x[2] = float("inf"), 0.0
    w, ws = d.int8_rows(N, K), torch.empty(N, device="cuda")
    d.quantize_rows(torch.randn(N, K, device="cuda"), w, ws)
    bias = torch.randn(N, device="cuda").to(x.dtype)
    y, want = m.empty(M, N, dtype=x.dtype), torch.empty(M, N, dtype=x.dtype, device="cuda")
    cfg = d.int8_config(x, w, y, act=act)
    d.int8_linear(cfg, x, w, ws, y, bias=bias, ws=m.empty(d.int8_linear_workspace_bytes(cfg), dtype=torch.uint8))
    m.check()
    q, xs = d.int8_rows(M, K), torch.empty(M, device="cuda")
    d.quantize_rows(x, q, xs)
    cfg = d.int8_config(q, w, want, act=act)
    d.int8_matmul(cfg, q, xs, w, ws, want, bias=bias, ws=d.workspace(d.int8_matmul_workspace_bytes(cfg)))
    assert torch.equal(y.view(torch.int8), want.view(torch.int8))
    if M > 2:
        assert torch.isnan(y[1].float()).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,K,N", [(1, 3072, 9000), (2, 700, 40), (1, 701, 17), (5, 512, 40), (40, 300, 2000), (5, 600, 40), (300, 3000, 70)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_linear_of_a_row_that_is_not_finite(d, M, K, N, bad, dtype):
    """NaN in that row of y, the bits of the rows alone in all others, wherever the value stands; a row of zeros gives the bias."""
    x = torch.randn(M, K, device="cuda").to(TYPES[dtype])
    if M > 2:
        x[2] = 0.0
    w, ws = d.int8_rows(N, K), torch.empty(N, device="cuda")
    d.quantize_rows(torch.randn(N, K, device="cuda"), w, ws)
    bias, y = torch.randn(N, device="cuda").to(x.dtype), torch.empty(M, N, dtype=x.dtype, device="cuda")
    cfg = d.int8_config(x, w, y)
    space = d.workspace(d.int8_linear_workspace_bytes(cfg))
    d.int8_linear(cfg, x, w, ws, y, bias=bias, ws=space)
    want = y.clone()
    assert torch.isfinite(want.float()).all()
    if M > 2:
        assert torch.equal(want[2], bias)
    for row, col in ((M - 1, 0), (0, K - 1), (M // 2, K // 2)):
        kept = x[row, col].clone()
        x[row, col] = bad
        d.int8_linear(cfg, x, w, ws, y, bias=bias, ws=space)
        assert torch.isnan(y[row].float()).all()
        rest = torch.arange(M, device="cuda") != row
        assert torch.equal(y[rest], want[rest])
        x[row, col] = kept


@pytest.mark.parametrize("M,N", [(3, 5), (40, 70), (300, 300)])
def test_offsets_past_32_bits(d, M, N):
    """Rows of x, w and y that start past 2^32 bytes."""
    row = (1 << 23) - 16
    rng = np.random.default_rng(5)
    base = torch.empty(row * 600, dtype=torch.int8, device="cuda")
    w0 = base.as_strided((600, 64), (row, 1))
    w0.copy_(torch.from_numpy(rng.integers(-127, 128, (600, 64)).astype(np.int8)))
    w, x = w0[600 - N:], w0[:M]
    ybase = torch.empty((1 << 22) * M, dtype=torch.float32, device="cuda")
    y = ybase.as_strided((M, N), (1 << 22, 1))
    xs, ws = torch.rand(M, device="cuda") + 0.5, torch.rand(N, device="cuda") + 0.5
    cfg = d.int8_config(x, w, y)
    d.int8_matmul(cfg, x, xs, w, ws, y, ws=d.workspace(d.int8_matmul_workspace_bytes(cfg)))
    a, b = host64(xs), host64(ws)
    want, total = U.int8_matmul(x.cpu().numpy(), a, w.cpu().numpy(), b)
    assert (np.abs(host64(y) - want) <= bound(total, a, b, None, want, False, "f32")).all()


def test_two_streams_at_once(d):
    ps = [Problem(d, M, 1500, 300, "bf16", gelu=True) for M in (150, 9)]
    for p in ps:
        p.run()
    torch.cuda.synchronize()
    want = [p.y.clone() for p in ps]
    streams = [torch.cuda.Stream() for _ in ps]
    for _ in range(5):
        for p, s in zip(ps, streams):
            with torch.cuda.stream(s):
                p.y.zero_()
                p.run()
        torch.cuda.synchronize()
        assert all(torch.equal(p.y, w) for p, w in zip(ps, want))
