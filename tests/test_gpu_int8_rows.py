"""quantize_rows against the oracle, integers, scales and values bit for bit."""
import numpy as np
import pytest
import torch

from oracle import update_oracle as U
from tests.gpu_util import host64
from tests.test_gpu_policy_guards import Guarded

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def d():
    from paper_2606_19004_amd import ditstep
    return ditstep


def check(d, x, q, scale, values):
    d.quantize_rows(x, q, scale, values=values)
    torch.cuda.synchronize()
    want_q, want_s = U.quantize_rows(host64(x) if values is not x else check.before)
    assert np.array_equal(q.cpu().numpy().astype(np.int64), want_q)
    assert np.array_equal(host64(scale), want_s, equal_nan=True)
    if values is not None:   # the product is rounded to fp32, then to the type
        want = torch.from_numpy(np.where(np.isnan(want_s)[:, None], np.nan, want_q * want_s[:, None])).float().to(x.dtype)
        assert np.array_equal(host64(values), host64(want), equal_nan=True)


def tensors(m, rows, cols, pad, dtype):
    """x, q, scale, values with row strides of cols + pad between guard bands."""
    cut = lambda t: t[:, :cols]  # noqa: E731
    return (cut(m.empty(rows, cols + pad, dtype=dtype)), cut(m.empty(rows, cols + 2 * pad, dtype=torch.int8)), m.empty(rows, dtype=torch.float32),
            cut(m.empty(rows, cols + pad, dtype=dtype)))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 0), (3, 7, 0), (5, 8, 3), (1, 12288, 0), (2, 511, 1), (7, 512, 0), (130, 513, 0), (9, 1024, 5), (6, 1025, 0),
                                           (4, 2047, 0), (300, 2048, 0), (3, 2056, 8), (3, 4096, 0), (2, 4099, 2), (5, 8192, 0), (2, 8200, 0), (3, 16384, 0),
                                           (2, 16385, 1), (3, 40003, 0), (70000, 24, 0)])
def test_rows(d, rows, cols, pad, dtype):
    m = Guarded()
    x, q, scale, values = tensors(m, rows, cols, pad, TYPES[dtype])
    g = torch.Generator(device="cuda").manual_seed(rows + cols)
    x.copy_(torch.randn(rows, cols, generator=g, device="cuda") * torch.exp(4 * torch.randn(rows, 1, generator=g, device="cuda")))
    gaps = [t.untyped_storage() for t in (q, values)]
    before = [torch.tensor([], dtype=torch.uint8, device="cuda").set_(s).clone() for s in gaps]
    check(d, x, q, scale, values)
    m.check()
    if pad:   # what lies between the rows is as it was
        for t, s, b in zip((q, values), gaps, before):
            now = torch.tensor([], dtype=torch.uint8, device="cuda").set_(s)
            es, hole = t.element_size(), t.stride(0) - cols
            rest = lambda u: u[4096:4096 + rows * t.stride(0) * es].view(rows, t.stride(0) * es)[:, cols * es:]  # noqa: E731
            assert hole > 0 and torch.equal(rest(now), rest(b))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [40, 700, 3000, 6000, 12000, 20000])
def test_rows_of_extreme_values(d, cols, dtype):
    """Zeros, NaN and infinities anywhere, the largest and smallest numbers, halves exactly and next to them."""
    t = TYPES[dtype]
    big = float(torch.finfo(t).max)
    x = torch.zeros(14, cols)
    x[1, cols - 1] = float("nan")
    x[2, 0], x[2, 1] = float("inf"), 3.0
    x[3, cols // 2], x[3, 0] = float("-inf"), float("nan")
    x[4] = big
    x[5, ::2], x[5, 1::2] = -big, big / 2
    x[6] = 2.0 ** -133                       # subnormal, also in bf16: scale 2^-126
    x[7, 3] = 2.0 ** -119                    # scale 2^-126 by 1.008
    x[8, cols - 1] = -1.0
    k = torch.arange(cols).remainder(254) - 127
    x[9] = (k + 0.5).clamp(-127, 127)        # scale 1: every half is a tie
    x[9, 0] = 127.0
    for r, top in ((10, 0.9), (11, 1.7), (12, 3.3e5)):
        s = np.float32(np.float64(np.float32(top)) / 127)
        h = ((k.numpy() + 0.5) * np.float64(s)).astype(np.float32)
        x[r] = torch.from_numpy(np.where(np.arange(cols) % 3 == 0, h, np.where(np.arange(cols) % 3 == 1, np.nextafter(h, np.float32(9e9)),
                                                                             np.nextafter(h, np.float32(-9e9))))).clamp(-top, top)
        x[r, 0] = top
    x[13] = torch.linspace(-1, 1, cols)
    x = x.to(t).cuda()
    q, scale, values = d.int8_rows(14, cols), torch.empty(14, device="cuda"), torch.empty_like(x)
    check(d, x, q, scale, values)
    assert torch.isnan(values[1:4].float()).all() and not q[1:4].any() and not q[0].any()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [100, 5000, 30000])
def test_values_in_place_and_left_out(d, cols, dtype):
    x = torch.randn(5, cols, device="cuda").to(TYPES[dtype])
    q, scale = d.int8_rows(5, cols), torch.empty(5, device="cuda")
    check(d, x, q, scale, None)
    first = q.clone()
    check.before = host64(x)
    check(d, x, q, scale, x)
    assert torch.equal(q, first)


@pytest.mark.parametrize("shift", [1, 2, 3, 5])
def test_any_alignment(d, shift):
    """x and values at element boundaries, q at any byte, an odd row stride."""
    for t in TYPES.values():
        x = torch.randn(6 * 1001 + shift, device="cuda").to(t)[shift:].view(6, 1001)[:, :999]
        q = torch.empty(6 * 1003 + shift, dtype=torch.int8, device="cuda")[shift:].view(6, 1003)[:, :999]
        values = torch.empty(6 * 1001 + shift, dtype=t, device="cuda")[shift:].view(6, 1001)[:, :999]
        check(d, x, q, torch.empty(6, device="cuda"), values)


def test_offsets_past_32_bits(d):
    """Rows that start past 2^32 bytes (and elements) of their tensors."""
    row = (1 << 30) - 64
    for t in TYPES.values():
        x = torch.empty(5 * row, dtype=t, device="cuda").as_strided((5, 600), (row, 1))
        x.copy_(torch.randn(5, 600, device="cuda"))
        q = torch.empty(5 * row, dtype=torch.int8, device="cuda").as_strided((5, 600), (row, 1))
        check(d, x, q, torch.empty(5, device="cuda"), None)
        del x, q
        torch.cuda.empty_cache()
