"""Rows of very small fp32 numbers: a scale in [2^-126, 2^-125) is a multiple of 2^-149, and half of an odd one is no fp32 number. The integers
have to be the nearest ones there too, bit for bit: of quantize_rows, and of the products that round their rows themselves."""
import numpy as np
import pytest
import torch

from oracle import update_oracle as U
from tests.gpu_util import host64

pytestmark = pytest.mark.gpu
F = np.float32
# (a row's largest value, a value next to a half of its scale, the integer)
KNOWN = [(1.8940565269892005e-36, 2.2370744870125284e-38, 1), (1.8151343212812062e-36, 3.5730992077004776e-38, 3)]


@pytest.fixture(scope="module")
def d():
    from paper_2606_19004_amd import ditstep
    return ditstep


def rows_next_to_halves(rows, cols, seed):
    """Rows whose scales are odd multiples of 2^-149 between 2^-126 and 2^-125, of values at the halves of the scale and on both sides of them."""
    rng = np.random.default_rng(seed)
    units = (1 << 23) + 1 + 2 * rng.integers(0, 1 << 22, rows)
    units[0], units[-1] = (1 << 23) + 1, (1 << 24) - 1
    top = (127.0 * units * 2.0 ** -149).astype(F)
    scale = np.maximum((top.astype(np.float64) / 127).astype(F), F(2.0 ** -126))
    assert (scale < F(2.0 ** -125)).all() and (units % 2 == 1).all()
    k = rng.integers(-127, 127, (rows, cols))
    k[:, : cols // 2] = rng.integers(-4, 4, (rows, cols // 2))
    half = ((k + 0.5) * scale.astype(np.float64)[:, None]).astype(F)
    side = np.arange(cols) % 3
    x = np.where(side == 0, half, np.where(side == 1, np.nextafter(half, F(1)), np.nextafter(half, F(-1))))
    x = np.clip(x, -top[:, None], top[:, None]).astype(F)
    x[:, cols - 1] = top
    for i, (most, value, _) in enumerate(KNOWN):
        if i + 1 < rows:
            x[i + 1] = np.where(np.abs(x[i + 1]) > F(most), F(0), x[i + 1])
            x[i + 1, 0], x[i + 1, cols - 1] = value, most
    return x


def test_the_known_values():
    """By the definition in 64 bits."""
    for most, value, q in KNOWN:
        assert U.quantize_rows(np.array([[F(value), F(most)]]))[0][0, 0] == q


@pytest.mark.parametrize("rows,cols", [(400, 128), (400, 250), (300, 999), (200, 4000), (60, 12288), (20, 33001)])
def test_rows(d, rows, cols):
    x = torch.from_numpy(rows_next_to_halves(rows, cols, cols)).cuda()
    q, scale, values = d.int8_rows(rows, cols), torch.empty(rows, device="cuda"), torch.empty_like(x)
    d.quantize_rows(x, q, scale, values=values)
    want_q, want_s = U.quantize_rows(host64(x))
    assert np.array_equal(host64(scale), want_s)
    assert np.array_equal(q.cpu().numpy(), want_q)
    assert np.array_equal(values.cpu().numpy(), (want_q * want_s[:, None]).astype(F))


@pytest.mark.parametrize("rows,cols", [(1, 500), (2, 999), (1, 6000), (3, 130), (100, 256), (50, 511), (40, 700)])
def test_products_that_round_their_rows(d, rows, cols):
    """Weights that pick one element each, with scales of 1: y is what the integers stand for."""
    x = torch.from_numpy(rows_next_to_halves(rows, cols, 7 * cols)).cuda()
    w = d.int8_rows(cols, cols).copy_(torch.eye(cols, dtype=torch.int8))
    y = torch.empty(rows, cols, device="cuda")
    cfg = d.int8_config(x, w, y)
    d.int8_linear(cfg, x, w, torch.ones(cols, device="cuda"), y, ws=d.workspace(d.int8_linear_workspace_bytes(cfg)))
    q, scale = U.quantize_rows(host64(x))
    assert np.array_equal(y.cpu().numpy(), (q * scale[:, None]).astype(F))
