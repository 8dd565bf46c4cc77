"""The oracle of the update's end and of 8-bit products, by values worked by hand and by what the definitions imply."""
from fractions import Fraction

import numpy as np

from oracle import update_oracle as U


def test_quantized_rows_worked():
    q, s = U.quantize_rows([[127.0, 2.5, -3.5, 0.5, 1.5, -127.0], [0] * 6, [2.0 ** -130, 0, 0, 0, 0, 0], [1, np.inf, 0, 0, 0, 0],
                            [np.nan, 0, 0, 0, 0, 3]])
    assert q[0].tolist() == [127, 2, -4, 0, 2, -127] and s[0] == 1.0
    assert not q[1].any() and s[1] == 2.0 ** -126                       # no division by zero
    assert not q[2].any() and s[2] == 2.0 ** -126                       # a sixteenth of the least scale
    assert not q[3:].any() and np.isnan(s[3:]).all()


def test_quotients_are_rounded_exactly():
    """Against rational arithmetic, at the fp32 neighbours of every half of a few scales."""
    rng = np.random.default_rng(1)
    for top in rng.uniform(0.5, 2, 20).astype(np.float32):
        s = float(np.float32(top / np.float64(127)))
        x = [float(top)]
        for k in range(-127, 127):
            h = np.float32((k + 0.5) * s)
            x += [float(h), float(np.nextafter(h, np.float32(np.inf))), float(np.nextafter(h, np.float32(-np.inf)))]
        x = [v for v in x if abs(v) <= float(top)]
        q, _ = U.quantize_rows([x])
        assert [round(Fraction(v) / Fraction(s)) for v in x] == q[0].tolist()   # round(Fraction): ties to even


def test_product_worked():
    y, total = U.int8_matmul(np.array([[1, 2], [-128, 127]]), np.array([0.5, 2.0]), np.array([[3, 4], [5, -6], [-128, 0]]),
                             np.array([1.0, 0.25, 2.0]), bias=np.array([1.0, 0.0, -1.0]))
    assert total.tolist() == [[11, -7, -128], [124, -1402, 16384]]
    assert y.tolist() == [[6.5, -0.875, -129.0], [249.0, -701.0, 65535.0]]
    assert np.allclose(U.gelu_tanh(np.array([0.0, 1.0, -1.0])), [0.0, 0.8411919906082768, -0.15880800939172324])


def test_norm_and_update_worked():
    assert U.grad_norm([[3.0], [[4.0]]], 10.0) == (5.0, 1.0)
    assert U.grad_norm([[3.0], [[4.0]]], 1.0)[1] == 1.0 / (5.0 + 1e-6)
    assert U.grad_norm([], 1.0) == (0.0, 1.0) and np.isnan(U.grad_norm([[np.inf]], 1.0)[1])
    # the first step from zero moments goes lr in the gradient's direction, whatever its size
    for g in (1e-3, -7.0):
        p, m, v = U.adamw(1.0, g, 0.0, 0.0, 0.1, 0.9, 0.999, 0.0, 0.5, 1)
        assert np.isclose(p, 1.0 - 0.1 * (np.sign(g) + 0.5)) and np.isclose(m, 0.1 * g) and np.isclose(v, 1e-3 * g * g)
    assert U.adamw(1.0, 2.0, 0.5, 0.25, 0.1, 0.9, 0.999, 0.0, 0.5, 1, scale=np.nan) == (1.0, 0.5, 0.25)
