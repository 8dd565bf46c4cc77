"""How many results a product of 8-bit integers may have (no GPU needed: every call here is refused before it reaches its tensors)."""
import ctypes as C

import pytest

from paper_2606_19004_amd import ditstep as d
from tests.int8_util import int8_form

INVALID, UNSUPPORTED, WORKSPACE = 1, 5, 7
A = 1 << 20      # an aligned stand-in for a device pointer


def statuses(rows, out, cols=2000):
    """Of a product without the scales of x, and of a layer without its workspace, which is what is looked at after the sizes."""
    cfg = d.Int8Config(rows, cols, out, 1, 0, -(-cols // 16) * 16, -(-cols // 16) * 16, out)
    lib = d.lib()
    return (lib.int8_matmul(C.byref(cfg), A, None, A, A, None, A, None, 0, None), lib.int8_linear(C.byref(cfg), A, A, A, None, A, None, 0, None))


# 2^34 results in 32 x 32 tiles would take 2^32 threads; in the tiles that these sizes get they take far fewer
@pytest.mark.parametrize("rows,out", [(1_500_000, 12288), (12288, 1_500_000), (1 << 20, 1 << 17), ((1 << 31) - 10000, 100), (1 << 30, 200), (5, (1 << 30) - 1)])
def test_many_results(rows, out):
    assert statuses(rows, out) == (INVALID, WORKSPACE)


@pytest.mark.parametrize("rows", [1, 2])
def test_one_or_two_rows_of_very_many_features(rows):
    """Dot products would take 2^32 threads, also those that round their rows themselves."""
    out = (1 << 30) - 1
    assert statuses(rows, out, 20000) == (INVALID, WORKSPACE)
    for cols in (5, 2000, 20000):
        assert int8_form(rows, cols, out) != "few rows"
        assert d.int8_linear_workspace_bytes(d.Int8Config(rows, cols, out, 1, 0, cols, -(-cols // 16) * 16, out)) > 0


@pytest.mark.parametrize("rows,out", [((1 << 31) - 1, (1 << 30) - 1), (1 << 21, 1 << 18), ((1 << 31) - 1, 256)])
def test_more_than_a_launch_takes(rows, out):
    assert statuses(rows, out) == (UNSUPPORTED, UNSUPPORTED)
