"""Sizes past what the policy-update kernels count in are refused before any launch (no GPU needed)."""
import pytest

from paper_2606_19004_amd import ditstep as d
from tests.test_policy_host import A, UNSUPPORTED, norm, norm_back, norm_cfg


@pytest.mark.parametrize("hidden", [64, 320, 8192])
@pytest.mark.parametrize("rows", [(1 << 28) + 1, (1 << 31) - 1])
def test_gated_norm_of_too_many_rows(rows, hidden):
    """A sequence's chunks of 8 rows are counted up to 2^25."""
    c = norm_cfg(rows=rows, hidden=hidden, x_row=hidden, y_row=hidden, h_row=hidden, mod_row=hidden)
    assert norm(c) == UNSUPPORTED
    assert norm_back(c, dt=A) == UNSUPPORTED
    assert d.gated_norm_backward_workspace_bytes(c) == 0
