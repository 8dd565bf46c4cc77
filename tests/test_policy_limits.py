"""Sizes past what the policy-update kernels count in are refused before any launch (no GPU needed)."""
import pytest

from paper_2606_19004_amd import ditstep as d
from tests.test_policy_host import A, UNSUPPORTED, backward, forward, loss, norm, norm_back, norm_cfg, packed


@pytest.mark.parametrize("hidden", [64, 320, 8192])
@pytest.mark.parametrize("rows", [(1 << 28) + 1, (1 << 31) - 1])
def test_gated_norm_of_too_many_rows(rows, hidden):
    """A sequence's chunks of 8 rows are counted up to 2^25."""
    c = norm_cfg(rows=rows, hidden=hidden, x_row=hidden, y_row=hidden, h_row=hidden, mod_row=hidden)
    assert norm(c) == UNSUPPORTED
    assert norm_back(c, dt=A) == UNSUPPORTED
    assert d.gated_norm_backward_workspace_bytes(c) == 0


@pytest.mark.parametrize("kw", [dict(sequences=(1 << 20) - 1, heads=32, kv_heads=32, total_q=(1 << 20) - 1, total_k=1 << 20, max_q=1),
                                dict(sequences=(1 << 20) - 1, heads=32, kv_heads=32, total_q=(1 << 20) - 1, total_k=1 << 20, max_q=1, dtype=0,
                                     q_head=256, k_head=256, v_head=256, o_head=256, q_row=8192, k_row=8192, v_row=8192, o_row=8192)])
def test_attention_of_more_workgroups_than_a_launch_takes(kw):
    """256 threads each of 2^25 (sequence, head) pairs: a launch takes fewer than 2^32."""
    cfg = packed(**{**dict(q_row=2048, k_row=2048, v_row=2048, o_row=2048), **kw})
    assert forward(cfg, ws=A, n=1 << 50) == UNSUPPORTED
    assert backward(cfg, n=1 << 50) == UNSUPPORTED


def test_attention_gradients_of_more_rows_than_a_launch_takes():
    """The rows' statistics: 16 lanes to a row of 128 bf16 elements."""
    cfg = packed(sequences=1, heads=32, kv_heads=32, head_dim=128, total_q=1 << 23, total_k=1 << 23, q_row=4096, k_row=4096, v_row=4096,
                 o_row=4096, q_head=128, k_head=128, v_head=128, o_head=128)
    assert backward(cfg, n=1 << 50) == UNSUPPORTED


def test_gated_norm_of_more_workgroups_than_a_launch_takes():
    wide = dict(hidden=8192, x_row=8192, y_row=8192, h_row=8192, mod_row=8192)
    assert norm(norm_cfg(rows=1 << 26, **wide)) == UNSUPPORTED                      # 1024 threads to 8 rows
    assert norm(norm_cfg(rows=1 << 28, hidden=256, x_row=256, y_row=256, h_row=256, mod_row=256)) == UNSUPPORTED   # 32 to a row
    c = norm_cfg(rows=1 << 18, sequences=1 << 18, **wide)
    assert norm_back(c, dt=A, n=1 << 50) == UNSUPPORTED                             # 256 threads to 64 columns of a sequence


def test_policy_loss_of_more_samples_than_a_launch_takes():
    assert loss(B=1 << 24, n=4, nb=1 << 40) == UNSUPPORTED


@pytest.mark.parametrize("sequences", [1000, 20000])
def test_workspace_is_for_sequences_that_are_shared_out(sequences):
    """One new token of each of many sequences of 64 keys. Partial results have room for the sequences whose keys could be in more
    than one part, not for all: with 512 workgroups' worth of parts, twice as many slots of 16 rows of 130 floats, and 2 x 8 more."""
    cfg = packed(sequences=sequences, heads=32, kv_heads=8, head_dim=128, total_q=sequences, total_k=64 * sequences, max_q=1, q_row=4096, q_head=128,
                 k_row=1024, k_head=128, v_row=1024, v_head=128, o_row=4096, o_head=128)
    assert 0 < d.packed_attention_workspace_bytes(cfg) <= (2 * 512 + 16) * 16 * 130 * 4 + 256
