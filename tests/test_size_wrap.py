"""Sizes past 31 bits: the library's are 32-bit integers, into which a tensor's would wrap (no GPU needed; the calls that pass reach a stand-in)."""
import pytest
import torch

from paper_2606_19004_amd import ditstep as d

FAR = 2 ** 32 + 1     # 1, where it wraps


@pytest.fixture(autouse=True)
def no_library(monkeypatch):
    class Lib:
        def __getattr__(self, name):
            return lambda *a: 0
    monkeypatch.setattr(d, "_lib", Lib())
    monkeypatch.setattr(d, "_current_device", lambda: -1)
    monkeypatch.setattr(d, "_s", lambda stream: None)


def many(shape, dtype):
    """A tensor of that shape without its memory."""
    return torch.zeros(shape[1:], dtype=dtype).expand(shape)


def test_quantize_rows():
    def call(rows):   # (the scales' memory is never touched)
        d.quantize_rows(many((rows, 8), torch.bfloat16), many((rows, 8), torch.int8), torch.empty(rows))
    call(4)
    with pytest.raises(ValueError, match="2\\^31"):
        call(FAR)


@pytest.mark.parametrize("dtype", [torch.int8, torch.bfloat16])
def test_int8_config(dtype):
    def config(rows, out):
        return d.int8_config(many((rows, 16), dtype), many((out, 16), torch.int8), many((rows, out), torch.bfloat16))
    assert (config(4, 5).rows, config(4, 5).out_features) == (4, 5)
    for sizes in ((FAR, 5), (4, FAR), (2 ** 31, 5)):
        with pytest.raises(ValueError, match="2\\^31"):
            config(*sizes)


def test_policy_configs():
    x = many((FAR, 16), torch.bfloat16)
    with pytest.raises(ValueError, match="2\\^31"):
        d.gated_norm_config(x, 1)
    q = many((FAR, 2, 16), torch.bfloat16)
    k = torch.zeros(4, 2, 16, dtype=torch.bfloat16)
    d.packed_config(k, k, k, k, 1)
    for a, b in ((q, k), (k, q)):
        with pytest.raises(ValueError, match="2\\^31"):
            d.packed_config(a, b, b, a, 1)


def test_samples_and_groups():
    one = torch.zeros(1, dtype=torch.float64)

    def logprob(rows):
        x = many((rows, 1), torch.float32)
        d.flow_logprob(x, x, x, 0.5, 0.4, 0.7, one)

    def loss(rows):
        x = many((rows, 1), torch.float32)
        d.flow_policy_loss(*[x.contiguous() if rows == 1 else x] * 3, one, torch.zeros(1), 0.5, 0.4, 0.7, one)
    for call in (logprob, loss, lambda rows: d.flow_policy_loss_workspace_bytes(rows, 5), lambda rows: d.group_reward_stats(many((rows, 2), torch.float32)),
                 lambda rows: d.group_reward_stats(many((2, rows), torch.float32)), lambda rows: d.group_reward_stats_async(many((rows, 2), torch.float32), one)):
        call(1)
        with pytest.raises(ValueError, match="2\\^31"):
            call(FAR)
