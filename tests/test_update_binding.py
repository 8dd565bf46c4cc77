"""What the binding refuses before the library is called, for the calls of ditupdate.h and ditint8.h (no GPU needed; the calls that pass
reach a stand-in)."""
import pytest
import torch

from paper_2606_19004_amd import ditstep as d

BF, F32, F64, I8 = torch.bfloat16, torch.float32, torch.float64, torch.int8


@pytest.fixture(autouse=True)
def no_library(monkeypatch):
    """The calls' C entries return success; CPU tensors count as on the current device."""
    class Lib:
        def __getattr__(self, name):
            return lambda *a: 0
    monkeypatch.setattr(d, "_lib", Lib())
    monkeypatch.setattr(d, "_current_device", lambda: -1)
    monkeypatch.setattr(d, "_s", lambda stream: None)


def refused(call, args, **change):
    call(**args)
    with pytest.raises(ValueError):
        call(**{**args, **change})


def test_gradient_lists():
    a, b = torch.zeros(10, 3, dtype=BF), torch.zeros(7)
    g = d.grad_list([a, None, b, torch.zeros(0)])
    assert g.count == 3 and (g.array[0].count, g.array[0].dtype, g.array[1].dtype) == (30, 1, 0)
    assert g.array[1].data == b.data_ptr()
    flat = torch.zeros(20)
    d.grad_list([flat[:10], flat[10:]])
    for bad in ([a.half()], [a[:, :2]], [a.t()], [b.double()], [a, a], [flat[:11], flat[10:]], [b, a, b.view(7, 1)]):
        with pytest.raises(ValueError):
            d.grad_list(bad)
    out = dict(grads=g, max_norm=1.0, norm=torch.zeros(1, dtype=F64), scale=torch.zeros(1), ws=torch.zeros(64, dtype=torch.uint8))
    refused(d.grad_norm, out, norm=torch.zeros(1))
    refused(d.grad_norm, out, scale=torch.zeros(1, dtype=F64))
    refused(d.grad_norm, out, scale=torch.zeros(0))
    refused(d.grad_clip, dict(grads=g, scale=torch.zeros(1)), scale=torch.zeros(1, dtype=BF))


def test_lists_of_another_device(monkeypatch):
    g = d.grad_list([torch.zeros(4)])
    w = d.adamw_list(*[[torch.zeros(4)] for _ in range(4)])
    monkeypatch.setattr(d, "_current_device", lambda: 1)
    for call in (lambda: d.grad_norm(g, 1.0), lambda: d.grad_clip(g, None), lambda: d.adamw_step(w, 1e-3)):
        with pytest.raises(ValueError, match="cuda"):
            call()


def weights():
    p = [torch.zeros(4, 5), torch.zeros(3, dtype=BF)]
    return dict(params=p, grads=[torch.zeros(4, 5, dtype=BF), torch.zeros(3)], m=[torch.zeros(4, 5), torch.zeros(3)],
                v=[torch.zeros(4, 5), torch.zeros(3)], copies=[torch.zeros(4, 5, dtype=BF), None])


@pytest.mark.parametrize("name", ["params", "grads", "m", "v", "copies"])
def test_weight_lists(name):
    w = weights()
    x = w[name][0]
    for bad in (x.half(), x.double(), torch.zeros(4, 6, dtype=x.dtype)[:, :5], torch.zeros(5, 4, dtype=x.dtype), torch.zeros(5, 4, dtype=x.dtype).t()):
        refused(d.adamw_list, w, **{name: [bad, w[name][1]]})
    if name in ("m", "v"):
        refused(d.adamw_list, w, **{name: [x.bfloat16(), w[name][1]]})
    if name == "copies":
        refused(d.adamw_list, w, copies=[x.float(), None])
    refused(d.adamw_list, w, **{name: w[name][:1]})


def test_weights_that_share_memory():
    w = weights()
    refused(d.adamw_list, w, v=w["m"])
    refused(d.adamw_list, w, m=[w["params"][0], w["m"][1]])
    a = d.adamw_list(**w)
    assert (a.array[0].param_dtype, a.array[0].grad_dtype, a.array[1].param_dtype, a.array[1].grad_dtype, a.array[1].copy) == (0, 1, 1, 0, None)
    refused(d.adamw_step, dict(weights=a, lr=1e-3, scale=torch.zeros(1), step_dev=torch.ones(1, dtype=torch.int64)), step_dev=torch.ones(1, dtype=torch.int32))
    refused(d.adamw_step, dict(weights=a, lr=1e-3, scale=torch.zeros(1)), scale=torch.zeros(1, dtype=F64))


def test_quantize_rows():
    t = dict(x=torch.zeros(5, 20, dtype=BF)[:, :13], q=d.int8_rows(5, 13, "cpu"), scale=torch.zeros(5), values=torch.zeros(5, 13, dtype=BF))
    for change in (dict(x=t["x"].half()), dict(x=torch.zeros(13, 5, dtype=BF).t()), dict(x=t["x"][:4]), dict(q=t["q"].to(torch.uint8)), dict(q=t["q"][:, :12]),
                   dict(q=torch.zeros(13, 5, dtype=I8).t()), dict(scale=torch.zeros(4)), dict(scale=torch.zeros(5, dtype=BF)), dict(values=torch.zeros(5, 13)),
                   dict(values=torch.zeros(4, 13, dtype=BF)), dict(x=torch.zeros(65, dtype=BF))):
        refused(d.quantize_rows, t, **change)


def int8(given):
    x = d.int8_rows(5, 13, "cpu") if given else torch.zeros(5, 20, dtype=BF)[:, :13]
    t = dict(x=x, w=d.int8_rows(7, 13, "cpu"), w_scale=torch.zeros(7), y=torch.zeros(5, 9, dtype=BF)[:, :7], bias=torch.zeros(7, dtype=BF),
             ws=torch.zeros(1024, dtype=torch.uint8))
    if given:
        t["x_scale"] = torch.zeros(5)
    cfg = d.int8_config(t["x"], t["w"], t["y"], act="gelu")
    return (d.int8_matmul if given else d.int8_linear), dict(t, cfg=cfg)


@pytest.mark.parametrize("given", [True, False])
def test_int8_calls(given):
    call, t = int8(given)
    c = t["cfg"]
    assert (c.rows, c.in_features, c.out_features, c.dtype, c.act, c.w_row, c.x_row, c.y_row) == (5, 13, 7, 1, 1, 16, 16 if given else 20, 9)
    for change in (dict(x=t["x"][:4]), dict(x=t["x"].float()), dict(w=t["w"][:6]), dict(w=t["w"].contiguous()), dict(w=t["w"].to(torch.uint8)), dict(w_scale=torch.zeros(6)),
                   dict(w_scale=torch.zeros(7, dtype=BF)), dict(y=torch.zeros(5, 7, dtype=BF)), dict(y=t["y"].float()), dict(bias=torch.zeros(7)),
                   dict(bias=torch.zeros(6, dtype=BF))):
        refused(call, t, **change)
    if given:
        refused(call, t, x_scale=torch.zeros(4))
    # rows whose last 16 bytes are not all there
    short = torch.zeros(6 * 16 + 13, dtype=I8).as_strided((7, 13), (16, 1))
    refused(call, t, w=short)


def test_int8_config():
    x, w, y = torch.zeros(5, 32, dtype=BF), torch.zeros(7, 32, dtype=I8), torch.zeros(5, 7, dtype=BF)
    refused(d.int8_config, dict(x=x, w=w, y=y), y=y.float())
    refused(d.int8_config, dict(x=x, w=w, y=y), w=w[:, :31])
    refused(d.int8_config, dict(x=x, w=w, y=y), y=y[:4])
    refused(d.int8_config, dict(x=x, w=w, y=y), x=x.half())
    refused(d.int8_config, dict(x=x, w=w, y=y), w=torch.zeros(32, 7, dtype=I8).t())
    d.int8_config(torch.zeros(5, 32, dtype=I8), w, y.float())
    with pytest.raises(KeyError):
        d.int8_config(x, w, y, act="relu")
    one = d.int8_config(torch.zeros(1, 13, dtype=I8), torch.zeros(1, 13, dtype=I8), torch.zeros(1, 1))
    assert (one.x_row, one.w_row) == (16, 16)
