"""What the binding refuses before the library is called: tensors that are not what their config says (no GPU needed; the calls
that pass reach a stand-in)."""
import pytest
import torch

from paper_2606_19004_amd import ditstep as d

BF, F32, F64, I32 = torch.bfloat16, torch.float32, torch.float64, torch.int32


@pytest.fixture(autouse=True)
def no_library(monkeypatch):
    """The calls' C entries return success; CPU tensors count as on the current device."""
    class Lib:
        def __getattr__(self, name):
            return lambda *a: 0
    monkeypatch.setattr(d, "_lib", Lib())
    monkeypatch.setattr(d, "_current_device", lambda: -1)
    monkeypatch.setattr(d, "_s", lambda stream: None)


def attention():
    p = torch.zeros(20, 8, 64, dtype=BF)              # slices of one projection
    t = dict(q=p[:, :4], k=p[:, 4:6], v=p[:, 6:], o=torch.zeros(20, 4, 64, dtype=BF), lse=torch.zeros(20, 4), q_offsets=torch.zeros(4, dtype=I32),
             k_offsets=torch.zeros(4, dtype=I32), k_lengths=torch.zeros(3, dtype=I32))
    cfg = d.packed_config(t["q"], t["k"], t["v"], t["o"], 3, True)
    g = torch.zeros_like(p)
    back = dict(t, d_o=torch.zeros_like(t["o"]), dq=g[:, :4], dk=g[:, 4:6], dv=g[:, 6:])
    return cfg, t, back


def refused(call, cfg, args, **change):
    call(cfg, **args)
    with pytest.raises(ValueError):
        call(cfg, **{**args, **change})


ATTENTION = [("q", lambda t: t.float()), ("k", lambda t: t.half()), ("o", lambda t: t.float()), ("lse", lambda t: t.bfloat16()),
             ("lse", lambda t: t.double()), ("lse", lambda t: t[:19]), ("lse", lambda t: t.t()), ("q", lambda t: t[:19]), ("v", lambda t: t.contiguous()),
             ("o", lambda t: torch.zeros(20, 8, 64, dtype=BF)[:, :4]), ("q_offsets", lambda t: t[:3]), ("k_offsets", lambda t: t.long()),
             ("k_lengths", lambda t: t[:2]), ("k_offsets", lambda t: torch.zeros(8, dtype=I32)[::2])]


@pytest.mark.parametrize("name,change", ATTENTION)
def test_attention(name, change):
    cfg, t, back = attention()
    refused(d.packed_attention, cfg, t, **{name: change(t[name])})
    refused(d.packed_attention_backward, cfg, back, **{name: change(back[name])})


@pytest.mark.parametrize("name,change", [("d_o", lambda t: t.float()), ("d_o", lambda t: t[:10]), ("dq", lambda t: t.float()),
                                         ("dk", lambda t: t.contiguous()), ("dv", lambda t: t[1:])])
def test_attention_gradients(name, change):
    cfg, _, back = attention()
    refused(d.packed_attention_backward, cfg, back, **{name: change(back[name])})


def norm():
    p = torch.zeros(2, 3, 32)
    r = lambda: torch.zeros(10, 40, dtype=BF)[:, :32]  # noqa: E731
    t = dict(x=r(), y=r(), x_out=r(), h=r(), gate=p[:, 0], scale=p[:, 1], shift=p[:, 2], post_w=torch.zeros(32, dtype=BF),
             pre_w=torch.zeros(32, dtype=BF), offsets=torch.zeros(3, dtype=I32))
    cfg = d.gated_norm_config(t["x"], 2, "rms", "layer", mod_row=96)
    g = torch.zeros(2, 3, 32)
    back = dict(x_out=r(), y=r(), dx_out=r(), dh=r(), dx=r(), dy=r(), gate=p[:, 0], scale=p[:, 1], post_w=t["post_w"], pre_w=t["pre_w"],
                offsets=t["offsets"], dgate=g[:, 0], dscale=g[:, 1], dshift=g[:, 2], dpost_w=torch.zeros(32), dpre_w=torch.zeros(32))
    return cfg, t, back


@pytest.mark.parametrize("change", [lambda t: t.float(), lambda t: t.contiguous(), lambda t: t[:9], lambda t: t[:, :31],
                                    lambda t: torch.zeros(10, 40, dtype=torch.float16)[:, :32]])
def test_norm_rows(change):
    cfg, t, back = norm()
    for name in ("x", "y", "x_out", "h"):
        refused(d.gated_norm, cfg, t, **{name: change(t[name])})
    for name in ("x_out", "y", "dx_out", "dh", "dx", "dy"):
        refused(d.gated_norm_backward, cfg, back, **{name: change(back[name])})


@pytest.mark.parametrize("change", [lambda t: t.bfloat16(), lambda t: t.contiguous(), lambda t: t[:1], lambda t: t[:, :31]])
def test_norm_vectors(change):
    cfg, t, back = norm()
    for name in ("gate", "scale", "shift"):
        refused(d.gated_norm, cfg, t, **{name: change(t[name])})
    for name in ("gate", "scale", "dgate", "dscale", "dshift"):
        refused(d.gated_norm_backward, cfg, back, **{name: change(back[name])})


def test_norm_weights_and_offsets():
    cfg, t, back = norm()
    for name in ("post_w", "pre_w"):
        for w in (torch.zeros(32), torch.zeros(31, dtype=BF), torch.zeros(64, dtype=BF)[::2]):
            refused(d.gated_norm, cfg, t, **{name: w})
            refused(d.gated_norm_backward, cfg, back, **{name: w})
    for name in ("dpost_w", "dpre_w"):
        for w in (torch.zeros(32, dtype=BF), torch.zeros(31)):
            refused(d.gated_norm_backward, cfg, back, **{name: w})
    for off in (torch.zeros(2, dtype=I32), torch.zeros(3, dtype=torch.int64)):
        refused(d.gated_norm, cfg, t, offsets=off)


def test_loss():
    f = lambda *s, t=F32: torch.zeros(*s, dtype=t)  # noqa: E731
    args = dict(x=f(3, 8), v=f(3, 8), x_next=f(3, 8), logp_old=f(3, t=F64), adv=f(3), t=0.6, t_next=0.5, noise_level=0.7, loss=f(1, t=F64),
                dv=f(3, 8), logp=f(3, t=F64), ratio=f(3, t=F64), v_ref=f(3, 8))
    call = lambda cfg, **kw: d.flow_policy_loss(**kw)  # noqa: E731
    for name in ("x", "v", "x_next", "v_ref", "dv"):
        for bad in (f(3, 8, t=F64), f(8, 3).t(), f(3, 16)[:, ::2]) + ((f(2, 8), f(3, 7)) if name != "x" else ()):
            refused(call, None, args, **{name: bad})
    for name in ("logp_old", "logp", "ratio"):
        for bad in (f(3), f(2, t=F64), f(6, t=F64)[::2]):
            refused(call, None, args, **{name: bad})
    for bad in (f(3, t=F64), f(2)):
        refused(call, None, args, adv=bad)
    refused(call, None, args, loss=f(1))


def test_layouts_that_hold_the_same_elements_pass():
    """More rows than the config's, any stride of a single row or head, any contiguous shape of dense rows, no rows at all."""
    cfg, t, _ = attention()
    d.packed_attention(cfg, **{**t, "o": torch.zeros(25, 256, dtype=BF), "lse": torch.zeros(80)})
    one = torch.zeros(1, 6, 64, dtype=BF)
    cfg = d.packed_config(one[:, :4], one[:, 4:5], one[:, 5:], one[:, :4], 1)
    d.packed_attention(cfg, torch.zeros(1, 4, 64, dtype=BF), torch.zeros(1, 1, 64, dtype=BF), torch.zeros(1, 1, 64, dtype=BF), one[:, :4])
    x = torch.zeros(1, 32)
    d.gated_norm(d.gated_norm_config(x, 1), x, None, x, x, gate=torch.zeros(32), scale=torch.zeros(1, 32))
    none = torch.zeros(0, 32)
    d.gated_norm(d.gated_norm_config(none, 1), x, x, none, none)
    d.flow_policy_loss(torch.zeros(2, 3, 4), torch.zeros(2, 12), torch.zeros(24), torch.zeros(2, dtype=F64), torch.zeros(2, 1), 0.6, 0.5, 0.7,
                       torch.zeros((), dtype=F64))
