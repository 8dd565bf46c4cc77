"""The operators of an update's end and of the 8-bit rollout as they are used together: gradients, their norm, the AdamW step with its
factor, the new weights to 8-bit integers, and a rollout block over packed sequences of unlike lengths that runs on these
(norm, q/k/v projection, attention, output projection, gated residual with the next norm, MLP, gated residual). Eager and captured.

Against float64 of the same step. After the update the weights are off by 2^-20 of the step's size at most, so integers flip only where a
quotient is that near a half; activations are rounded to fp32 (2^-24) or bf16 (2^-8) before they are rounded to integers. A flipped
integer is off by one step, 1/127 of its row's largest value. The reference rounds its own float64 activations to integers,
so the two differ by flips: with rounding errors of size r relative to the row's largest value, a share 127 r of the integers flips (each
quotient is moved by 127 r at most), and each flip moves a sum over K terms by one step of x times a weight. In the 2-norm over K
independent terms the flips' part is sqrt(127 r) steps of a root mean square 1/127 where rounding itself is off by 1/sqrt(12): in fp32
(r about 2^-20 after the sums before it) sqrt(127 2^-20) / 127 = 9e-5 relative to the largest value, four layers deep and times the ratio of
largest to root mean square (about 4) 1.5e-3; in bf16 (r = 2^-7) every second integer may flip: 1/127 times 4 x 4, 0.12, and 2^-8
for each of 8 stored tensors, 0.03."""
import math

import numpy as np
import pytest
import torch

from oracle import policy_oracle as P
from oracle import update_oracle as U
from tests.gpu_util import host64

pytestmark = pytest.mark.gpu
D, H, G, HD, F = 256, 4, 2, 64, 640
LENS = [5, 40, 1, 23]
HYPER = dict(lr=1e-2, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.1)
TOL = {torch.float32: 1.5e-3, torch.bfloat16: 0.15}
SHAPES = {"qkv": ((H + 2 * G) * HD, D), "out": (D, H * HD), "up": (F, D), "down": (D, F)}


@pytest.fixture(scope="module")
def d():
    from paper_2606_19004_amd import ditstep
    return ditstep


class Step:
    """Everything on the GPU, into preallocated tensors; run() may be captured."""

    def __init__(self, d, dtype):
        self.d, self.dtype = d, dtype
        g = torch.Generator().manual_seed(11)
        n = lambda *s, std=1.0: std * torch.randn(*s, generator=g)  # noqa: E731
        self.S, self.R = len(LENS), sum(LENS)
        off = [0]
        for ln in LENS:
            off.append(off[-1] + ln)
        self.off_host, self.off = off, torch.tensor(off, dtype=torch.int32, device="cuda")
        # fp32 master weights, gradients in the model's type, moments; biases in the model's type
        self.w = {k: n(*s, std=s[1] ** -0.5).cuda() for k, s in SHAPES.items()}
        self.grad = {k: n(*s, std=0.05).to(dtype).cuda() for k, s in SHAPES.items()}
        self.m = {k: n(*s, std=0.01).cuda() for k, s in SHAPES.items()}
        self.v = {k: n(*s, std=0.02).square().cuda() for k, s in SHAPES.items()}
        self.bias = {k: n(s[0], std=0.1).to(dtype).cuda() for k, s in SHAPES.items()}
        self.step = torch.zeros(1, dtype=torch.int64, device="cuda")
        self.x = n(self.R, D).to(dtype).cuda()
        self.mod = n(self.S, 5, D, std=0.5).cuda()
        e = lambda *s, t=dtype: torch.empty(*s, dtype=t, device="cuda")  # noqa: E731
        self.copy = {k: e(*s, t=torch.bfloat16) for k, s in SHAPES.items()}
        self.norm, self.scale = e(1, t=torch.float64), e(1, t=torch.float32)
        self.gl = d.grad_list(self.grad.values())
        self.al = d.adamw_list(self.w.values(), self.grad.values(), self.m.values(), self.v.values(), self.copy.values())
        self.q = {k: d.int8_rows(*s) for k, s in SHAPES.items()}
        self.qs = {k: e(s[0], t=torch.float32) for k, s in SHAPES.items()}
        R = self.R
        self.h, self.h2, self.x1, self.x2, self.y, self.y2 = (e(R, D) for _ in range(6))
        self.qkv, self.o, self.u = e(R, H + 2 * G, HD), e(R, H, HD), e(R, F)
        self.flat = self.qkv.view(R, -1)
        self.c1 = d.gated_norm_config(self.x, self.S, "none", "layer", mod_row=5 * D)
        self.c2 = d.gated_norm_config(self.x, self.S, "rms", "layer", mod_row=5 * D)
        self.ca = d.packed_config(self.qkv[:, :H], self.qkv[:, H:H + G], self.qkv[:, H + G:], self.o, self.S, max_q=max(LENS))
        io = {"qkv": (self.h, self.flat), "out": (self.o.view(R, -1), self.y), "up": (self.h2, self.u), "down": (self.u, self.y2)}
        self.io = {k: (x, y, d.int8_config(x, self.q[k], y, act="gelu" if k == "up" else "none")) for k, (x, y) in io.items()}
        need = [d.int8_linear_workspace_bytes(c) for _, _, c in self.io.values()]
        need += [d.grad_norm_workspace_bytes(self.gl), d.packed_attention_workspace_bytes(self.ca)]
        self.ws = d.workspace(max(need))

    def linear(self, k):
        x, y, cfg = self.io[k]
        self.d.int8_linear(cfg, x, self.q[k], self.qs[k], y, bias=self.bias[k], ws=self.ws)

    def run(self):
        d, m = self.d, [self.mod[:, i] for i in range(5)]
        self.step += 1
        d.grad_norm(self.gl, 1.0, self.norm, self.scale, ws=self.ws)
        d.adamw_step(self.al, scale=self.scale, step_dev=self.step, **HYPER)
        for k in SHAPES:
            d.quantize_rows(self.w[k], self.q[k], self.qs[k])
        d.gated_norm(self.c1, self.x, None, None, self.h, scale=m[1], shift=m[0], offsets=self.off)
        self.linear("qkv")
        d.packed_attention(self.ca, self.qkv[:, :H], self.qkv[:, H:H + G], self.qkv[:, H + G:], self.o, q_offsets=self.off,
                           k_offsets=self.off, ws=self.ws)
        self.linear("out")
        d.gated_norm(self.c2, self.x, self.y, self.x1, self.h2, gate=m[2], scale=m[3], shift=m[4], offsets=self.off)
        self.linear("up")
        self.linear("down")
        d.gated_norm(self.c1, self.x1, self.y2, self.x2, None, offsets=self.off)
        return {"x": self.x2, "norm": self.norm, "scale": self.scale, **{f"w.{k}": t for k, t in self.w.items()},
                **{f"copy.{k}": t for k, t in self.copy.items()}, **{f"q.{k}": t for k, t in self.q.items()}}

    def state(self):
        return [*self.w.values(), *self.m.values(), *self.v.values(), self.step]


def reference(s):
    """The step from s's state in float64: output, weights, norm and scale."""
    norm, scale = U.grad_norm([host64(g) for g in s.grad.values()], 1.0)
    t = int(s.step) + 1
    w = {k: U.adamw(host64(s.w[k]), host64(s.grad[k]), host64(s.m[k]), host64(s.v[k]), HYPER["lr"], HYPER["beta1"], HYPER["beta2"], HYPER["eps"],
                    HYPER["weight_decay"], t, scale)[0] for k in SHAPES}

    def linear(k, x):
        xq, xs = U.quantize_rows(x)
        wq, ws = U.quantize_rows(w[k].astype(np.float32))
        return U.int8_matmul(xq, xs, wq, ws, host64(s.bias[k]), k == "up")[0]

    def by_sequence(f):
        return np.concatenate([f(i, slice(a, b)) for i, (a, b) in enumerate(zip(s.off_host, s.off_host[1:]))])

    mod, one = host64(s.mod), np.ones(D)
    x = host64(s.x)
    h = by_sequence(lambda i, r: P.gated_norm(x[r], None, one, mod[i, 1], mod[i, 0], one, one, "none", "layer", 1e-6, 1.0)[1])
    qkv = linear("qkv", h).reshape(-1, H + 2 * G, HD)
    o = by_sequence(lambda i, r: np.stack([P.attention(qkv[r, j], qkv[r, H + j * G // H], qkv[r, H + G + j * G // H], 1 / math.sqrt(HD), False)[0]
                                           for j in range(H)], 1))
    y = linear("out", o.reshape(-1, H * HD))
    pair = [P.gated_norm(x[a:b], y[a:b], mod[i, 2], mod[i, 3], mod[i, 4], one, one, "rms", "layer", 1e-6, 1.0)
            for i, (a, b) in enumerate(zip(s.off_host, s.off_host[1:]))]
    x1, h2 = (np.concatenate(t) for t in zip(*pair))
    return x1 + linear("down", linear("up", h2)), w, norm, scale


def off_by(got, want):
    return np.linalg.norm(host64(got) - want) / np.linalg.norm(want)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_update_then_rollout(d, dtype):
    s = Step(d, dtype)
    for _ in range(2):
        x, w, norm, scale = reference(s)
        out = s.run()
        torch.cuda.synchronize()
        assert abs(float(out["norm"]) - norm) <= 1e-12 * norm and abs(float(out["scale"]) - scale) <= 2.0 ** -24 * scale and scale < 1
        for k in SHAPES:
            assert off_by(out[f"w.{k}"], w[k]) <= 2.0 ** -21
            assert torch.equal(out[f"copy.{k}"], out[f"w.{k}"].to(torch.bfloat16))
            assert np.array_equal(s.q[k].cpu().numpy(), U.quantize_rows(host64(s.w[k]))[0])
        assert off_by(out["x"], x) <= TOL[dtype]


def test_captured(d):
    """Replays give the bits of eager steps from the same state, with eager work, and another captured step on the same workspace,
    between them; the step's number counts on the device. A gradient that is not finite leaves the weights as they were."""
    s = Step(d, torch.bfloat16)
    start = [t.clone() for t in s.state()]

    def reset():
        for t, b in zip(s.state(), start):
            t.copy_(b)

    want = []
    for _ in range(3):
        out = s.run()
        torch.cuda.synchronize()
        want.append({k: t.clone() for k, t in out.items()})
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            out = s.run()
        graphs.append(g)
    reset()
    for i in range(3):
        graphs[i % 2].replay()
        d.quantize_rows(torch.randn(9, D, device="cuda"), d.int8_rows(9, D), torch.empty(9, device="cuda"))   # eager work between replays
        torch.cuda.synchronize()
        for k, t in out.items():
            assert torch.equal(t, want[i][k]), (i, k)
        assert int(s.step) == i + 1
    kept = [t.clone() for t in s.state()[:-1]]
    good = s.grad["up"][3, 5].clone()
    s.grad["up"][3, 5] = float("inf")
    graphs[0].replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(kept, s.state()[:-1])) and math.isnan(float(s.scale))
    s.grad["up"][3, 5] = good
    reset()
    for i in range(2):
        graphs[1].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(t, want[i][k]) for k, t in out.items())
