"""The policy-update operators as a training step uses them: one transformer block over packed joint sequences (prompts of
unlike lengths, images of one size), the velocity of the image tokens, the policy loss, and the way back to every
parameter; the projections between them are torch products. Compared with automatic differentiation of the same step in
float64 on the CPU.

fp32: every operator and product is off by at most some 100 roundings (sums of up to 256 terms) of 2^-24 relative to its
result's size, and there are about 15 of them on the longest path, so 2000 roundings, 1.2e-4, bound what a gradient may be off by
relative to its largest element. bf16: 8 stored tensors (x, h, q/k/v, o, the branch, x, h, v's input) of 2^-8 and as many
gradients on the way back, 16 x 2^-8 = 6e-2 in the worst case."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

D, H, G, HD, IMG, C = 256, 4, 2, 64, 12, 8
TEXT = [5, 40, 1, 23]
T, TN, LVL = 0.62, 0.57, 0.7
EPS = 1e-6
TOL = {torch.float32: 1.2e-4, torch.bfloat16: 6e-2}


@pytest.fixture(scope="module")
def d():
    from paper_2606_19004_amd import ditstep
    return ditstep


def make(dtype):
    g = torch.Generator().manual_seed(3)
    S = len(TEXT)
    lens = [t + IMG for t in TEXT]
    R = sum(lens)
    draw = lambda *s, std=1.0: (std * torch.randn(*s, generator=g, dtype=torch.float64)).to(dtype).double()  # noqa: E731
    p = {"x0": draw(R, D), "qkv": draw((H + 2 * G) * HD, D, std=0.06), "out": draw(D, H * HD, std=0.06), "head": draw(C, D, std=0.06),
         "pre1": 1 + draw(D, std=0.1), "post": 1 + draw(D, std=0.1), "pre2": 1 + draw(D, std=0.1)}
    p = {k: v.to(dtype).double() for k, v in p.items()}
    p["mod"] = (0.5 * torch.randn(S, 6, D, generator=g, dtype=torch.float64)).float().double()
    n = IMG * C
    f32 = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64).float().double()  # noqa: E731
    q = {"x": f32(S, n), "noise": f32(S, n), "adv": f32(S), "drift": 0.3 * f32(S, n)}
    off = [0]
    for ln in lens:
        off.append(off[-1] + ln)
    img = torch.cat([torch.arange(e - IMG, e) for e in off[1:]])
    seq = torch.repeat_interleave(torch.arange(S), torch.tensor(lens))
    return p, q, off, img, seq, n


def norm64(kind, x):
    if kind == "layer":
        x = x - x.mean(1, keepdim=True)
    return x / (x.pow(2).mean(1, keepdim=True) + EPS).sqrt()


def reference(p, q, off, img, seq, n):
    leaf = {k: v.clone().requires_grad_(True) for k, v in p.items()}
    m = leaf["mod"][seq]                                          # shift1, scale1, gate, shift2, scale2, (unused)
    h = norm64("layer", leaf["x0"]) * leaf["pre1"] * (1 + m[:, 1]) + m[:, 0]
    qkv = (h @ leaf["qkv"].T).view(-1, H + 2 * G, HD)
    o = []
    for a, b in zip(off, off[1:]):
        for j in range(H):
            k, v = qkv[a:b, H + j * G // H], qkv[a:b, H + G + j * G // H]
            o.append(torch.softmax(qkv[a:b, j] @ k.T / math.sqrt(HD), -1) @ v)
    o = torch.cat([torch.stack(o[i * H:(i + 1) * H], 1) for i in range(len(TEXT))]).reshape(-1, H * HD)
    x1 = leaf["x0"] + m[:, 2] * norm64("rms", o @ leaf["out"].T) * leaf["post"]
    h2 = norm64("layer", x1) * leaf["pre2"] * (1 + m[:, 4]) + m[:, 3]
    v = (h2[img] @ leaf["head"].T).reshape(len(TEXT), n)
    hh, s2 = TN - T, LVL ** 2 * T / (1 - T)
    mean = lambda vel: q["x"] + hh * (vel + s2 / (2 * T) * (q["x"] + (1 - T) * vel))  # noqa: E731
    var = s2 * -hh
    logp = lambda vel, xn: torch.distributions.Normal(mean(vel), math.sqrt(var)).log_prob(xn).sum(1)  # noqa: E731
    old_v = v.detach() + q["drift"]
    xn = (mean(old_v) + math.sqrt(var) * q["noise"]).float().double()
    old = logp(old_v, xn)
    ratio = ((logp(v, xn) - old) / n).exp()
    ref = (v.detach() + 0.2 * q["noise"].flip(0)).float().double()
    loss = -torch.minimum(ratio * q["adv"], ratio.clamp(0.8, 1.2) * q["adv"]).mean() + 0.04 * ((mean(v) - mean(ref)) ** 2 / (2 * var)).mean()
    loss.backward()
    return loss.detach(), {k: t.grad for k, t in leaf.items()}, xn, old, ref


class Step:
    """Forward, loss and backward on the GPU into preallocated tensors; run() may be captured."""

    def __init__(self, d, dtype, p, q, off, img, xn, old, ref):
        dev = lambda t: t.to(dtype).cuda()  # noqa: E731
        self.d, S, R, n = d, len(TEXT), off[-1], IMG * C
        self.p = {k: (v.float().cuda() if k == "mod" else dev(v)) for k, v in p.items()}
        self.off = torch.tensor(off, dtype=torch.int32, device="cuda")
        self.img = img.cuda()
        self.q = {k: v.float().cuda() for k, v in q.items()}
        self.xn, self.old, self.ref = xn.float().cuda(), old.cuda(), ref.float().cuda()
        e = lambda *s, t=dtype: torch.empty(*s, dtype=t, device="cuda")  # noqa: E731
        self.h, self.h2, self.x1, self.o = e(R, D), e(R, D), e(R, D), e(R, H, HD)
        self.lse, self.loss, self.dv = e(R, H, t=torch.float32), e(1, t=torch.float64), e(S, n, t=torch.float32)
        self.dx1, self.dy, self.dx, self.dqkv = e(R, D), e(R, D), e(R, D), e(R, H + 2 * G, HD)
        self.grad = {k: e(*v.shape, t=torch.float32) for k, v in p.items() if k in ("mod", "pre1", "post", "pre2")}
        x0 = self.p["x0"]
        self.c1 = d.gated_norm_config(x0, S, "none", "layer", EPS, mod_row=6 * D)
        self.c2 = d.gated_norm_config(x0, S, "rms", "layer", EPS, mod_row=6 * D)
        qkv = e(R, H + 2 * G, HD)
        self.ca = d.packed_config(qkv[:, :H], qkv[:, H:H + G], qkv[:, H + G:], self.o, S, max_q=max(TEXT) + IMG)
        nb = max(d.packed_attention_workspace_bytes(self.ca), d.packed_attention_backward_workspace_bytes(self.ca),
                 d.gated_norm_backward_workspace_bytes(self.c1), d.gated_norm_backward_workspace_bytes(self.c2),
                 d.flow_policy_loss_workspace_bytes(S, n))
        self.ws = d.workspace(nb)                                  # one workspace serves the calls of one stream

    def run(self):
        d, p, off, S = self.d, self.p, self.off, len(TEXT)
        m = [p["mod"][:, i] for i in range(6)]
        g = [self.grad["mod"][:, i] for i in range(6)]
        d.gated_norm(self.c1, p["x0"], None, None, self.h, scale=m[1], shift=m[0], pre_w=p["pre1"], offsets=off)
        qkv = (self.h @ p["qkv"].t()).view(-1, H + 2 * G, HD)
        q, k, v = qkv[:, :H], qkv[:, H:H + G], qkv[:, H + G:]
        d.packed_attention(self.ca, q, k, v, self.o, lse=self.lse, q_offsets=off, k_offsets=off, ws=self.ws)
        flat = self.o.view(-1, H * HD)
        y = flat @ p["out"].t()
        d.gated_norm(self.c2, p["x0"], y, self.x1, self.h2, gate=m[2], scale=m[4], shift=m[3], post_w=p["post"], pre_w=p["pre2"], offsets=off)
        hi = self.h2[self.img]
        vel = (hi @ p["head"].t()).float().reshape(S, -1)
        d.flow_policy_loss(self.q["x"], vel, self.xn, self.old, self.q["adv"], T, TN, LVL, self.loss, dv=self.dv, v_ref=self.ref,
                           kl_weight=0.04, ws=self.ws)
        dvel = self.dv.reshape(-1, C).to(hi.dtype)
        out = {"head": dvel.t().contiguous() @ hi}
        dh2 = torch.zeros_like(self.h2)
        dh2[self.img] = dvel @ p["head"]
        d.gated_norm_backward(self.c2, self.x1, y, None, dh2, self.dx1, self.dy, gate=m[2], scale=m[4], post_w=p["post"], pre_w=p["pre2"],
                              offsets=off, dgate=g[2], dscale=g[4], dshift=g[3], dpost_w=self.grad["post"], dpre_w=self.grad["pre2"], ws=self.ws)
        out["out"] = self.dy.t().contiguous() @ flat
        do = (self.dy @ p["out"]).view(-1, H, HD)
        b = self.dqkv
        d.packed_attention_backward(self.ca, q, k, v, self.o, self.lse, do, b[:, :H], b[:, H:H + G], b[:, H + G:], q_offsets=off,
                                    k_offsets=off, ws=self.ws)
        bf = b.view(-1, (H + 2 * G) * HD)
        out["qkv"] = bf.t().contiguous() @ self.h
        dh = bf @ p["qkv"]
        d.gated_norm_backward(self.c1, p["x0"], None, self.dx1, dh, self.dx, None, scale=m[1], pre_w=p["pre1"], offsets=off, dscale=g[1],
                              dshift=g[0], dpre_w=self.grad["pre1"], ws=self.ws)
        g[5].zero_()
        out["x0"] = self.dx
        return {**out, **self.grad}


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_gradients_of_a_training_step(d, dtype):
    p, q, off, img, seq, n = make(dtype)
    loss, want, xn, old, ref = reference(p, q, off, img, seq, n)
    step = Step(d, dtype, p, q, off, img, xn, old, ref)
    got = step.run()
    torch.cuda.synchronize()
    assert abs(step.loss.item() - loss.item()) <= TOL[dtype] * max(1.0, abs(loss.item()))
    for k, w in want.items():
        g = got[k].double().cpu()
        if k == "mod":
            g, w = g[:, :5], w[:, :5]
        err = ((g - w).abs().max() / w.abs().max()).item()
        assert err <= TOL[dtype], (k, err)


def test_a_captured_step_replays(d):
    """The whole step in one graph: replays between eager runs give the eager run's bits."""
    dtype = torch.bfloat16
    p, q, off, img, seq, n = make(dtype)
    _, _, xn, old, ref = reference(p, q, off, img, seq, n)
    step = Step(d, dtype, p, q, off, img, xn, old, ref)
    names = ["h", "o", "lse", "x1", "h2", "loss", "dv", "dx1", "dy", "dqkv", "dx"]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for _ in range(2):
            step.run()
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    want = [getattr(step, k).clone() for k in names] + [step.grad["mod"].clone()]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step.run()
    for _ in range(3):
        for k in names:
            getattr(step, k).zero_()
        graph.replay()
        torch.cuda.synchronize()
        for k, w in zip(names, want):
            assert torch.equal(getattr(step, k), w), k
        assert torch.equal(step.grad["mod"], want[-1])
        step.run()
        torch.cuda.synchronize()
