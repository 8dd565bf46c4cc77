"""The end of a policy update and the 8-bit products of the next rollout, as measurable cases.

After the gradients of a policy update come the norm over all of them, clipping by it and the weights' AdamW step; the
new weights are then rounded to 8-bit integers, with a scale for each output channel, and the rollout's linear layers
round their rows to 8-bit integers as well, with a scale for each token, and multiply integers.

A case gives an operator and its sizes. Sizes come from `seeded_inputs.py` (hidden 3072, MLP 12288, 1024 + 256 tokens
at 512x512, 16 seeds, the fp32 model of hidden 256, the weights of a dual-stream block) or are generic.
"""
from __future__ import annotations

import math
import zlib

import torch

own = False            # False: the plain forms below; True: the library's kernels

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
SMALLEST = 2.0 ** -126                 # least scale of a row: the smallest normal fp32 number
MAX_NORM, NORM_EPS = 1.0, 1e-6
LR, BETA1, BETA2, EPS, DECAY, STEP = 1e-4, 0.9, 0.999, 1e-8, 0.01, 7


# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------
def _quant(rows, cols, dtype):
    """Rows to 8-bit integers with a scale each, and the values that those stand for."""
    return {"kind": "quant", "rows": rows, "cols": cols, "dtype": dtype}


def _linear(rows, cin, cout, dtype, act="none", bias=True, given=False):
    """act(x W^T + b) in 8-bit integers; `given`: x comes as integers and scales."""
    return {"kind": "linear", "rows": rows, "in": cin, "out": cout, "dtype": dtype, "act": act, "bias": bias,
            "given": given}


def _grads(kind, hidden, blocks, dtype, params=None, align=64):
    """The gradients (and weights) of dual-stream blocks, each tensor at a multiple of `align` elements."""
    return {"kind": kind, "hidden": hidden, "blocks": blocks, "dtype": dtype, "params": params, "align": align}


def listed():
    cases = {
        # the MLP's hidden row of a single token: the smallest call, all latency
        "quant_token": _quant(1, 12288, "bf16"),
        # the MLP's up projection after an update, from the fp32 master weights
        "quant_weight_f32": _quant(12288, 3072, "f32"),
        # the MLP's hidden rows of a 16-seed group at 512x512
        "quant_rows_512_k16": _quant(20480, 12288, "bf16"),
        # one token through the MLP's up projection: bound by reading the weights
        "linear_token": _linear(1, 3072, 12288, "bf16"),
        # the fused q, k, v projection of a few prompts, rows that are there as integers already
        "linear_prompts_qkv": _linear(333, 3072, 9216, "bf16", given=True),
        # odd sizes in fp32: no dimension fills its tiles, rows of the weights end inside a vector
        "linear_odd_f32": _linear(333, 1001, 515, "f32"),
        # the MLP's down projection of one seed at 512x512: long sums, few tiles
        "linear_down_one_seed": _linear(1280, 12288, 3072, "bf16"),
        # the MLP's up projection with its activation, a 16-seed group at 512x512: the largest product
        "linear_up_512_k16": _linear(20480, 3072, 12288, "bf16", act="gelu"),
        # clipping the gradients of the fp32 model's block: 20 small tensors
        "clip_tiny_f32": _grads("clip", 256, 1, "f32"),
        # clipping the bf16 gradients of a block of hidden 3072, 340 M values
        "clip_block": _grads("clip", 3072, 1, "bf16"),
        # norm and AdamW step of the fp32 model's block
        "update_tiny_f32": _grads("update", 256, 1, "f32", "f32"),
        # norm and AdamW step of a block of hidden 3072: fp32 master weights, bf16 gradients and weights
        "update_block_master": _grads("update", 3072, 1, "bf16", "master"),
    }
    return [{"name": n, **c} for n, c in cases.items()]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """A width: mostly a multiple of 64, now and then any number."""
    n = _log_int(rng, lo, hi)
    return n if rng.random() < 0.3 else max(64, n // 64 * 64)


def draw(rng):
    caps = {}
    for c in listed():
        w = work(c)
        for k in w:
            caps[k] = max(caps.get(k, 0), w[k])
    while True:
        kind = rng.choice(["quant", "linear", "linear", "linear", "clip", "update"])
        dtype = rng.choice(["bf16", "bf16", "f32"])
        if kind == "quant":
            c = _quant(_log_int(rng, 1, 20480), _size(rng, 8, 16384), dtype)
        elif kind == "linear":
            c = _linear(_log_int(rng, 1, 20480), _size(rng, 16, 16384), _size(rng, 8, 16384), dtype,
                        rng.choice(["none", "none", "gelu"]), rng.random() < 0.7, rng.random() < 0.3)
        else:
            params = rng.choice(["f32", "master", "bf16"]) if kind == "update" else None
            c = _grads(kind, _size(rng, 16, 2048), _log_int(rng, 1, 60), dtype, params, rng.choice([64, 64, 1]))
        w = work(c)
        if all(w[k] <= caps[k] for k in w):
            return c


def _shapes(case):
    """(elements) of each tensor: the weights and biases of the two streams of every block."""
    D = case["hidden"]
    stream = [6 * D * D, 6 * D, 3 * D * D, 3 * D, D * D, D, 4 * D * D, 4 * D, 4 * D * D, D]
    return stream * 2 * case["blocks"]


def _places(case):
    """Where each tensor starts in its buffer, and the buffer's length."""
    at, total, align = [], 0, case["align"]
    for n in _shapes(case):
        at.append(total)
        total += -(-n // align) * align
    return at, total


def work(case):
    kind = case["kind"]
    es = 2 if case["dtype"] == "bf16" else 4
    if kind == "quant":
        n = case["rows"] * case["cols"]
        return {"bytes": (2 * es + 1) * n + 4 * case["rows"], "flops": 4 * n}
    if kind == "linear":
        M, K, N = case["rows"], case["in"], case["out"]
        x = M * K + 4 * M if case["given"] else es * M * K
        return {"bytes": x + N * K + 4 * N + es * N * case["bias"] + es * M * N, "flops": 2 * M * N * K}
    n = sum(_shapes(case))
    if kind == "clip":
        return {"bytes": 2 * es * n, "flops": 3 * n}
    weights = {"f32": 8, "bf16": 4, "master": 10}[case["params"]]
    return {"bytes": (es + weights + 16) * n, "flops": 18 * n}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
class _Draws:
    """Named seeded draws on the GPU; each tensor depends on its name and the seed alone."""

    def __init__(self, seed):
        self.seed = seed

    def _gen(self, name):
        return torch.Generator(device="cuda").manual_seed((self.seed * 1000003 + zlib.crc32(name.encode())) & 0x7FFFFFFF)

    def normal(self, name, shape, dtype=torch.float32, std=1.0):
        return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=self._gen(name))

    def rows(self, name, shape, dtype):
        """Activations: rows of unlike size, and a few columns far larger than the rest."""
        x = self.normal(name, shape)
        x *= torch.exp(0.5 * self.normal(name + ".rows", (shape[0], 1)))
        x *= torch.exp(torch.clamp(self.normal(name + ".cols", (1, shape[1])) - 2.0, min=0.0) * 2.0)
        return x.to(dtype)


def _int8_buffer(rows, cols):
    """Rows of 8-bit integers start at multiples of 16 bytes."""
    return torch.empty((rows, -(-cols // 16) * 16), dtype=torch.int8, device="cuda")[:, :cols]


def prepare(case, seed):
    state = _inputs(case, _Draws(seed))
    if own:
        _handles(case, state)
    return state


def _inputs(case, dr):
    dt, kind = DT[case["dtype"]], case["kind"]
    if kind == "quant":
        shape = (case["rows"], case["cols"])
        x = dr.rows("x", shape, dt) if case["dtype"] == "bf16" else dr.normal("x", shape, dt, 0.02)
        return {"case": case, "x": x}
    if kind == "linear":
        M, K, N = case["rows"], case["in"], case["out"]
        st = {"case": case, "x": dr.rows("x", (M, K), dt), "w": _int8_buffer(N, K), "bias": None, "x_scale": None}
        q, st["w_scale"] = _quantized(dr.normal("w", (N, K), torch.float32, 0.02))
        st["w"].copy_(q)
        if case["bias"]:
            st["bias"] = dr.normal("bias", (N,), dt, 0.02)
        if case["given"]:
            q, st["x_scale"] = _quantized(st["x"])
            st["x"] = _int8_buffer(M, K).copy_(q)
        return st
    at, total = _places(case)
    st = {"case": case, "grad": dr.normal("grad", (total,), dt, 1e-3)}
    gap = torch.ones(total, dtype=torch.bool, device="cuda")
    for a, n in zip(at, _shapes(case)):
        gap[a:a + n] = False
    st["grad"].masked_fill_(gap, 0.0)
    if kind == "update":
        st["param"] = dr.normal("param", (total,), DT["bf16" if case["params"] == "bf16" else "f32"], 0.02).masked_fill_(gap, 0.0)
        st["m"] = dr.normal("m", (total,), std=2e-4).masked_fill_(gap, 0.0)
        st["v"] = dr.normal("v", (total,), std=1e-3).square_().mul_(1e-2).masked_fill_(gap, 0.0)
        st["copy"] = st["param"].to(torch.bfloat16) if case["params"] == "master" else None
    return st


def _handles(case, st):
    """What a program that calls the library keeps: outputs, lists of tensors, configurations, workspaces."""
    from paper_2606_19004_amd import ditstep as lib
    if case["kind"] == "quant":
        st["q"], st["values"] = _int8_buffer(*st["x"].shape), torch.empty_like(st["x"])
        st["scale"] = torch.empty(case["rows"], dtype=torch.float32, device="cuda")
    elif case["kind"] == "linear":
        st["y"] = torch.empty((case["rows"], case["out"]), dtype=DT[case["dtype"]], device="cuda")
        st["cfg"] = lib.int8_config(st["x"], st["w"], st["y"], act=case["act"])
        size = lib.int8_matmul_workspace_bytes if case["given"] else lib.int8_linear_workspace_bytes
        st["ws"] = lib.workspace(size(st["cfg"]))
    else:
        at, _ = _places(case)
        parts = lambda t: [t[a:a + n] for a, n in zip(at, _shapes(case))]  # noqa: E731
        st["norm"] = torch.empty(1, dtype=torch.float64, device="cuda")
        st["scale"] = torch.empty(1, dtype=torch.float32, device="cuda")
        st["grads"] = lib.grad_list(parts(st["grad"]))
        st["ws"] = lib.workspace(lib.grad_norm_workspace_bytes(st["grads"]))
        if case["kind"] == "update":
            st["weights"] = lib.adamw_list(parts(st["param"]), parts(st["grad"]), parts(st["m"]), parts(st["v"]),
                                           copies=None if st["copy"] is None else parts(st["copy"]))


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"quant": _own_quant, "linear": _own_linear, "clip": _own_clip, "update": _own_update}[kind](state)
    return {"quant": _plain_quant, "linear": _plain_linear, "clip": _plain_clip, "update": _plain_update}[kind](state)


def _own_quant(st):
    from paper_2606_19004_amd import ditstep as lib
    lib.quantize_rows(st["x"], st["q"], st["scale"], values=st["values"])
    return {"values": st["values"], "scale": st["scale"]}


def _own_linear(st):
    from paper_2606_19004_amd import ditstep as lib
    if st["x_scale"] is None:
        lib.int8_linear(st["cfg"], st["x"], st["w"], st["w_scale"], st["y"], bias=st["bias"], ws=st["ws"])
    else:
        lib.int8_matmul(st["cfg"], st["x"], st["x_scale"], st["w"], st["w_scale"], st["y"], bias=st["bias"], ws=st["ws"])
    return {"y": st["y"]}


def _own_clip(st):
    from paper_2606_19004_amd import ditstep as lib
    lib.grad_norm(st["grads"], MAX_NORM, st["norm"], scale=st["scale"], ws=st["ws"])
    lib.grad_clip(st["grads"], st["scale"])
    return {"norm": st["norm"], "scale": st["scale"], "grad": st["grad"]}


def _own_update(st):
    from paper_2606_19004_amd import ditstep as lib
    lib.grad_norm(st["grads"], MAX_NORM, st["norm"], scale=st["scale"], ws=st["ws"])
    lib.adamw_step(st["weights"], lr=LR, beta1=BETA1, beta2=BETA2, eps=EPS, weight_decay=DECAY, step=STEP, scale=st["scale"])
    return _update_outputs(st, st["norm"], st["scale"])


def _update_outputs(st, norm, scale):
    out = {"norm": norm, "scale": scale, "param": st["param"], "m": st["m"], "v": st["v"]}
    if st["copy"] is not None:
        out["copy"] = st["copy"]
    return out


# --- plain forms ------------------------------------------------------------
def _quantized(x):
    """Integers (as fp64, in -127..127) and scales of the rows of x. The quotient is rounded in 64 bits: in 32 it may
    end up on the wrong side of a half."""
    top = x.abs().amax(-1).double()
    scale = torch.clamp((top / 127).float(), min=SMALLEST)
    return torch.round(x.double() / scale.double()[:, None]), scale


def _plain_quant(st):
    q, scale = _quantized(st["x"])
    return {"values": (q.float() * scale[:, None]).to(st["x"].dtype), "scale": scale}


def _plain_linear(st):
    q, x_scale = (st["x"], st["x_scale"]) if st["x_scale"] is not None else _quantized(st["x"])
    y = torch.matmul(q.float(), st["w"].float().t().contiguous())
    y = y * x_scale[:, None] * st["w_scale"]
    if st["bias"] is not None:
        y = y + st["bias"].float()
    if st["case"]["act"] == "gelu":
        y = 0.5 * y * (1 + torch.tanh(math.sqrt(2 / math.pi) * (y + 0.044715 * y * y * y)))
    return {"y": y.to(DT[st["case"]["dtype"]])}


def _norm_and_scale(grad):
    """The norm in 64 bits: it sums hundreds of millions of squares."""
    norm = grad.double().square().sum().sqrt().reshape(1)
    return norm, torch.clamp(MAX_NORM / (norm + NORM_EPS), max=1.0).float()


def _plain_clip(st):
    norm, scale = _norm_and_scale(st["grad"])
    st["grad"].copy_(st["grad"].float() * scale)
    return {"norm": norm, "scale": scale, "grad": st["grad"]}


def _plain_update(st):
    norm, scale = _norm_and_scale(st["grad"])
    g = st["grad"].float() * scale
    m = BETA1 * st["m"] + (1 - BETA1) * g
    v = BETA2 * st["v"] + (1 - BETA2) * g * g
    step = (m / (1 - BETA1 ** STEP)) / (torch.sqrt(v / (1 - BETA2 ** STEP)) + EPS)
    p = st["param"].float()
    p = p - LR * (step + DECAY * p)
    for name, value in (("param", p), ("m", m), ("v", v), ("copy", p)):
        if st[name] is not None:
            st[name].copy_(value)
    return _update_outputs(st, norm, scale)


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------
def exact(case, seed):
    st = _inputs(case, _Draws(seed))
    f = torch.float64

    def integers(x):
        """Nearest integers to x / scale, by what is left over; the scale is an fp32 number."""
        s = (x.to(f).abs().max(dim=1).values / 127).to(torch.float32).to(f)
        s = torch.maximum(s, torch.tensor(SMALLEST, dtype=f, device="cuda"))[:, None]
        low = torch.floor(x.to(f) / s)
        left = x.to(f) - low * s
        up = (left > s / 2) | ((left == s / 2) & (low % 2 != 0))
        return low + up.to(f), s

    if case["kind"] == "quant":
        q, s = integers(st["x"])
        return {"values": q * s, "scale": s[:, 0]}
    if case["kind"] == "linear":
        q, s = (st["x"].to(f), st["x_scale"].to(f)[:, None]) if case["given"] else integers(st["x"])
        y = (q * s) @ (st["w"].to(f) * st["w_scale"].to(f)[:, None]).t().contiguous()
        if st["bias"] is not None:
            y += st["bias"].to(f)
        if case["act"] == "gelu":
            # z sigmoid(2u) with u the argument of the tanh
            y = y * torch.sigmoid(2 * math.sqrt(2 / math.pi) * y * (1 + 0.044715 * y ** 2))
        return {"y": y}
    g = st["grad"].to(f)
    norm = torch.linalg.vector_norm(g).reshape(1)
    scale = torch.minimum(MAX_NORM / (norm + NORM_EPS), torch.ones_like(norm))
    g *= scale
    if case["kind"] == "clip":
        return {"norm": norm, "scale": scale, "grad": g}
    m = torch.lerp(g, st["m"].to(f), BETA1)
    v = torch.lerp(g ** 2, st["v"].to(f), BETA2)
    m_hat, v_hat = m / -math.expm1(STEP * math.log(BETA1)), v / -math.expm1(STEP * math.log(BETA2))
    p = st["param"].to(f) * (1 - LR * DECAY) - LR * m_hat / (v_hat.sqrt() + EPS)
    out = {"norm": norm, "scale": scale, "param": p, "m": m, "v": v}
    if st["copy"] is not None:
        out["copy"] = p
    return out
