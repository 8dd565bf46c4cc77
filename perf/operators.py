"""Packed attention, the gated norm and the policy loss, as measurable cases.

These are the operators that a policy update adds to the rollout: attention over packed sequences of
different lengths (joint text+image sequences of mixed sizes without a mask, a text encoder's prompts
with a causal one, one new token per sequence against a cache) and its gradients; the residual update
of a block with the norms on both sides of it, and its gradients; the clipped policy loss of one SDE
step with its gradient for the velocity.

A case gives an operator and its sizes; the lengths of its sequences follow from the case alone. Sizes
come from `seeded_inputs.py` (hidden 3072 with 24 heads of 128, 1024 + 256 tokens at 512x512, the fp32
model of hidden 256, 64 latent values per token) or are generic (grouped heads 28/4 and 32/8).
"""
from __future__ import annotations

import math
import random
import zlib

import torch

own = False            # False: the plain forms below; True: the library's kernels

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
LATENT = 64
T, T_NEXT, NOISE = 0.62, 0.57, 0.7
EPS = 1e-6


# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------
def _attn(kind, sequences, lo, hi, mix, heads, kv_heads, head_dim, causal, dtype="bf16", new=0):
    """Sequences of lo..hi keys; as many queries as keys, or `new` queries each when new > 0."""
    return {"kind": kind, "sequences": sequences, "lo": lo, "hi": hi, "mix": mix, "heads": heads,
            "kv_heads": kv_heads, "head_dim": head_dim, "causal": causal, "dtype": dtype, "new": new}


def _norm(kind, sequences, lo, hi, mix, hidden, dtype, post, pre, weights, modulated):
    return {"kind": kind, "sequences": sequences, "lo": lo, "hi": hi, "mix": mix, "hidden": hidden,
            "dtype": dtype, "post": post, "pre": pre, "weights": weights, "modulated": modulated}


def _loss(batch, n, reference):
    return {"kind": "loss", "batch": batch, "n": n, "reference": reference}


def listed():
    cases = {
        # a text encoder over the prompts of a batch: 32 causal sequences of unlike lengths, grouped heads
        "attn_prompts_causal": _attn("attn", 32, 13, 512, 1, 28, 4, 128, True),
        # joint text+image sequences of mixed image sizes (512x512 to 768x768) in one call, no mask
        "attn_joint_mixed": _attn("attn", 8, 1101, 2560, 2, 24, 24, 128, False),
        # one new token of a single sequence against a short cache: the smallest call, all latency
        "attn_token_1x700": _attn("attn", 1, 700, 700, 3, 32, 8, 128, True, new=1),
        # one new token of each of 32 sequences against caches of very unlike lengths: bound by reading them
        "attn_token_32_cache": _attn("attn", 32, 100, 16384, 4, 32, 8, 128, True, new=1),
        # the fp32 model's heads, gradients at ragged lengths: what a numerics check runs
        "attn_grad_f32": _attn("grad", 3, 80, 333, 5, 4, 4, 64, False, "f32"),
        # gradients of the joint attention of four samples at 512x512 with prompts of unlike lengths
        "attn_grad_joint_512": _attn("grad", 4, 1037, 1280, 6, 24, 24, 128, False),
        # gradients of causal attention with grouped heads, one long sequence: the largest call
        "attn_grad_causal_8k": _attn("grad", 1, 8192, 8192, 7, 32, 8, 128, True),
        # the fp32 model's block boundary, one token grid: a small call
        "norm_tiny_f32": _norm("norm", 2, 80, 80, 8, 256, "f32", "none", "layer", False, True),
        # the boundary between attention and MLP of a 16-seed group at 512x512
        "norm_512_k16": _norm("norm", 16, 1280, 1280, 9, 3072, "bf16", "none", "layer", False, True),
        # gradients at a boundary with norms on both sides and their weights, packed samples of unlike lengths
        "norm_grad_packed": _norm("norm_grad", 8, 1037, 1701, 10, 3072, "bf16", "rms", "rms", True, True),
        # one SDE step of a 16-seed group at 512x512
        "loss_512_k16": _loss(16, 1024 * LATENT, False),
        # one SDE step of 24 samples at 1280x1280, held near a reference policy
        "loss_1280_k24": _loss(24, 6400 * LATENT, True),
    }
    return [{"name": n, **c} for n, c in cases.items()]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    caps = {}
    for c in listed():
        w = work(c)
        for k in w:
            caps[k] = max(caps.get(k, 0), w[k])
    while True:
        kind = rng.choice(["attn", "attn", "token", "grad", "grad", "norm", "norm_grad", "loss"])
        mix = rng.randrange(1 << 20)
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        if kind in ("attn", "token", "grad"):
            kv = rng.choice([1, 2, 3, 4, 8, 12])
            heads = kv * rng.choice([1, 1, 2, 4, 5, 7, 8])
            if heads > 40:
                continue
            d = rng.choice([64, 128])
            if kind == "token":
                hi = _log_int(rng, 64, 16384)
                c = _attn("attn", _log_int(rng, 1, 64), max(1, hi // rng.choice([1, 4, 64])), hi, mix, heads, kv, d,
                          True, dtype, new=rng.choice([1, 1, 1, 2, 5]))
                c["lo"] = max(c["lo"], c["new"])
                c["hi"] = max(c["hi"], c["lo"])
            else:
                top = 4096 if dtype == "bf16" else 1024
                hi = _log_int(rng, 16, top)
                c = _attn(kind, _log_int(rng, 1, 24), max(1, hi // rng.choice([1, 2, 16])), hi, mix, heads, kv, d,
                          rng.random() < 0.5, dtype)
        elif kind in ("norm", "norm_grad"):
            hidden = 64 * _log_int(rng, 1, 64)
            if rng.random() < 0.2:
                hidden += rng.choice([-63, -24, 8, 17])
            hi = _log_int(rng, 1, 4096)
            c = _norm(kind, _log_int(rng, 1, 32), max(1, hi // rng.choice([1, 2, 8])), hi, mix, max(8, hidden),
                      dtype, rng.choice(["none", "none", "layer", "rms"]), rng.choice(["layer", "rms"]),
                      rng.random() < 0.5, rng.random() < 0.8)
        else:
            c = _loss(rng.randint(1, 32), LATENT * _log_int(rng, 16, 6400) + rng.choice([0, 0, 0, -3, 1]),
                      rng.random() < 0.5)
        w = work(c)
        if all(w[k] <= caps[k] for k in w):
            return c


def _lengths(case):
    """Keys (or rows) of each sequence, spread over lo..hi on a logarithmic scale."""
    r = random.Random(case["mix"])
    return [_log_int(r, case["lo"], case["hi"]) for _ in range(case["sequences"])]


def work(case):
    if case["kind"] in ("attn", "grad"):
        es = 2 if case["dtype"] == "bf16" else 4
        H, G, d = case["heads"], case["kv_heads"], case["head_dim"]
        pairs = rows = keys = 0
        for n in _lengths(case):
            m = case["new"] or n
            rows, keys = rows + m, keys + n
            pairs += m * n - (m * (m - 1) // 2 if case["causal"] else 0)
        if case["kind"] == "attn":
            return {"bytes": es * d * (2 * rows * H + 2 * keys * G) + 4 * rows * H, "flops": 4 * pairs * H * d}
        # reads q, o, do, k, v and the row sums; writes dq, dk, dv
        return {"bytes": es * d * (4 * rows * H + 4 * keys * G) + 4 * rows * H, "flops": 10 * pairs * H * d}
    if case["kind"] in ("norm", "norm_grad"):
        es = 2 if case["dtype"] == "bf16" else 4
        D, rows = case["hidden"], sum(_lengths(case))
        mod = 3 * 4 * D * case["sequences"] if case["modulated"] else 0
        if case["kind"] == "norm":
            return {"bytes": 4 * es * rows * D + mod, "flops": 12 * rows * D}
        return {"bytes": 6 * es * rows * D + 2 * mod, "flops": 30 * rows * D}
    per = 5 if case["reference"] else 4
    return {"bytes": 4 * per * case["batch"] * case["n"], "flops": 12 * case["batch"] * case["n"]}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
class _Draws:
    """Named seeded draws on the GPU; each tensor depends on its name and the seed alone."""

    def __init__(self, seed):
        self.seed = seed

    def _gen(self, name):
        return torch.Generator(device="cuda").manual_seed((self.seed * 1000003 + zlib.crc32(name.encode())) & 0x7FFFFFFF)

    def normal(self, name, shape, dtype=torch.float32, std=1.0, mean=0.0):
        return torch.empty(shape, dtype=dtype, device="cuda").normal_(mean, std, generator=self._gen(name))


def _offsets(lengths):
    out = [0]
    for n in lengths:
        out.append(out[-1] + n)
    return out


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    return _prepare(case, seed, own)


def _prepare(case, seed, handles):
    """`handles`: also what a program that calls the library keeps, its configuration, workspace and outputs."""
    make = {"attn": _prepare_attn, "grad": _prepare_attn, "norm": _prepare_norm, "norm_grad": _prepare_norm,
            "loss": _prepare_loss}[case["kind"]]
    return make(case, _Draws(seed), handles)


def _prepare_attn(case, dr, handles):
    dt, d, H, G = DT[case["dtype"]], case["head_dim"], case["heads"], case["kv_heads"]
    lens = _lengths(case)
    st = {"case": case, "scale": 1.0 / math.sqrt(d)}
    if case["new"]:
        # a cache that every sequence grows in: its region has room for more keys than it holds
        st["q_off"] = [i * case["new"] for i in range(len(lens) + 1)]
        st["k_off"], st["k_len"] = _offsets([-(-(n + 64) // 64) * 64 for n in lens]), lens
        st["q"] = dr.normal("q", (st["q_off"][-1], H, d), dt)
        st["k"] = dr.normal("k", (st["k_off"][-1], G, d), dt)
        st["v"] = dr.normal("v", (st["k_off"][-1], G, d), dt)
        st["lengths"] = _i32(lens)
    else:
        # q, k and v are slices of one projection's output
        st["q_off"] = st["k_off"] = _offsets(lens)
        st["k_len"], st["lengths"] = lens, None
        qkv = dr.normal("qkv", (st["q_off"][-1], H + 2 * G, d), dt)
        st["q"], st["k"], st["v"] = qkv[:, :H], qkv[:, H:H + G], qkv[:, H + G:]
    st["q_offsets"] = _i32(st["q_off"])
    st["k_offsets"] = st["q_offsets"] if st["k_off"] is st["q_off"] else _i32(st["k_off"])
    if case["kind"] == "grad":
        st["do"] = dr.normal("do", (st["q_off"][-1], H, d), dt)
        st["o"], st["lse"] = _attention(st, torch.float32)
        st["o"] = st["o"].to(dt)
        st["lse"] = st["lse"].float()
    if handles:
        from paper_2606_19004_amd import ditstep as lib
        o = st["o"] if case["kind"] == "grad" else torch.empty((st["q_off"][-1], H, d), dtype=dt, device="cuda")
        cfg = lib.packed_config(st["q"], st["k"], st["v"], o, len(lens), causal=case["causal"], scale=st["scale"],
                                max_q=case["new"] or max(lens))
        st["cfg"] = cfg
        if case["kind"] == "grad":
            dqkv = torch.empty_like(qkv)
            st["dq"], st["dk"], st["dv"] = dqkv[:, :H], dqkv[:, H:H + G], dqkv[:, H + G:]
            st["ws"] = lib.workspace(lib.packed_attention_backward_workspace_bytes(cfg))
        else:
            st["out"] = o
            st["out_lse"] = torch.empty((st["q_off"][-1], H), dtype=torch.float32, device="cuda")
            st["ws"] = lib.workspace(lib.packed_attention_workspace_bytes(cfg))
    return st


def _prepare_norm(case, dr, handles):
    dt, D, S = DT[case["dtype"]], case["hidden"], case["sequences"]
    lens = _lengths(case)
    off = _offsets(lens)
    R = off[-1]
    st = {"case": case, "off": off, "offsets": _i32(off), "x": dr.normal("x", (R, D), dt),
          "y": dr.normal("y", (R, D), dt), "gate": None, "scale": None, "shift": None, "post_w": None, "pre_w": None}
    if case["modulated"]:
        mod = dr.normal("mod", (S, 3, D), torch.float32, 0.6)
        st["shift"], st["scale"], st["gate"] = mod[:, 0], mod[:, 1], mod[:, 2]
    if case["weights"]:
        st["pre_w"] = dr.normal("pre_w", (D,), dt, 0.1, 1.0)
        if case["post"] != "none":
            st["post_w"] = dr.normal("post_w", (D,), dt, 0.1, 1.0)
    if case["kind"] == "norm_grad":
        st["dx_out"], st["dh"] = dr.normal("dx_out", (R, D), dt), dr.normal("dh", (R, D), dt)
    if handles:
        from paper_2606_19004_amd import ditstep as lib
        st["cfg"] = lib.gated_norm_config(st["x"], S, post=case["post"], pre=case["pre"], eps=EPS,
                                          mod_row=3 * D if case["modulated"] else D)
        if case["kind"] == "norm":
            st["x_out"], st["h"] = torch.empty_like(st["x"]), torch.empty_like(st["x"])
        else:
            st["dx"], st["dy"] = torch.empty_like(st["x"]), torch.empty_like(st["x"])
            st["dmod"] = torch.empty((S, 3, D), dtype=torch.float32, device="cuda") if case["modulated"] else None
            st["dpost_w"] = torch.empty(D, device="cuda") if st["post_w"] is not None else None
            st["dpre_w"] = torch.empty(D, device="cuda") if st["pre_w"] is not None else None
            st["ws"] = lib.workspace(lib.gated_norm_backward_workspace_bytes(st["cfg"]))
    return st


def _prepare_loss(case, dr, handles):
    B, n = case["batch"], case["n"]
    x, v = dr.normal("x", (B, n)), dr.normal("v", (B, n))
    h = T_NEXT - T
    sigma = NOISE * math.sqrt(T / (1 - T))
    k = sigma * sigma / (2 * T)
    # the step was taken under a slightly older policy's velocity
    v_old = v + 0.05 * dr.normal("drift", (B, n))
    x_next = x + h * (v_old + k * (x + (1 - T) * v_old)) + sigma * math.sqrt(-h) * dr.normal("eps", (B, n))
    st = {"case": case, "x": x, "v": v, "x_next": x_next, "v_ref": None,
          "adv": dr.normal("adv", (B,)), "clip": (0.2, 0.2), "kl_weight": 0.0}
    st["logp_old"] = _density(x, v_old, x_next).clone()
    if case["reference"]:
        st["v_ref"], st["kl_weight"] = v + 0.1 * dr.normal("ref", (B, n)), 0.04
    if handles:
        from paper_2606_19004_amd import ditstep as lib
        st["loss"] = torch.empty(1, dtype=torch.float64, device="cuda")
        st["logp"], st["ratio"] = (torch.empty(B, dtype=torch.float64, device="cuda") for _ in range(2))
        st["dv"] = torch.empty_like(v)
        st["ws"] = lib.workspace(lib.flow_policy_loss_workspace_bytes(B, n))
    return st


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"attn": _own_attn, "grad": _own_grad, "norm": _own_norm, "norm_grad": _own_norm_grad,
                "loss": _own_loss}[kind](state)
    if kind == "attn":
        o, lse = _attention(state, torch.float32)
        return {"o": o.to(state["q"].dtype), "lse": lse}
    return {"grad": _plain_grad, "norm": _plain_norm, "norm_grad": _plain_norm_grad, "loss": _plain_loss}[kind](state)


def _own_attn(st):
    from paper_2606_19004_amd import ditstep as lib
    lib.packed_attention(st["cfg"], st["q"], st["k"], st["v"], st["out"], lse=st["out_lse"], q_offsets=st["q_offsets"],
                         k_offsets=st["k_offsets"], k_lengths=st["lengths"], ws=st["ws"])
    return {"o": st["out"], "lse": st["out_lse"]}


def _own_grad(st):
    from paper_2606_19004_amd import ditstep as lib
    lib.packed_attention_backward(st["cfg"], st["q"], st["k"], st["v"], st["o"], st["lse"], st["do"], st["dq"],
                                  st["dk"], st["dv"], q_offsets=st["q_offsets"], k_offsets=st["k_offsets"],
                                  k_lengths=st["lengths"], ws=st["ws"])
    return {"dq": st["dq"], "dk": st["dk"], "dv": st["dv"]}


def _own_norm(st):
    from paper_2606_19004_amd import ditstep as lib
    lib.gated_norm(st["cfg"], st["x"], st["y"], st["x_out"], st["h"], gate=st["gate"], scale=st["scale"],
                   shift=st["shift"], post_w=st["post_w"], pre_w=st["pre_w"], offsets=st["offsets"])
    return {"x_out": st["x_out"], "h": st["h"]}


def _own_norm_grad(st):
    from paper_2606_19004_amd import ditstep as lib
    m = st["dmod"]
    dshift, dscale, dgate = (m[:, 0], m[:, 1], m[:, 2]) if m is not None else (None, None, None)
    lib.gated_norm_backward(st["cfg"], st["x"], st["y"], st["dx_out"], st["dh"], st["dx"], st["dy"],
                            gate=st["gate"], scale=st["scale"], post_w=st["post_w"], pre_w=st["pre_w"],
                            offsets=st["offsets"], dgate=dgate, dscale=dscale, dshift=dshift,
                            dpost_w=st["dpost_w"], dpre_w=st["dpre_w"], ws=st["ws"])
    return _norm_outputs(st, st["dx"], st["dy"], dgate, dscale, dshift, st["dpost_w"], st["dpre_w"])


def _own_loss(st):
    from paper_2606_19004_amd import ditstep as lib
    lib.flow_policy_loss(st["x"], st["v"], st["x_next"], st["logp_old"], st["adv"], T, T_NEXT, NOISE, st["loss"],
                         dv=st["dv"], logp=st["logp"], ratio=st["ratio"], v_ref=st["v_ref"], clip_low=st["clip"][0],
                         clip_high=st["clip"][1], kl_weight=st["kl_weight"], ws=st["ws"])
    return {"loss": st["loss"], "logp": st["logp"], "ratio": st["ratio"], "dv": st["dv"]}


# --- plain forms ------------------------------------------------------------
def _sequences(st):
    for i in range(st["case"]["sequences"]):
        yield (slice(st["q_off"][i], st["q_off"][i + 1]), slice(st["k_off"][i], st["k_off"][i] + st["k_len"][i]))


def _visible(m, n):
    """Query i of m sees key j of n where j <= i + n - m."""
    i = torch.arange(m, device="cuda")[:, None]
    return torch.arange(n, device="cuda")[None, :] <= i + (n - m)


def _attention(st, ft):
    """o and the rows' log-sum-exp, not rounded."""
    c = st["case"]
    H, G, d = c["heads"], c["kv_heads"], c["head_dim"]
    o = torch.zeros((st["q"].shape[0], H, d), dtype=ft, device="cuda")
    lse = torch.full((st["q"].shape[0], H), -math.inf, dtype=ft, device="cuda")
    for qs, ks in _sequences(st):
        m, n = qs.stop - qs.start, ks.stop - ks.start
        hidden = ~_visible(m, n) if c["causal"] else None
        for g in range(G):
            hs = slice(g * (H // G), (g + 1) * (H // G))
            q = st["q"][qs, hs].to(ft).transpose(0, 1)
            s = torch.matmul(q, st["k"][ks, g].to(ft).t().contiguous()) * st["scale"]
            if hidden is not None:
                s = s.masked_fill(hidden, -math.inf)
            top = s.amax(-1, keepdim=True)
            p = torch.exp(s - top)
            total = p.sum(-1, keepdim=True)
            o[qs, hs] = (torch.matmul(p, st["v"][ks, g].to(ft)) / total).transpose(0, 1)
            lse[qs, hs] = (top + torch.log(total))[..., 0].t()
    return o, lse


def _attention_gradients(st, ft):
    c = st["case"]
    H, G, d = c["heads"], c["kv_heads"], c["head_dim"]
    dq = torch.zeros((st["q"].shape[0], H, d), dtype=ft, device="cuda")
    dk = torch.zeros((st["k"].shape[0], G, d), dtype=ft, device="cuda")
    dv = torch.zeros_like(dk)
    for qs, ks in _sequences(st):
        m, n = qs.stop - qs.start, ks.stop - ks.start
        hidden = ~_visible(m, n) if c["causal"] else None
        for g in range(G):
            hs = slice(g * (H // G), (g + 1) * (H // G))
            q, do, o = (st[x][qs, hs].to(ft).transpose(0, 1).contiguous() for x in ("q", "do", "o"))
            k, v = st["k"][ks, g].to(ft).contiguous(), st["v"][ks, g].to(ft).contiguous()
            p = torch.exp(torch.matmul(q, k.t().contiguous()) * st["scale"] - st["lse"][qs, hs].to(ft).t()[..., None])
            if hidden is not None:
                p = p.masked_fill(hidden, 0.0)
            dv[ks, g] = torch.matmul(p.reshape(-1, n).t().contiguous(), do.reshape(-1, d))
            ds = p * (torch.matmul(do, v.t().contiguous()) - (do * o).sum(-1, keepdim=True)) * st["scale"]
            dq[qs, hs] = torch.matmul(ds, k).transpose(0, 1)
            dk[ks, g] = torch.matmul(ds.reshape(-1, n).t().contiguous(), q.reshape(-1, d))
    return dq, dk, dv


def _plain_grad(st):
    dt = st["q"].dtype
    return {n: x.to(dt) for n, x in zip(("dq", "dk", "dv"), _attention_gradients(st, torch.float32))}


def _normed(kind, x):
    """(normalised rows, their reciprocal deviations)"""
    if kind == "none":
        return x, None
    c = x - x.mean(-1, keepdim=True) if kind == "layer" else x
    r = torch.rsqrt((c * c).mean(-1, keepdim=True) + EPS)
    return c * r, r


def _normed_gradient(kind, xhat, r, g):
    if kind == "none":
        return g
    out = g - xhat * (g * xhat).mean(-1, keepdim=True)
    if kind == "layer":
        out = out - g.mean(-1, keepdim=True)
    return out * r


def _sequence_of_row(st):
    lens = torch.tensor([b - a for a, b in zip(st["off"], st["off"][1:])], device="cuda")
    return torch.repeat_interleave(torch.arange(len(lens), device="cuda"), lens, output_size=st["off"][-1])


def _plain_norm(st):
    c, seq, f = st["case"], _sequence_of_row(st), torch.float32
    u, _ = _normed(c["post"], st["y"].to(f))
    if st["post_w"] is not None:
        u = u * st["post_w"].to(f)
    if st["gate"] is not None:
        u = u * st["gate"][seq]
    x = st["x"].to(f) + u
    h, _ = _normed(c["pre"], x)
    if st["pre_w"] is not None:
        h = h * st["pre_w"].to(f)
    if st["scale"] is not None:
        h = h * (1 + st["scale"][seq]) + st["shift"][seq]
    return {"x_out": x.to(st["x"].dtype), "h": h.to(st["x"].dtype)}


def _norm_outputs(st, dx, dy, dgate, dscale, dshift, dpost_w, dpre_w):
    out = {"dx": dx, "dy": dy}
    if st["gate"] is not None:
        out.update(dgate=dgate, dscale=dscale, dshift=dshift)
    if dpost_w is not None:
        out["dpost_w"] = dpost_w
    if dpre_w is not None:
        out["dpre_w"] = dpre_w
    return out


def _norm_gradients(st, f):
    """Gradients of x and y, and of the vectors, at x_out = st["x"]."""
    c, seq, S = st["case"], _sequence_of_row(st), st["case"]["sequences"]

    def by_sequence(rows):
        return torch.stack([rows[a:b].sum(0) for a, b in zip(st["off"], st["off"][1:])])

    xhat, r = _normed(c["pre"], st["x"].to(f))
    yhat, ry = _normed(c["post"], st["y"].to(f))
    dh = st["dh"].to(f)
    pre_w = 1.0 if st["pre_w"] is None else st["pre_w"].to(f)
    post_w = 1.0 if st["post_w"] is None else st["post_w"].to(f)
    up = (1 + st["scale"].to(f))[seq] if st["scale"] is not None else 1.0
    gate = st["gate"].to(f)[seq] if st["gate"] is not None else 1.0
    dx = st["dx_out"].to(f) + _normed_gradient(c["pre"], xhat, r, dh * up * pre_w)
    dy = _normed_gradient(c["post"], yhat, ry, dx * gate * post_w)
    dgate, dscale, dshift = by_sequence(dx * yhat * post_w), by_sequence(dh * xhat * pre_w), by_sequence(dh)
    dpost_w = (dx * gate * yhat).sum(0) if st["post_w"] is not None else None
    dpre_w = (dh * up * xhat).sum(0) if st["pre_w"] is not None else None
    return dx, dy, dgate, dscale, dshift, dpost_w, dpre_w


def _plain_norm_grad(st):
    dx, dy, *rest = _norm_gradients(st, torch.float32)
    return _norm_outputs(st, dx.to(st["x"].dtype), dy.to(st["x"].dtype), *rest)


def _step_terms():
    h = T_NEXT - T
    k = NOISE * NOISE / (2 * (1 - T))                     # sigma^2 / (2 t)
    return 1 + h * k, h * (1 + k * (1 - T)), NOISE * NOISE * T / (1 - T) * -h


def _density(x, v, x_next):
    """Log-density of x_next per sample, in 64 bits: the terms are differences of near values, the sums long."""
    cx, cv, var = _step_terms()
    e = x_next.double() - cx * x.double() - cv * v.double()
    return -(e * e).sum(-1) / (2 * var) - 0.5 * x.shape[1] * math.log(2 * math.pi * var)


def _plain_loss(st):
    cx, cv, var = _step_terms()
    B, n = st["x"].shape
    logp = _density(st["x"], st["v"], st["x_next"])
    ratio = torch.exp((logp - st["logp_old"]) / n)
    adv = st["adv"].double()
    lo, hi = 1 - st["clip"][0], 1 + st["clip"][1]
    free, clipped = ratio * adv, ratio.clamp(lo, hi) * adv
    loss = -torch.minimum(free, clipped).sum() / B
    slope = torch.where(free <= clipped, -free, torch.zeros_like(free)) / (B * n)
    e = st["x_next"].double() - cx * st["x"].double() - cv * st["v"].double()
    dv = slope[:, None] * (cv / var) * e
    if st["v_ref"] is not None:
        apart = st["v"].double() - st["v_ref"].double()
        weight = st["kl_weight"] * cv * cv / (var * B * n)
        loss = loss + 0.5 * weight * (apart * apart).sum()
        dv = dv + weight * apart
    return {"loss": loss.reshape(1), "logp": logp, "ratio": ratio, "dv": dv.float()}


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------
def exact(case, seed):
    st = _prepare(case, seed, False)
    f = torch.float64
    if case["kind"] in ("attn", "grad"):
        return _exact_attention(case, st)
    if case["kind"] == "norm":
        return _exact_norm(case, st)
    if case["kind"] == "norm_grad":
        leaves = {n: st[n].to(f).requires_grad_(True) for n in ("y", "gate", "scale", "shift", "post_w", "pre_w")
                  if st[n] is not None}
        # x_out is given: x is what makes it so, and dx is the gradient there
        base = dict(st, **leaves)
        with torch.no_grad():
            step = _exact_rows(case, base, torch.zeros_like(st["x"], dtype=f), leaves["y"])[0]
        x = (st["x"].to(f) - step).requires_grad_(True)
        x_out, h = _exact_rows(case, base, x, leaves["y"])
        total = (x_out * st["dx_out"].to(f)).sum() + (h * st["dh"].to(f)).sum()
        names = ["x"] + list(leaves)
        grads = dict(zip(names, torch.autograd.grad(total, [x] + list(leaves.values()), allow_unused=True)))
        return _norm_outputs(st, grads["x"], grads["y"], grads.get("gate"), grads.get("scale"), grads.get("shift"),
                             grads.get("post_w"), grads.get("pre_w"))
    return _exact_loss(case, st)


def _exact_attention(case, st):
    f, H, G = torch.float64, case["heads"], case["kv_heads"]
    grad = case["kind"] == "grad"
    q, k, v = st["q"].to(f), st["k"].to(f), st["v"].to(f)
    out = ({"dq": torch.zeros_like(q), "dk": torch.zeros_like(k), "dv": torch.zeros_like(v)} if grad else
           {"o": torch.zeros_like(q), "lse": torch.zeros(q.shape[:2], dtype=f, device="cuda")})
    for i, n in enumerate(st["k_len"]):
        a, b, ka = st["q_off"][i], st["q_off"][i + 1], st["k_off"][i]
        for j in range(H):
            g = j * G // H
            qj, kj, vj = q[a:b, j], k[ka:ka + n, g], v[ka:ka + n, g]
            s = (qj @ kj.T) * st["scale"]
            if case["causal"]:
                # the last query sees every key
                s = s + torch.full_like(s, -math.inf).triu(n - (b - a) + 1)
            if not grad:
                out["lse"][a:b, j] = torch.logsumexp(s, -1)
                out["o"][a:b, j] = torch.softmax(s, -1) @ vj
                continue
            doj = st["do"][a:b, j].to(f)
            p = (s - st["lse"][a:b, j].to(f)[:, None]).exp()
            out["dv"][ka:ka + n, g] += p.T @ doj
            delta = torch.linalg.vecdot(doj, st["o"][a:b, j].to(f))
            ds = p * (doj @ vj.T - delta[:, None]) * st["scale"]
            out["dq"][a:b, j] = ds @ kj
            out["dk"][ka:ka + n, g] += ds.T @ qj
    return out


def _exact_rows(case, st, x, y):
    """x_out and h, sequence by sequence."""
    f = torch.float64

    def norm(kind, r, w):
        if kind != "none":
            if kind == "layer":
                r = (r - r.mean(1, keepdim=True)) / (r.var(1, unbiased=False, keepdim=True) + EPS).sqrt()
            else:
                r = r / ((r ** 2).mean(1, keepdim=True) + EPS).sqrt()
        return r if w is None else r * w.to(f)

    xs, hs = [], []
    for i, (a, b) in enumerate(zip(st["off"], st["off"][1:])):
        u = norm(case["post"], y[a:b], st["post_w"])
        xo = x[a:b] + (u if st["gate"] is None else st["gate"][i].to(f) * u)
        h = norm(case["pre"], xo, st["pre_w"])
        if st["scale"] is not None:
            h = h + h * st["scale"][i].to(f) + st["shift"][i].to(f)
        xs.append(xo)
        hs.append(h)
    return torch.cat(xs), torch.cat(hs)


def _exact_norm(case, st):
    x_out, h = _exact_rows(case, st, st["x"].double(), st["y"].double())
    return {"x_out": x_out, "h": h}


def _exact_loss(case, st):
    f = torch.float64
    x, xn = st["x"].to(f), st["x_next"].to(f)
    v = st["v"].to(f).requires_grad_(True)
    h, sigma = T_NEXT - T, NOISE * math.sqrt(T / (1 - T))
    var = sigma ** 2 * -h

    def mean(vel):
        return x + h * (vel + sigma ** 2 / (2 * T) * (x + (1 - T) * vel))

    logp = torch.distributions.Normal(mean(v), math.sqrt(var)).log_prob(xn).sum(1)
    ratio = ((logp - st["logp_old"]) / case["n"]).exp()
    adv = st["adv"].to(f)
    kept = torch.where(adv >= 0, ratio.clamp(max=1 + st["clip"][1]), ratio.clamp(min=1 - st["clip"][0]))
    loss = -(kept * adv).mean()
    if st["v_ref"] is not None:
        apart = (mean(v) - mean(st["v_ref"].to(f))) ** 2 / (2 * var)
        loss = loss + st["kl_weight"] * apart.mean()
    dv, = torch.autograd.grad(loss, v)
    return {"loss": loss.detach().reshape(1), "logp": logp.detach(), "ratio": ratio.detach(), "dv": dv}
