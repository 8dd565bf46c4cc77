"""Shared pieces of the policy-update GPU tests: packed inputs, the oracle over a packed batch, and element-wise bounds.

Bounds. A rounding to bf16 is off by at most 2^-8 of the value (half a step of 2^-7), one to fp32 by 2^-24. For
attention, with e_s the error of a score (fp32 products and sums over d terms, the running sum, the exponential):
  o    <= U |o| + (P + 2 e_s) sum p |v|        U: rounding of the output type; P: of p, 2^-8 for bf16, 0 for fp32
  dv   <= U |dv| + (P + e_s) sum p |do|
  ds   <= (P + e_s) |ds| + p (e_dp + e_delta)  e_dp, e_delta: fp32 sums of d products
  dq   <= U |dq| + scale sum_j (bound of ds) |k|,  dk likewise over the rows
"""
import numpy as np
import torch

import seeded_inputs as si
from oracle import policy_oracle as P

F32 = 2.0 ** -24
UNIT = {"bf16": 2.0 ** -8, "f32": F32}


def stored(x, dtype):
    """float64 values the device will hold."""
    return si.as_f64(si.stored(np.asarray(x, np.float32), dtype), dtype)


def to_dev(x, dtype):
    t = torch.from_numpy(np.ascontiguousarray(x)).to(torch.float32)
    return t.to(torch.bfloat16).cuda() if dtype == "bf16" else t.cuda()


def offsets(lengths, start=0):
    return np.concatenate([[start], start + np.cumsum(lengths)]).astype(np.int32)


def i32(x):
    return torch.tensor(np.asarray(x, np.int32), device="cuda")


def attention_reference(q, k, v, q_off, k_off, k_len, scale, causal, dtype, do=None, o=None, lse=None):
    """Over the packed batch: values and bounds, NaN in the rows that belong to no sequence."""
    H, G, d = q.shape[1], k.shape[1], q.shape[2]
    U, Pr = UNIT[dtype], UNIT["bf16"] if dtype == "bf16" else 0.0
    out = {}

    def blank(like):
        return np.full(like.shape, np.nan), np.full(like.shape, np.nan)

    names = ("o", "lse") if do is None else ("dq", "dk", "dv")
    likes = (q, q[:, :, 0]) if do is None else (q, k, v)
    for n, l in zip(names, likes):
        out[n], out[n + "_tol"] = blank(l)
    for i in range(len(k_len)):
        qs, ks = slice(q_off[i], q_off[i + 1]), slice(k_off[i], k_off[i] + k_len[i])
        m, n = qs.stop - qs.start, ks.stop - ks.start
        if do is not None:
            for nm in ("dk", "dv"):
                out[nm][ks] = 0.0
                out[nm + "_tol"][ks] = 0.0
        for j in range(H):
            g = j // (H // G)
            qj, kj, vj = q[qs, j], k[ks, g], v[ks, g]
            big = scale * float((np.abs(qj) @ np.abs(kj).T).max(initial=0.0))
            e_s = (d + 8) * F32 * big + (n + 8) * F32 + 2.0 ** -21
            if do is None:
                oj, lj, p = P.attention(qj, kj, vj, scale, causal)
                out["o"][qs, j], out["lse"][qs, j] = oj, lj
                out["o_tol"][qs, j] = U * np.abs(oj) + (Pr + 2 * e_s) * (p @ np.abs(vj))
                out["lse_tol"][qs, j] = e_s + 2.0 ** -22 * (np.abs(np.where(lj > -np.inf, lj, 0)) + 1)
                continue
            oj, doj = o[qs, j], do[qs, j]
            dq, dk, dv, p, ds = P.attention_gradients(qj, kj, vj, oj, lse[qs, j], doj, scale, causal)
            lj = np.abs(np.where(lse[qs, j] > -np.inf, lse[qs, j], 0.0)).max(initial=0.0)
            e_p = e_s + 2.0 ** -22 * (lj + 1)
            e_dp = (d + 8) * F32 * (np.abs(doj) @ np.abs(vj).T + (np.abs(doj) * np.abs(oj)).sum(1)[:, None])
            b = (Pr + e_p + F32 * 8) * np.abs(ds) + p * e_dp * (1 + Pr)
            out["dq"][qs, j], out["dq_tol"][qs, j] = dq, U * np.abs(dq) + scale * (b + n * F32 * np.abs(ds)) @ np.abs(kj)
            out["dk"][ks, g] += dk
            out["dv"][ks, g] += dv
            out["dk_tol"][ks, g] += scale * (b + m * F32 * np.abs(ds)).T @ np.abs(qj)
            out["dv_tol"][ks, g] += ((Pr + e_p + m * F32) * p).T @ np.abs(doj)
        if do is not None:
            for nm in ("dk", "dv"):   # the heads of a group meet in fp32, the sum is rounded once
                out[nm + "_tol"][ks] += U * np.abs(out[nm][ks])
    return out


def check(got, want, tol, what):
    """Within the bound everywhere (and finite where the reference is, -inf where it is)."""
    rows = ~np.isnan(want)
    assert np.array_equal(np.isneginf(got[rows]), np.isneginf(want[rows])), what
    fin = rows & np.isfinite(want)
    assert np.isfinite(got[fin]).all(), f"{what}: not finite"
    over = np.abs(got[fin] - want[fin]) - (tol[fin] * 1.02 + 1e-37)
    assert over.max(initial=-1.0) <= 0, f"{what}: {over.max():.3e} past the bound {tol[fin][over.argmax()]:.3e}"
