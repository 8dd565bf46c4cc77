"""gated_norm and gated_norm_backward against the float64 oracle.

Bounds: K = (D / 64 + 16) 2^-24 covers the fp32 sums over a row (8 successive terms per lane, then a tree) and
the few operations after them; U is the rounding of the output type (2^-8 or 2^-24 relative). A normalised row is off by at
most 4 K (|xhat| + mean|x| r + 1); what follows from it is multiplied through. Vector gradients add rows 2^-24 for their sums."""
import numpy as np
import pytest
import torch

from oracle import policy_oracle as P
from tests.gpu_util import host64
from tests.policy_util import F32, UNIT, check, i32, offsets, stored, to_dev

pytestmark = pytest.mark.gpu
EPS = 1e-5


@pytest.fixture(scope="module")
def d():
    from paper_2606_19004_amd import ditstep
    return ditstep


class Problem:
    def __init__(self, d, dtype, D, lengths, post, pre, weights=True, modulated=True, branch=True, alpha=1.0, pad=0, lead=0,
                 tail=0, seed=0, mean=0.0):
        rng = np.random.default_rng(seed)
        S = len(lengths)
        self.d, self.dtype, self.D, self.lengths, self.post, self.pre, self.alpha = d, dtype, D, lengths, post, pre, alpha
        self.off = offsets(lengths, lead)
        R = int(self.off[-1]) + tail
        self.R, self.S, self.pad, self.branch = R, S, pad, branch

        def rows():
            return stored(mean + rng.standard_normal((R, D)), dtype)

        self.x, self.y, self.dxo, self.dh = rows(), rows(), rows(), rows()
        f32 = lambda *s: rng.standard_normal(s).astype(np.float32).astype(np.float64)  # noqa: E731
        self.gate, self.scale, self.shift = (f32(S, D), f32(S, D), f32(S, D)) if modulated else (None,) * 3
        self.post_w = stored(1 + 0.2 * rng.standard_normal(D), dtype) if weights else None
        self.pre_w = stored(1 + 0.2 * rng.standard_normal(D), dtype) if weights else None
        self.mod_row = 3 * D + pad
        self.offsets = i32(self.off)

    def rows_dev(self, x):
        """Row stride D + pad."""
        buf = torch.full((self.R, self.D + self.pad), 7.0, dtype=torch.bfloat16 if self.dtype == "bf16" else torch.float32, device="cuda")
        if x is not None:
            buf[:, :self.D] = to_dev(x, self.dtype)
        return buf[:, :self.D]

    def mods(self, values=True):
        buf = torch.full((self.S, self.mod_row), 7.0, device="cuda")
        out = [buf[:, i * self.D:(i + 1) * self.D] for i in range(3)]
        if not values:
            return out
        if self.gate is None:
            return [None] * 3
        for t, v in zip(out, (self.gate, self.scale, self.shift)):
            t.copy_(torch.from_numpy(v))
        return out

    def cfg(self, x):
        return self.d.gated_norm_config(x, self.S, self.post, self.pre, EPS, self.alpha, mod_row=self.mod_row)

    def vec(self, v, i, default):
        return v[i] if v is not None else np.full(self.D, default)

    def weights_dev(self):
        return [to_dev(w, self.dtype) if w is not None else None for w in (self.post_w, self.pre_w)]

    def hat(self, kind, x, K):
        h, r = P.norm(kind, x, EPS)
        return h, r, (4 * K * (np.abs(h) + np.abs(x).mean(1, keepdims=True) * r + 1) if kind != "none" else 0.0 * h)

    def check_forward(self, in_place=False):
        K, U = (self.D / 64 + 16) * F32, UNIT[self.dtype]
        x, y = self.rows_dev(self.x), self.rows_dev(self.y) if self.branch else None
        xo, h = (x if in_place else self.rows_dev(None)), self.rows_dev(None)
        gate, scale, shift = self.mods()
        pw, rw = self.weights_dev()
        self.d.gated_norm(self.cfg(x), x, y, xo, h, gate=gate, scale=scale, shift=shift, post_w=pw, pre_w=rw, offsets=self.offsets)
        torch.cuda.synchronize()
        gx, gh = host64(xo.contiguous()), host64(h.contiguous())
        ones, zeros = np.ones(self.D), np.zeros(self.D)
        pw, rw = (self.post_w if self.post_w is not None else ones), (self.pre_w if self.pre_w is not None else ones)
        seen = np.zeros(self.R, bool)
        for i, (a, b) in enumerate(zip(self.off, self.off[1:])):
            seen[a:b] = True
            if a == b:
                continue
            g, s, t = self.vec(self.gate, i, 1.0), self.vec(self.scale, i, 0.0), self.vec(self.shift, i, 0.0)
            yi = self.y[a:b] if self.branch else None
            wx, wh = P.gated_norm(self.x[a:b], yi, g, s, t, pw, rw, self.post, self.pre, EPS, self.alpha)
            ex = 4 * F32 * np.abs(self.alpha * self.x[a:b])
            if self.branch:
                u, _, eu = self.hat(self.post, yi, K)
                ex = ex + np.abs(g * pw) * (eu + 8 * F32 * np.abs(u))
            check(gx[a:b], wx, U * np.abs(wx) + ex, "x_out")
            xh, r, eh = self.hat(self.pre, wx, K)
            if self.pre != "none":     # r (1 + xhat^2 + mean terms) times the error of x_out
                eh = eh + r * (ex + ex.mean(1, keepdims=True)) + np.abs(xh) * r * np.sqrt((ex * ex).mean(1, keepdims=True))
            else:
                eh = ex
            check(gh[a:b], wh, U * np.abs(wh) + np.abs(rw * (1 + s)) * (eh + 8 * F32 * np.abs(xh)) + 4 * F32 * np.abs(t), "h")
        if not in_place:
            assert np.all(gx[~seen] == 7.0)
        assert np.all(gh[~seen] == 7.0)
        if self.pad:
            base = h._base if h._base is not None else h
            assert torch.all(base[:, self.D:] == 7.0)

    def check_backward(self, rows_only=False):
        K, U = (self.D / 64 + 16) * F32, UNIT[self.dtype]
        x, y = self.rows_dev(self.x), self.rows_dev(self.y) if self.branch else None
        dxo, dh = self.rows_dev(self.dxo), self.rows_dev(self.dh)
        dx, dy = self.rows_dev(None), self.rows_dev(None) if self.branch else None
        gate, scale, _ = self.mods()
        dgate, dscale, dshift = self.mods(False)
        pw, rw = self.weights_dev()
        dpw, drw = torch.full((self.D,), 7.0, device="cuda"), torch.full((self.D,), 7.0, device="cuda")
        cfg = self.cfg(x)
        ws = self.d.workspace(self.d.gated_norm_backward_workspace_bytes(cfg)).fill_(255)
        vectors = {} if rows_only else dict(dgate=dgate if self.branch else None, dscale=dscale, dshift=dshift,
                                            dpost_w=dpw if self.branch else None, dpre_w=drw)
        self.d.gated_norm_backward(cfg, x, y, dxo, dh, dx, dy, gate=gate, scale=scale, post_w=pw, pre_w=rw,
                                   offsets=self.offsets, ws=ws, **vectors)
        torch.cuda.synchronize()
        got = {n: host64(t.contiguous()) for n, t in (("dx", dx), ("dy", dy), ("dgate", dgate), ("dscale", dscale),
                                                       ("dshift", dshift), ("dpost_w", dpw), ("dpre_w", drw)) if t is not None}
        ones = np.ones(self.D)
        pw, rw = (self.post_w if self.post_w is not None else ones), (self.pre_w if self.pre_w is not None else ones)
        total = {n: (np.zeros(self.D), np.zeros(self.D)) for n in ("dpost_w", "dpre_w")}
        seen = np.zeros(self.R, bool)
        for i, (a, b) in enumerate(zip(self.off, self.off[1:])):
            seen[a:b] = True
            n = b - a
            xi, yi, dxi, dhi = self.x[a:b], self.y[a:b] if self.branch else None, self.dxo[a:b], self.dh[a:b]
            g, s = self.vec(self.gate, i, 1.0), self.vec(self.scale, i, 0.0)
            if n == 0:
                if not rows_only:
                    for nm in ("dscale", "dshift") + (("dgate",) if self.branch else ()):
                        assert np.all(got[nm][i] == 0.0), nm
                continue
            w = P.gated_norm_gradients(xi, yi, g, s, pw, rw, dxi, dhi, self.post, self.pre, EPS, self.alpha)
            xh, r, exh = self.hat(self.pre, xi, K)

            def back(kind, hat, r, e_hat, grad, e_grad):
                """bound of norm_gradient, given those of the row and of the incoming gradient"""
                if kind == "none":
                    return e_grad
                m = np.abs(grad).mean(1, keepdims=True)
                mh = np.abs(grad * hat).mean(1, keepdims=True)
                size = np.abs(grad) + m + np.abs(hat) * mh
                e = e_grad + e_grad.mean(1, keepdims=True) + np.abs(hat) * (e_grad * np.abs(hat)).mean(1, keepdims=True)
                e = e + e_hat * mh + np.abs(hat) * (np.abs(grad) * e_hat).mean(1, keepdims=True)
                return r * (e + 8 * K * (1 + np.abs(xi).mean(1, keepdims=True) * r) * size)

            gx = dhi * (1 + s) * rw
            et = 4 * F32 * np.abs(dxi) + back(self.pre, xh, r, exh, gx, 4 * F32 * np.abs(gx))
            check(got["dx"][a:b], w["dx"], U * np.abs(w["dx"]) + np.abs(self.alpha) * (et + 4 * F32 * np.abs(w["dx"])), "dx")
            t = w["dx"] / self.alpha
            if self.branch:
                yh, ry, eyh = self.hat(self.post, yi, K)
                gy, egy = t * g * pw, np.abs(g * pw) * (et + 4 * F32 * np.abs(t))
                check(got["dy"][a:b], w["dy"], U * np.abs(w["dy"]) + back(self.post, yh, ry, eyh, gy, egy), "dy")
            if rows_only:
                continue
            sums = (n + 16) * F32
            check(got["dshift"][i], w["dshift"], sums * np.abs(dhi).sum(0), "dshift")
            ep = (np.abs(dhi) * exh).sum(0) + sums * np.abs(dhi * xh).sum(0)
            check(got["dscale"][i], w["dscale"], np.abs(rw) * ep, "dscale")
            total["dpre_w"][0][:] += w["dpre_w"]
            total["dpre_w"][1][:] += np.abs(1 + s) * ep + F32 * self.S * np.abs(w["dpre_w"])
            if self.branch:
                eq = (np.abs(t) * eyh + et * np.abs(yh)).sum(0) + sums * np.abs(t * yh).sum(0)
                check(got["dgate"][i], w["dgate"], np.abs(pw) * eq, "dgate")
                total["dpost_w"][0][:] += w["dpost_w"]
                total["dpost_w"][1][:] += np.abs(g) * eq + F32 * self.S * np.abs(w["dpost_w"])
        assert np.all(got["dx"][~seen] == 7.0)
        if not rows_only:
            check(got["dpre_w"], total["dpre_w"][0], total["dpre_w"][1] + 1e-30, "dpre_w")
            if self.branch:
                check(got["dpost_w"], total["dpost_w"][0], total["dpost_w"][1] + 1e-30, "dpost_w")


KINDS = [("none", "layer"), ("layer", "rms"), ("rms", "layer"), ("rms", "rms"), ("none", "none")]
SIZES = [(256, [80, 80]), (8, [3, 1]), (64, [1, 0, 200]), (520, [37, 5]), (1023, [9, 4]), (3, [70]), (513, [2]), (4096, [5, 12]),
         (8192, [3]), (8191, [2]), (192, [1]), (257, [6, 30]), (512, [40, 3]), (300, [20])]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("post,pre", KINDS)
@pytest.mark.parametrize("D,lengths", SIZES)
def test_forward_and_backward(d, dtype, post, pre, D, lengths):
    p = Problem(d, dtype, D, lengths, post, pre, lead=2, tail=1, seed=D, alpha=0.75)
    p.check_forward()
    p.check_backward()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kw", [dict(weights=False), dict(modulated=False), dict(weights=False, modulated=False), dict(branch=False),
                                dict(pad=8), dict(pad=3), dict(mean=20.0)])
def test_optional_inputs_and_strides(d, dtype, kw):
    p = Problem(d, dtype, 320, [33, 7], "rms", "layer", seed=4, **kw)
    p.check_forward()
    p.check_backward()


def test_in_place_and_rows_alone(d):
    p = Problem(d, "bf16", 640, [50, 20], "none", "layer", seed=8)
    p.check_forward(in_place=True)
    p.check_backward(rows_only=True)


def test_many_sequences_and_long_ones(d):
    rng = np.random.default_rng(0)
    Problem(d, "f32", 64, list(rng.integers(0, 6, 200)), "rms", "layer", seed=1).check_forward()
    Problem(d, "f32", 64, list(rng.integers(0, 6, 200)), "rms", "layer", seed=1).check_backward()
    p = Problem(d, "bf16", 128, [3000, 1, 1500], "layer", "rms", seed=2)
    p.check_forward()
    p.check_backward()


def test_equal_lengths_need_no_offsets(d):
    p = Problem(d, "bf16", 256, [40, 40, 40], "rms", "layer", seed=3)
    p.offsets = None
    p.check_forward()
    p.check_backward()


def test_bad_offsets_stay_inside_the_tensors(d):
    p = Problem(d, "bf16", 256, [40, 40], "rms", "layer", seed=3)
    x, xo, h = p.rows_dev(p.x), p.rows_dev(None), p.rows_dev(None)
    ws = d.workspace(d.gated_norm_backward_workspace_bytes(p.cfg(x)))
    dg, ds, dt = p.mods(False)
    for off in ([-9, 90, 10], [70, 10, 1000]):
        d.gated_norm(p.cfg(x), x, xo, xo, h, offsets=i32(off))
        d.gated_norm_backward(p.cfg(x), x, p.rows_dev(p.y), xo, h, None, None, offsets=i32(off), dgate=dg, dscale=ds, dshift=dt, ws=ws)
        torch.cuda.synchronize()


def test_dx_may_replace_dx_out_and_runs_repeat(d):
    p = Problem(d, "bf16", 1024, [65, 30], "rms", "rms", seed=6)
    x, y, dh = p.rows_dev(p.x), p.rows_dev(p.y), p.rows_dev(p.dh)
    g, s, _ = p.mods()
    cfg = p.cfg(x)
    ws = d.workspace(d.gated_norm_backward_workspace_bytes(cfg))
    outs = []
    for shared in (False, True, True):
        dxo = p.rows_dev(p.dxo)
        dx = dxo if shared else p.rows_dev(None)
        dy = p.rows_dev(None)
        v = p.mods(False)
        d.gated_norm_backward(cfg, x, y, dxo, dh, dx, dy, gate=g, scale=s, offsets=p.offsets, dgate=v[0], dscale=v[1], dshift=v[2], ws=ws)
        outs.append([t.contiguous() for t in (dx, dy, *v)])
    torch.cuda.synchronize()
    for o in outs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(outs[0], o))


def test_graph_replays_match_eager(d):
    p = Problem(d, "bf16", 512, [65, 30], "rms", "rms", seed=6)
    x, y, dxo, dh, dx, dy, xo, h = (p.rows_dev(v) for v in (p.x, p.y, p.dxo, p.dh, None, None, None, None))
    g, s, t = p.mods()
    v = p.mods(False)
    dw = [torch.zeros(p.D, device="cuda") for _ in range(2)]
    cfg = p.cfg(x)
    ws = d.workspace(d.gated_norm_backward_workspace_bytes(cfg))

    def both():
        d.gated_norm(cfg, x, y, xo, h, gate=g, scale=s, shift=t, offsets=p.offsets)
        d.gated_norm_backward(cfg, xo, y, dxo, dh, dx, dy, gate=g, scale=s, offsets=p.offsets, dgate=v[0], dscale=v[1],
                              dshift=v[2], dpost_w=dw[0], dpre_w=dw[1], ws=ws)

    both()
    outs = [xo, h, dx, dy, *v, *dw]
    want = [o.clone() for o in outs]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for _ in range(3):
        for o in outs:
            o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))
        both()


def test_no_rows(d):
    """Sequences without rows have gradients of zero; no sequence and no row is a call that writes the weights' zeros."""
    for S in (3, 0):
        x = torch.empty((0, 64), device="cuda")
        cfg = d.gated_norm_config(x, S, "rms", "layer")
        y = torch.empty((0, 64), device="cuda")
        v = [torch.full((max(S, 1), 64), 7.0, device="cuda") for _ in range(3)]
        w = [torch.full((64,), 7.0, device="cuda") for _ in range(2)]
        ws = d.workspace(d.gated_norm_backward_workspace_bytes(cfg))
        d.gated_norm(cfg, x, y, x, y)
        one = torch.zeros((1, 64), device="cuda")     # (an empty tensor has no address)
        d.gated_norm_backward(cfg, one, one, one, one, one, one, dgate=v[0], dscale=v[1], dshift=v[2], dpost_w=w[0], dpre_w=w[1], ws=ws)
        torch.cuda.synchronize()
        for t in v:
            assert torch.all(t[:S] == 0.0) and torch.all(t[S:] == 7.0)
        assert all(torch.all(t == 0.0) for t in w)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [258, 259, 260, 261, 262, 263, 509, 517, 1, 2, 5, 7, 13, 246, 1535])
def test_every_end_of_a_row(d, dtype, D):
    """Rows whose last lane holds one to seven elements, one wave and several; what lies behind a row stays."""
    for pad in (0, 3):
        p = Problem(d, dtype, D, [9, 0, 26], "rms", "layer", seed=D, lead=1, tail=2, **({"pad": pad} if pad else {}))
        p.check_forward()
        p.check_backward()


@pytest.mark.parametrize("D", [64, 320])
@pytest.mark.parametrize("count", [65, 257, 600])
def test_hundreds_of_sequences(d, D, count):
    lengths = np.random.default_rng(count).integers(0, 6, count)
    lengths[0], lengths[-1] = 0, 2
    p = Problem(d, "bf16", D, list(lengths), "rms", "layer", seed=count, lead=1, tail=2)
    p.check_forward()
    p.check_backward()
