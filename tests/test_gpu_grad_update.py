"""grad_norm, grad_clip and adamw_step against the oracle.

norm: squares are exact in fp64 and their sum of n terms is off by at most n 2^-53 of itself (in the worst order; the root halves
that), plus the root's rounding: (n / 2 + 2) 2^-53. scale: fp64, one rounding to fp32. clip: one product and one rounding to the
type, 2^-24 + U of the value.
adamw: m = b1 m + r1 g with g = s grad: constants and products are off by 2^-24 each, at most 5 for either term, so
5 (|b1 m| + |r1 g|) 2^-24; v the same with 7. The step's quotient adds 2^-24 for each of: step1, the root (half of v's error,
and its own), root2, the product and sum under it, the quotient and the product: 10 with m's and v's own relative errors, where
cancellation in m is counted by m's absolute bound; p: 3 more on the whole, then one rounding to its type."""
import math

import numpy as np
import pytest
import torch

from oracle import update_oracle as U
from tests.gpu_util import host64
from tests.policy_util import F32, UNIT
from tests.test_gpu_policy_guards import Guarded

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
HYPER = dict(lr=1e-2, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.1, step=3)


@pytest.fixture(scope="module")
def d():
    from paper_2606_19004_amd import ditstep
    return ditstep


def lists(name):
    """(elements of each tensor): one element, odd ones, empty ones among them, more than a launch's table, one long one."""
    rng = np.random.default_rng(7)
    return {"one": [1], "few": [5, 1, 8, 7, 0, 4096, 4097, 2048, 33], "empty": [0, 0], "none": [],
            "odd": [int(n) for n in rng.integers(1, 9000, 60)], "many": [int(n) for n in rng.integers(0, 300, 1000)],
            "long": [3_000_001, 5, 1_000_000]}[name]


def spread(m, counts, dtypes, seed, shift=1):
    """Tensors of the given lengths, each between guard bands, at addresses that its type allows and 16 does not."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    if len(counts) > 200:   # one buffer for all
        flat = {t: torch.randn(sum(counts), generator=g, device="cuda").to(t) for t in set(dtypes)}
        at = np.concatenate([[0], np.cumsum(counts)])
        return [flat[dtypes[i % len(dtypes)]][at[i]:at[i] + n] for i, n in enumerate(counts)]
    out = []
    for i, n in enumerate(counts):
        t = m.empty(n + shift, dtype=dtypes[i % len(dtypes)])[shift:]
        t.copy_(torch.randn(n, generator=g, device="cuda") * 10.0 ** (i % 5 - 2))
        out.append(t)
    return out


KINDS = {"bf16": [torch.bfloat16], "f32": [torch.float32], "mixed": [torch.bfloat16, torch.float32, torch.float32]}


def outputs():
    return torch.full((1,), -7.0, dtype=torch.float64, device="cuda"), torch.full((1,), -7.0, device="cuda")


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("name", ["one", "few", "empty", "none", "odd", "many", "long"])
def test_norm_and_clip(d, name, kind):
    counts = lists(name)
    m = Guarded()
    grads = spread(m, counts, KINDS[kind], 3)
    before = [host64(g) for g in grads]
    gl = d.grad_list(grads)
    for max_norm in (1.0, math.inf, 0.0):
        for g, b in zip(grads, before):
            g.copy_(torch.from_numpy(b))
        norm, scale = outputs()
        d.grad_norm(gl, max_norm, norm, scale, ws=m.empty(d.grad_norm_workspace_bytes(gl), dtype=torch.uint8))
        d.grad_clip(gl, scale)
        m.check()
        want, k = U.grad_norm(before, max_norm)
        assert abs(float(norm) - want) <= (sum(counts) / 2 + 2) * 2.0 ** -53 * want
        assert abs(float(scale) - k) <= (F32 + sum(counts) * 2.0 ** -53) * k
        for g, b in zip(grads, before):
            u = UNIT["bf16" if g.dtype == torch.bfloat16 else "f32"] if float(scale) != 1.0 else 0.0
            v = b * float(scale)
            assert (np.abs(host64(g) - v) <= (F32 * (u > 0) + u) * np.abs(v) + (2.0 ** -133 if u else 0.0)).all()


def test_norm_of_large_and_small_gradients(d):
    """Squares past fp32's range, below it, and a few large values among many small ones."""
    for fill, n in ((3e38, 1000), (1e-40, 1000), (1e-30, 100000)):
        g = torch.full((n,), fill, device="cuda")
        gl = d.grad_list([g])
        norm, scale = outputs()
        d.grad_norm(gl, 1.0, norm, scale, ws=d.workspace(d.grad_norm_workspace_bytes(gl)))
        want = U.grad_norm([host64(g)], 1.0)
        assert abs(float(norm) - want[0]) <= n * 2.0 ** -53 * want[0]
        # a scale below the least normal number, 2^-126 (1 / 9.5e39 here), is a multiple of 2^-149: its rounding is off by 2^-150 at most
        assert abs(float(scale) - want[1]) <= max(F32 * want[1], 2.0 ** -150)
    g = torch.full((1 << 22,), 1e-4, device="cuda")
    g[12345] = 100.0
    gl = d.grad_list([g])
    d.grad_norm(gl, 1.0, norm, None, ws=d.workspace(d.grad_norm_workspace_bytes(gl)))
    assert abs(float(norm) - U.grad_norm([host64(g)], 1.0)[0]) <= (1 << 22) * 2.0 ** -53 * 101


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("at", [(0, 0), (2, 4096), (2, 4999), (1, 0)])
def test_gradients_that_are_not_finite(d, bad, at):
    """The scale is NaN, an update changes nothing, clipping makes every gradient NaN."""
    grads = [torch.randn(n, device="cuda").to(t) for n, t in ((700, torch.bfloat16), (1, torch.float32), (5000, torch.float32))]
    grads[at[0]][at[1]] = bad
    gl = d.grad_list(grads)
    norm, scale = outputs()
    d.grad_norm(gl, 1.0, norm, scale, ws=d.workspace(d.grad_norm_workspace_bytes(gl)))
    assert math.isnan(float(scale)) and not math.isfinite(float(norm))
    p, m, v = ([torch.rand(g.shape, device="cuda") for g in grads] for _ in range(3))
    copies = [t.to(torch.bfloat16) + 1 for t in p]
    kept = [t.clone() for t in p + m + v + copies]
    d.adamw_step(d.adamw_list(p, grads, m, v, copies), scale=scale, **HYPER)
    assert all(torch.equal(a, b) for a, b in zip(p + m + v + copies, kept))
    d.grad_clip(gl, scale)
    assert all(torch.isnan(g.float()).all() for g in grads)


def check_adam(new, old, scale, h, step):
    """new: tensors (p, m, v, copy) after the call; old: float64 (p, g, m, v) before it."""
    p, g, m, v = old
    wp, wm, wv = U.adamw(p, g, m, v, h["lr"], h["beta1"], h["beta2"], h["eps"], h["weight_decay"], step, scale)
    gs = scale * g
    em = 5 * F32 * (np.abs(h["beta1"] * m) + np.abs((1 - h["beta1"]) * gs)) + 2.0 ** -148
    ev = 7 * F32 * wv + 2.0 ** -147
    assert (np.abs(host64(new[1]) - wm) <= em * 1.01).all()
    assert (np.abs(host64(new[2]) - wv) <= ev * 1.01).all()
    c1, c2 = 1 - h["beta1"] ** step, 1 - h["beta2"] ** step
    den = np.sqrt(wv / c2) + h["eps"]
    # a root of what is off by ev is off by at most sqrt(ev), and by ev / (2 root)
    er = np.minimum(np.sqrt(ev / c2), ev / np.maximum(2 * np.sqrt(wv * c2), 1e-300))
    low = np.maximum(den - er, den / 2)
    # (|lr|: the size of the step's error is that of its factors, whatever their signs)
    e = abs(h["lr"]) * ((em / c1 + np.abs(wm / c1) * er / low) / low + 10 * F32 * np.abs(wm / c1) / den) + 3 * F32 * (np.abs(wp) + np.abs(p))
    u = UNIT["bf16" if new[0].dtype == torch.bfloat16 else "f32"]
    assert (np.abs(host64(new[0]) - wp) <= (e + u * (np.abs(wp) + e)) * 1.01 + 2.0 ** -133).all()
    if new[3] is not None:
        assert torch.equal(new[3], new[0].to(torch.bfloat16))


@pytest.mark.parametrize("params", TYPES)
@pytest.mark.parametrize("grads", TYPES)
@pytest.mark.parametrize("name", ["one", "few", "empty", "none", "odd", "many", "long"])
def test_adamw(d, name, params, grads):
    counts = lists(name)
    m = Guarded()
    p, g = spread(m, counts, [TYPES[params]], 1), spread(m, counts, [TYPES[grads]], 2, shift=3)
    a, b = spread(m, counts, [torch.float32], 3, shift=0), spread(m, counts, [torch.float32], 4, shift=2)
    for t in b:
        t.square_()
    copies = [c if i % 3 else None for i, c in enumerate(spread(m, counts, [torch.bfloat16], 5))]
    old = [[host64(t) for t in row] for row in zip(p, g, a, b)]
    scale = torch.tensor([0.37], device="cuda")
    w = d.adamw_list(p, g, a, b, copies)
    d.adamw_step(w, scale=scale, **HYPER)
    m.check()
    for row, before in zip(zip(p, a, b, copies), old):
        check_adam(row, before, float(scale), HYPER, 3)
    for t, before in zip(g, old):
        assert np.array_equal(host64(t), before[1])


@pytest.mark.parametrize("change", [dict(beta1=0.0), dict(beta2=0.0), dict(eps=0.0, step=1), dict(weight_decay=0.0), dict(step=1), dict(step=10 ** 9),
                                    dict(lr=0.0), dict(beta1=0.5, beta2=0.999999, step=2), dict(lr=-1e-3)])
def test_adamw_settings(d, change):
    h = {**HYPER, **change}
    n = 3001
    rng = np.random.default_rng(9)
    old = [rng.normal(size=n), rng.normal(size=n), rng.normal(size=n), rng.normal(size=n) ** 2]
    old = [x.astype(np.float32).astype(np.float64) for x in old]
    for on_device in (False, True):
        p, g, m, v = (torch.from_numpy(x).float().cuda() for x in old)
        w = d.adamw_list([p], [g], [m], [v])
        if on_device:
            d.adamw_step(w, step_dev=torch.tensor([h["step"]], device="cuda"), **{**h, "step": 0})
        else:
            d.adamw_step(w, **h)
        check_adam((p, m, v, None), old, 1.0, h, h["step"])


@pytest.mark.parametrize("step", [0, -1, -2 ** 63])
def test_a_device_step_below_1_changes_nothing(d, step):
    tensors = [torch.randn(5000, device="cuda") for _ in range(4)]
    tensors[3].square_()
    copy = torch.zeros(5000, dtype=torch.bfloat16, device="cuda")
    old = [t.clone() for t in tensors] + [copy.clone()]
    d.adamw_step(d.adamw_list(*([t] for t in tensors), [copy]), step_dev=torch.tensor([step], device="cuda"), **{**HYPER, "step": 0})
    for t, before in zip([*tensors, copy], old):
        assert torch.equal(t, before)


def test_a_small_decay_is_not_lost(d):
    """lr weight_decay = 2^-27, below what 1 - lr weight_decay can hold, beside steps of unlike sizes. p lies in [64, 128), where a unit is 2^-17:
    the decay is 0.094 units on average and turns the rounding of the weights whose step ends that near a half. So the weights move, on average, by
    what the float64 results move when each is rounded once (which is less than the decay where many steps are below half a unit, and those
    of 0.1 and less are lost whatever the kernel does). A weight can differ from that only where its exact value lies within the error e of its
    step from a half, a share of 2 e / unit of them: e is lr times 12 roundings of the quotient and of the decay, each 2^-24."""
    n, lr, decay, unit = 1 << 20, 2.0 ** -15, 2.0 ** -12, 2.0 ** -17
    g = torch.Generator(device="cuda").manual_seed(2)
    start, grad, mean, square = 64 * torch.rand(n, generator=g, device="cuda") + 64, *(torch.randn(n, generator=g, device="cuda") for _ in range(3))
    out, want = [], []
    for wd in (0.0, decay):
        p, m, v = start.clone(), mean.clone(), square.square() + 0.1
        exact = U.adamw(host64(p), host64(grad), host64(m), host64(v), lr, 0.9, 0.999, 1e-8, wd, 5)[0]
        want.append(exact.astype(np.float32).astype(np.float64))
        d.adamw_step(d.adamw_list([p], [grad], [m], [v]), lr=lr, weight_decay=wd, step=5)
        out.append(host64(p))
    moved, rounded = (out[0] - out[1]).mean(), (want[0] - want[1]).mean()
    e = 12 * F32 * np.abs(exact - host64(start)).mean()
    assert rounded > 0.5 * lr * decay * 96                       # there is something to lose
    assert abs(moved - rounded) <= 2 * (2 * e / unit) * unit     # (both runs)


def test_a_gradient_of_zero_and_a_zero_state(d):
    """v = 0: the step is m / eps times lr, here 0; nothing is NaN."""
    p, g, m, v = (torch.zeros(100, device="cuda") for _ in range(4))
    p.fill_(2.0)
    d.adamw_step(d.adamw_list([p], [g], [m], [v]), **HYPER)
    assert torch.equal(p, torch.full_like(p, 2.0 * (1 - 1e-3))) and not m.any() and not v.any()


def test_offsets_past_32_bits(d):
    """A tensor of more than 2^32 bytes, and of more than 2^31 elements."""
    n = (1 << 31) + 12345
    g = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g[::65536] = 3.0
    g[-1] = 4.0
    gl = d.grad_list([g])
    norm, scale = outputs()
    d.grad_norm(gl, 1.0, norm, scale, ws=d.workspace(d.grad_norm_workspace_bytes(gl)))
    want = math.sqrt(9.0 * len(range(0, n, 65536)) + 16.0)
    assert abs(float(norm) - want) <= 1e-12 * want
    d.grad_clip(gl, scale)
    assert abs(float(g[-1]) - 4.0 / want) <= 2.0 ** -7 * 4 / want and float(g[-2]) == 0.0
    p, m, v = torch.ones(n, dtype=torch.bfloat16, device="cuda"), torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    d.adamw_step(d.adamw_list([p], [g], [m], [v]), lr=0.25, eps=0.0, weight_decay=0.0, step=1, scale=None)
    # eps 0: 0 / 0 where the gradient is zero
    assert float(p[-1]) == 0.75 and float(p[65536]) == 0.75 and math.isnan(float(p[-2])) and float(m[-1]) == float(g[-1]) * np.float32(1 - 0.9)


def test_the_same_bits_every_time_and_on_two_streams(d):
    grads = [torch.randn(n, device="cuda") for n in (100001, 77, 5_000_000)]
    gl = d.grad_list(grads)
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [outputs() for _ in range(8)]
    spaces = [d.workspace(d.grad_norm_workspace_bytes(gl)) for _ in streams]
    torch.cuda.synchronize()
    for i, (norm, scale) in enumerate(outs):
        with torch.cuda.stream(streams[i % 2]):
            d.grad_norm(gl, 1.0, norm, scale, ws=spaces[i % 2])
    torch.cuda.synchronize()
    assert len({float(n) for n, _ in outs}) == 1 and len({float(s) for _, s in outs}) == 1
