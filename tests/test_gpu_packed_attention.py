"""packed_attention and packed_attention_backward against the float64 oracle, within element-wise bounds
(tests/policy_util.py)."""
import numpy as np
import pytest
import torch

from tests.gpu_util import host64
from tests.policy_util import attention_reference, check, i32, offsets, stored, to_dev

pytestmark = pytest.mark.gpu

SENTINEL = 7.0


@pytest.fixture(scope="module")
def d():
    from paper_2606_19004_amd import ditstep
    return ditstep


class Problem:
    """A packed batch on the device. Rows before the first sequence and after the last, and cache rows past a
    sequence's keys, hold NaN; outputs start at SENTINEL."""

    def __init__(self, d, dtype, hd, H, G, q_len, k_len=None, causal=False, slack=0, lead=0, tail=0, seed=0, scale=None,
                 layout="packed", q_gain=1.0):
        rng = np.random.default_rng(seed)
        self.d, self.dtype, self.causal, self.scale = d, dtype, causal, scale or hd ** -0.5
        self.q_len, self.k_len = np.asarray(q_len), np.asarray(q_len if k_len is None else k_len)
        self.q_off, self.k_off = offsets(self.q_len, lead), offsets(self.k_len + slack, lead)
        self.slack = slack
        tq, tk = int(self.q_off[-1]) + tail, int(self.k_off[-1]) + tail

        def draw(rows, heads, off, lens, gain=1.0):
            x = np.full((rows, heads, hd), np.nan)
            for o, n in zip(off, lens):
                x[o:o + n] = gain * rng.standard_normal((n, heads, hd))
            return stored(x, dtype)

        self.q = draw(tq, H, self.q_off, self.q_len, q_gain)
        self.k, self.v = draw(tk, G, self.k_off, self.k_len), draw(tk, G, self.k_off, self.k_len)
        self.do = draw(tq, H, self.q_off, self.q_len)
        if layout == "packed" and k_len is None and not slack:      # slices of one projection
            buf = to_dev(np.concatenate([self.q, self.k, self.v], 1), dtype)
            self.tq, self.tk, self.tv = buf[:, :H], buf[:, H:H + G], buf[:, H + G:]
        elif layout == "head_major":                                # [heads][rows][d], as a cache may lie
            self.tq, self.tk, self.tv = (to_dev(x.transpose(1, 0, 2), dtype).transpose(0, 1) for x in (self.q, self.k, self.v))
        else:
            self.tq, self.tk, self.tv = (to_dev(x, dtype) for x in (self.q, self.k, self.v))
        self.to = torch.full_like(to_dev(self.q, dtype), SENTINEL)
        self.lse = torch.full((tq, H), SENTINEL, device="cuda")
        self.dq_off, self.dk_off = i32(self.q_off), i32(self.k_off)
        self.lengths = i32(self.k_len) if slack else None
        self.cfg = d.packed_config(self.tq, self.tk, self.tv, self.to, len(self.q_len), causal, self.scale,
                                   max_q=int(self.q_len.max(initial=0)))

    def forward(self, **kw):
        ws = self.d.workspace(self.d.packed_attention_workspace_bytes(self.cfg)).fill_(255)
        self.d.packed_attention(self.cfg, self.tq, self.tk, self.tv, self.to, lse=self.lse, q_offsets=self.dq_off,
                                k_offsets=self.dk_off, k_lengths=self.lengths, ws=ws, **kw)
        torch.cuda.synchronize()
        return host64(self.to), self.lse.double().cpu().numpy()

    def reference(self):
        return attention_reference(self.q, self.k, self.v, self.q_off, self.k_off, self.k_len, self.scale, self.causal, self.dtype)

    def check_forward(self):
        o, lse = self.forward()
        ref = self.reference()
        check(o, ref["o"], ref["o_tol"], "o")
        check(lse, ref["lse"], ref["lse_tol"], "lse")
        assert np.all(o[np.isnan(ref["o"])] == SENTINEL) and np.all(lse[np.isnan(ref["lse"])] == SENTINEL)

    def backward(self):
        ref = self.reference()
        self.o64 = stored(np.where(np.isnan(ref["o"]), 0.0, ref["o"]), self.dtype)
        self.lse64 = np.where(np.isnan(ref["lse"]), 0.0, ref["lse"]).astype(np.float32).astype(np.float64)
        o, do = to_dev(self.o64, self.dtype), to_dev(self.do, self.dtype)
        grads = [torch.empty_strided(t.shape, t.stride(), dtype=t.dtype, device="cuda").fill_(SENTINEL) if t.is_contiguous()
                 else torch.full(t.shape[1::-1] + t.shape[2:], SENTINEL, dtype=t.dtype, device="cuda").transpose(0, 1)
                 if t.stride(1) > t.stride(0) else None for t in (self.tq, self.tk, self.tv)]
        if grads[0] is None or grads[1] is None:                     # slices of one gradient
            H, G = self.tq.shape[1], self.tk.shape[1]
            buf = torch.full((self.tq.shape[0], H + 2 * G, self.tq.shape[2]), SENTINEL, dtype=self.tq.dtype, device="cuda")
            grads = [buf[:, :H], buf[:, H:H + G], buf[:, H + G:]]
        ws = self.d.workspace(self.d.packed_attention_backward_workspace_bytes(self.cfg)).fill_(255)
        self.d.packed_attention_backward(self.cfg, self.tq, self.tk, self.tv, o, torch.from_numpy(self.lse64).float().cuda(),
                                         do, *grads, q_offsets=self.dq_off, k_offsets=self.dk_off, k_lengths=self.lengths, ws=ws)
        torch.cuda.synchronize()
        return grads

    def check_backward(self):
        grads = self.backward()
        ref = attention_reference(self.q, self.k, self.v, self.q_off, self.k_off, self.k_len, self.scale, self.causal,
                                  self.dtype, self.do, self.o64, self.lse64)
        for n, g in zip(("dq", "dk", "dv"), grads):
            got = host64(g.contiguous())
            check(got, ref[n], ref[n + "_tol"], n)
            assert np.all(got[np.isnan(ref[n])] == SENTINEL), n


# lengths of one and of none, whole and ragged tiles, more queries than keys (rows that see nothing)
SHAPES = [
    # H, G, q lengths, k lengths (None: the same), causal
    (2, 2, [1], None, True),
    (4, 2, [64, 128], None, False),
    (6, 2, [5, 0, 77, 1, 130], None, True),
    (3, 1, [129, 31, 65], None, True),
    (4, 4, [200, 63], None, False),
    (7, 1, [40, 3], [333, 70], True),
    (4, 2, [70, 9, 4], [33, 0, 1], True),
    (2, 1, [5, 0, 3], [0, 40, 100], False),
    (1, 1, [300], [257], True),
    (4, 1, [700], None, True),
    (8, 1, [300, 90], None, False),
]


@pytest.mark.parametrize("dtype,hd", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("H,G,ql,kl,causal", SHAPES)
def test_forward(d, dtype, hd, H, G, ql, kl, causal):
    Problem(d, dtype, hd, H, G, ql, kl, causal, lead=3, tail=2, seed=hd + len(ql)).check_forward()


@pytest.mark.parametrize("dtype,hd", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("H,G,ql,kl,causal", SHAPES)
def test_backward(d, dtype, hd, H, G, ql, kl, causal):
    Problem(d, dtype, hd, H, G, ql, kl, causal, lead=3, tail=2, seed=hd + 7 * len(ql)).check_backward()


@pytest.mark.parametrize("dtype,hd", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("H,G,new,keys", [
    (8, 2, 1, [1, 7, 700, 64, 1500]), (32, 8, 1, [2100]), (4, 4, 1, [513, 40]), (10, 2, 3, [900, 3, 65]),
    (40, 5, 1, [333]), (8, 1, 5, [2000, 5]), (2, 2, 33, [1030, 40])])
def test_few_queries_against_a_cache(d, dtype, hd, H, G, new, keys):
    """One or a few new tokens per sequence: keys are shared out between workgroups and joined."""
    Problem(d, dtype, hd, H, G, [new] * len(keys), keys, True, slack=11, seed=hd + new).check_forward()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_cache_gradients_leave_the_room_alone(d, dtype):
    Problem(d, dtype, 64, 4, 2, [5, 30], [20, 90], True, slack=9, lead=1, tail=4, seed=3).check_backward()


@pytest.mark.parametrize("dtype,hd", [("bf16", 128), ("bf16", 64), ("f32", 64)])
def test_head_major_layout(d, dtype, hd):
    p = Problem(d, dtype, hd, 6, 3, [50, 90], None, True, layout="head_major", seed=hd)
    p.check_forward()
    p.check_backward()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_scores_stay_finite(d, dtype):
    Problem(d, dtype, 64, 2, 1, [100, 70], None, True, seed=5, q_gain=40.0).check_forward()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_equal_lengths_need_no_offsets(d, dtype):
    p = Problem(d, dtype, 64, 4, 2, [37, 37, 37], None, False, seed=6)
    want, lse = (t.clone() for t in (p.forward() and (p.to, p.lse)))
    p.dq_off = p.dk_off = None
    p.to.fill_(SENTINEL)
    p.lse.fill_(SENTINEL)
    p.forward()
    assert torch.equal(p.to, want) and torch.equal(p.lse, lse)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_runs_give_the_same_bits(d, dtype):
    for kw in ({"q_len": [300, 41, 90]}, {"q_len": [1, 1], "k_len": [3000, 200], "slack": 1}):
        p = Problem(d, dtype, 64, 8, 2, causal=True, seed=9, **kw)
        p.forward()
        o, lse = p.to.clone(), p.lse.clone()
        p.forward()
        assert torch.equal(o, p.to) and torch.equal(lse, p.lse)
        a, b = p.backward(), p.backward()
        assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_many_sequences(d):
    """More sequences than a wave looks through at once."""
    rng = np.random.default_rng(1)
    ql = rng.integers(0, 9, 150)
    p = Problem(d, "bf16", 64, 4, 2, ql, None, True, seed=11)
    p.check_forward()
    p.check_backward()
    kl = ql * 0 + rng.integers(1, 200, 150)
    Problem(d, "bf16", 64, 4, 2, np.ones(150, int), kl, True, slack=2, seed=12).check_forward()


def test_bad_offsets_stay_inside_the_tensors(d):
    """Offsets that run backwards or past the end are clamped: the call returns, and rows past them are untouched."""
    p = Problem(d, "bf16", 64, 4, 2, [100, 60], None, True, seed=13)
    p.dq_off, p.dk_off = i32([-5, 400, 20]), i32([90, 10, 1000])
    o, _ = p.forward()
    p.backward()
    assert o.shape[0] == 160


def test_on_a_stream_and_in_a_graph(d):
    """The call runs on the stream it is given, and a captured one replays to the same bits between eager calls."""
    for kw in ({"q_len": [70, 130]}, {"q_len": [1, 1, 1], "k_len": [900, 1, 300], "slack": 1}):
        p = Problem(d, "bf16", 64, 4, 2, causal=True, seed=15, **kw)
        p.forward()
        want, lse = p.to.clone(), p.lse.clone()
        ws = d.workspace(d.packed_attention_workspace_bytes(p.cfg))
        args = dict(lse=p.lse, q_offsets=p.dq_off, k_offsets=p.dk_off, k_lengths=p.lengths, ws=ws)
        s = torch.cuda.Stream()
        p.to.zero_()
        s.wait_stream(torch.cuda.current_stream())
        d.packed_attention(p.cfg, p.tq, p.tk, p.tv, p.to, stream=s, **args)
        s.synchronize()
        assert torch.equal(p.to, want)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            d.packed_attention(p.cfg, p.tq, p.tk, p.tv, p.to, **args)
        for _ in range(3):
            p.to.zero_()
            p.lse.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(p.to, want) and torch.equal(p.lse, lse)
            p.forward()


def test_a_cache_past_32_bit_offsets(d):
    """Keys whose elements lie further than 2^32 bytes from the tensor's start."""
    rows, G, hd = 300, 2, 64
    row = 1 << 23                                                 # 300 rows of 16 MiB: 4.7 GiB
    store = torch.empty(rows * row + 4096, dtype=torch.bfloat16, device="cuda")
    rng = np.random.default_rng(2)
    k, v, q = (stored(rng.standard_normal((n, h, hd)), "bf16") for n, h in ((rows, G), (rows, G), (3, 4)))
    tk = store.as_strided((rows, G, hd), (row, hd, 1), 0)
    tv = store.as_strided((rows, G, hd), (row, hd, 1), 2048)
    tk.copy_(to_dev(k, "bf16"))
    tv.copy_(to_dev(v, "bf16"))
    tq, o, lse = to_dev(q, "bf16"), to_dev(q * 0, "bf16"), torch.zeros((3, 4), device="cuda")
    cfg = d.packed_config(tq, tk, tv, o, 1, True, 0.125, max_q=3)
    ws = d.workspace(d.packed_attention_workspace_bytes(cfg))
    d.packed_attention(cfg, tq, tk, tv, o, lse=lse, ws=ws)
    ref = attention_reference(q, k, v, [0, 3], [0, rows], [rows], 0.125, True, "bf16")
    check(host64(o), ref["o"], ref["o_tol"], "o")
    check(lse.double().cpu().numpy(), ref["lse"], ref["lse_tol"], "lse")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_cache_of_equal_regions(d, dtype):
    """[sequences][room] caches: k_lengths without offsets."""
    S, room, H, G, hd = 3, 50, 4, 2, 64
    rng = np.random.default_rng(4)
    lens = np.array([50, 1, 33])
    q, k, v = (stored(rng.standard_normal(s), dtype) for s in ((S, H, hd), (S * room, G, hd), (S * room, G, hd)))
    for i, n in enumerate(lens):
        k[i * room + n:(i + 1) * room] = v[i * room + n:(i + 1) * room] = np.nan
    tq, tk, tv = (to_dev(x, dtype) for x in (q, k, v))
    o, lse = torch.zeros_like(tq), torch.zeros((S, H), device="cuda")
    cfg = d.packed_config(tq, tk, tv, o, S, True)
    ws = d.workspace(d.packed_attention_workspace_bytes(cfg))
    d.packed_attention(cfg, tq, tk, tv, o, lse=lse, k_lengths=i32(lens), ws=ws)
    ref = attention_reference(q, k, v, list(range(S + 1)), [i * room for i in range(S)], lens, hd ** -0.5, True, dtype)
    check(host64(o), ref["o"], ref["o_tol"], "o")
    check(lse.double().cpu().numpy(), ref["lse"], ref["lse_tol"], "lse")


def test_two_streams_at_once(d):
    """Calls on two streams with buffers and workspaces of their own."""
    ps = [Problem(d, "bf16", 64, 8, 2, [200, 300], None, True, seed=s) for s in (1, 2)]
    want = []
    for p in ps:
        p.forward()
        want.append((p.to.clone(), p.lse.clone(), [g.clone() for g in p.backward()]))
    streams = [torch.cuda.Stream() for _ in ps]
    torch.cuda.synchronize()
    keep = []
    for _ in range(3):
        for p, s in zip(ps, streams):
            ws = d.workspace(d.packed_attention_workspace_bytes(p.cfg))
            keep.append(ws)
            d.packed_attention(p.cfg, p.tq, p.tk, p.tv, p.to, lse=p.lse, q_offsets=p.dq_off, k_offsets=p.dk_off, ws=ws, stream=s)
    torch.cuda.synchronize()
    for p, w in zip(ps, want):
        assert torch.equal(p.to, w[0]) and torch.equal(p.lse, w[1])


def test_backward_in_a_graph(d):
    p = Problem(d, "bf16", 128, 8, 2, [300, 41], None, True, seed=21)
    want = [g.clone() for g in p.backward()]
    o, do, lse = to_dev(p.o64, "bf16"), to_dev(p.do, "bf16"), torch.from_numpy(p.lse64).float().cuda()
    buf = torch.zeros((p.tq.shape[0], 12, 128), dtype=torch.bfloat16, device="cuda")
    grads = [buf[:, :8], buf[:, 8:10], buf[:, 10:]]
    ws = d.workspace(d.packed_attention_backward_workspace_bytes(p.cfg))

    def call():
        d.packed_attention_backward(p.cfg, p.tq, p.tk, p.tv, o, lse, do, *grads, q_offsets=p.dq_off, k_offsets=p.dk_off, ws=ws)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(3):
        buf.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(grads, want))
        call()


# enough workgroups for the widest tiles of each type: many heads, or so many queries that a key tile's rows are shared out
WIDE = [
    # H, G, q lengths, k lengths (None: the same), causal
    (16, 16, [40, 0, 150, 1, 64, 17] * 7, None, True),
    (32, 16, [33, 9, 65] * 10, [70, 1, 0] * 10, False),
    (16, 2, [4100, 5000], [20, 33], False),
]


@pytest.mark.parametrize("dtype,hd", [("f32", 128), ("f32", 64), ("bf16", 128), ("bf16", 64)])
@pytest.mark.parametrize("H,G,ql,kl,causal", WIDE)
def test_problems_that_fill_the_chip(d, dtype, hd, H, G, ql, kl, causal):
    p = Problem(d, dtype, hd, H, G, ql, kl, causal, lead=2, tail=3, seed=hd + len(ql))
    p.check_forward()
    p.check_backward()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kw", [dict(q_len=[5, 90], k_len=[40, 130]), dict(q_len=[1, 1], k_len=[1500, 3], slack=2)])
def test_lse_may_be_left_out(d, dtype, kw):
    p = Problem(d, dtype, 64, 4, 2, causal=True, seed=31, **kw)
    p.forward()
    want, lse = p.to.clone(), p.lse.clone()
    p.to.fill_(SENTINEL)
    p.lse.fill_(SENTINEL)
    ws = d.workspace(d.packed_attention_workspace_bytes(p.cfg))
    d.packed_attention(p.cfg, p.tq, p.tk, p.tv, p.to, q_offsets=p.dq_off, k_offsets=p.dk_off, k_lengths=p.lengths, ws=ws)
    torch.cuda.synchronize()
    assert torch.equal(p.to, want) and bool((p.lse == SENTINEL).all())
    assert lse.isfinite().all()


def test_two_captured_calls_share_a_workspace(d):
    """Graphs of two problems over one workspace, replayed in turn on one stream."""
    ps = [Problem(d, "bf16", 64, 4, 2, [1, 1], [1500, 900], True, slack=1, seed=s) for s in (41, 42)]
    ws = d.workspace(max(d.packed_attention_workspace_bytes(p.cfg) for p in ps))
    assert ws.numel() > 0
    want, graphs = [], []
    for p in ps:
        p.forward()
        want.append((p.to.clone(), p.lse.clone()))
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            d.packed_attention(p.cfg, p.tq, p.tk, p.tv, p.to, lse=p.lse, q_offsets=p.dq_off, k_offsets=p.dk_off,
                               k_lengths=p.lengths, ws=ws)
    for _ in range(3):
        for p in ps:
            p.to.zero_()
            p.lse.zero_()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p.to, w[0]) and torch.equal(p.lse, w[1]) for p, w in zip(ps, want))


@pytest.mark.parametrize("dtype,hd", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("H,G,ql,kl,causal", [
    (2, 1, [40], [3000], True), (2, 2, [33, 130, 0], [3100, 2700, 900], True), (4, 1, [90, 1], [4100, 5], False),
    (1, 1, [2500], [2500], True)])
def test_many_queries_against_long_keys(d, dtype, hd, H, G, ql, kl, causal):
    """So few tiles of rows that their keys are shared out and joined, a part without visible keys among them."""
    p = Problem(d, dtype, hd, H, G, ql, kl, causal, lead=1, tail=2, seed=hd + len(ql))
    assert d.packed_attention_workspace_bytes(p.cfg) > 0
    p.check_forward()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("count", [64, 65, 256, 257, 700])
def test_hundreds_of_sequences(d, dtype, count):
    """As many as a wave looks at in one go, and past it, empty ones at both ends among them."""
    rng = np.random.default_rng(count)
    ql = rng.integers(0, 7, count)
    ql[0] = 0
    ql[-2:] = (3, 0)
    p = Problem(d, dtype, 64, 4, 2, ql, None, True, lead=2, tail=1, seed=count)
    p.check_forward()
    p.check_backward()
    Problem(d, dtype, 64, 4, 2, np.ones(count, int), rng.integers(0, 50, count), True, slack=1, seed=count + 1).check_forward()
