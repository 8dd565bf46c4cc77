"""Thin Python binding of libditstep.so (include/ditstep.h, include/ditpolicy.h).

Argument marshalling only: every function takes torch tensors that already
live on the GPU, passes their device pointers, sizes and the current HIP
stream through ctypes, and raises DitError on a non-OK status. All
computation happens in the library's HIP kernels; there is no fallback. The
import fails loudly if the library has not been built
(``python -m paper_2606_19004_amd.build``).
"""
from __future__ import annotations

import ctypes as C
import math
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
# DITSTEP_LIB selects another build of the library (the DITSTEP_DEBUG build, libditstep_debug.so)
LIB_PATH = os.environ.get("DITSTEP_LIB") or os.path.join(_HERE, "libditstep.so")

if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2606_19004_amd.build`")
_lib = C.CDLL(LIB_PATH)

DIT_F32, DIT_BF16 = 0, 1
STATUS = {0: "DIT_OK", 1: "DIT_ERR_INVALID_ARG", 2: "DIT_ERR_SHAPE", 3: "DIT_ERR_DOMAIN", 4: "DIT_ERR_NAN",
          5: "DIT_ERR_UNSUPPORTED", 6: "DIT_ERR_HIP", 7: "DIT_ERR_WORKSPACE"}
EXPORTS = ("dit_abi_version", "dit_status_string", "dit_last_error_message", "dit_block_workspace_bytes",
           "dit_block_forward", "dit_block_mlp", "joint_attention", "flow_step", "flow_logprob", "group_reward_stats",
           "group_reward_stats_async", "dit_timestep_embed", "dit_timestep_embed_noalloc", "dit_patch_embed", "dit_final_layer", "dit_denoise_workspace_bytes",
           "dit_denoise_step", "dit_profile_begin", "dit_profile_end", "dit_teacache_init", "dit_teacache_gate",
           "dit_teacache_cache_bytes", "dit_denoise_step_teacache",
           "packed_attention_workspace_bytes", "packed_attention", "packed_attention_backward_workspace_bytes",
           "packed_attention_backward", "gated_norm", "gated_norm_backward_workspace_bytes", "gated_norm_backward",
           "flow_policy_loss_workspace_bytes", "flow_policy_loss")


class DitError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{STATUS.get(status, status)}: {message}")
        self.status = status
        self.name = STATUS.get(status, str(status))


class BlockConfig(C.Structure):
    _fields_ = [("hidden", C.c_int32), ("heads", C.c_int32), ("head_dim", C.c_int32), ("mlp_hidden", C.c_int32),
                ("n_img", C.c_int32), ("n_txt", C.c_int32), ("grid_h", C.c_int32), ("grid_w", C.c_int32),
                ("rope", C.c_int32), ("ln_eps", C.c_float), ("rope_theta", C.c_float), ("dtype", C.c_int32)]


_P2 = C.c_void_p * 2
_BLOCK_TENSORS = ("mod_w", "mod_b", "qkv_w", "qkv_b", "out_w", "out_b", "mlp1_w", "mlp1_b", "mlp2_w", "mlp2_b")
_STEP_TENSORS = ("t1_w", "t1_b", "t2_w", "t2_b", "in_w", "in_b", "fmod_w", "fmod_b", "fout_w", "fout_b")


class BlockWeights(C.Structure):
    _fields_ = [(n, _P2) for n in _BLOCK_TENSORS]


class StepWeights(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in _STEP_TENSORS]


class TeaCacheState(C.Structure):
    _fields_ = [("threshold", C.c_double), ("n_coef", C.c_int32), ("coef", C.c_double * 8),
                ("accumulated", C.c_double), ("has_prev", C.c_int32), ("has_residual", C.c_int32)]


class PackedConfig(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("sequences", "heads", "kv_heads", "head_dim", "total_q", "total_k", "max_q",
                                         "causal", "dtype")] + [("scale", C.c_float)] + [
        (n, C.c_int64) for n in ("q_row", "q_head", "k_row", "k_head", "v_row", "v_head", "o_row", "o_head")]


class GatedNormConfig(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("sequences", "rows", "hidden", "dtype", "post_norm", "pre_norm")] + [
        ("eps", C.c_float), ("residual_scale", C.c_float)] + [
        (n, C.c_int64) for n in ("x_row", "y_row", "h_row", "mod_row")]


class KernelStat(C.Structure):
    _fields_ = [("name", C.c_char * 40), ("launches", C.c_int32), ("total_ms", C.c_double),
                ("flops", C.c_double), ("bytes", C.c_double)]


_stream = C.c_void_p
_i32, _i64, _f32, _sz = C.c_int32, C.c_int64, C.c_float, C.c_size_t
_vp = C.c_void_p
_sigs = {
    "dit_abi_version": ([], _i32),
    "dit_status_string": ([_i32], C.c_char_p),
    "dit_last_error_message": ([], C.c_char_p),
    "dit_block_workspace_bytes": ([C.POINTER(BlockConfig), _i32], _sz),
    "dit_block_forward": ([C.POINTER(BlockConfig), C.POINTER(BlockWeights), _i32, _vp, _vp, _vp, _vp, _sz, _stream], _i32),
    "dit_block_mlp": ([C.POINTER(BlockConfig), C.POINTER(BlockWeights), _i32, _vp, _vp, _vp, _vp, _sz, _stream], _i32),
    "joint_attention": ([_vp, _vp, _vp, _vp, _i32, _i32, _i32, _i32, _i64, _i64, _i64, _i64, _i64, _i64, _f32, _i32,
                         _stream], _i32),
    "flow_step": ([_vp, _vp, _vp, _i64, _f32, _f32, _f32, _stream], _i32),
    "flow_logprob": ([_vp, _vp, _vp, _i32, _i64, _f32, _f32, _f32, _vp, _stream], _i32),
    "group_reward_stats": ([_vp, _i32, _i32, _f32, _i32, _vp, _vp, _vp, _vp, _vp, _stream], _i32),
    "group_reward_stats_async": ([_vp, _i32, _i32, _f32, _i32, _vp, _vp, _vp, _vp, _vp, _vp, _stream], _i32),
    "dit_timestep_embed": ([C.POINTER(BlockConfig), C.POINTER(StepWeights), _i32, _vp, _vp, _vp, _sz, _stream], _i32),
    "dit_timestep_embed_noalloc": ([C.POINTER(BlockConfig), C.POINTER(StepWeights), _i32, _vp, _vp, _stream], _i32),
    "dit_patch_embed": ([C.POINTER(BlockConfig), C.POINTER(StepWeights), _i32, _i32, _vp, _vp, _vp, _sz, _stream], _i32),
    "dit_final_layer": ([C.POINTER(BlockConfig), C.POINTER(StepWeights), _i32, _i32, _vp, _vp, _vp, _vp, _sz,
                         _stream], _i32),
    "dit_denoise_workspace_bytes": ([C.POINTER(BlockConfig), _i32, _i32], _sz),
    "dit_denoise_step": ([C.POINTER(BlockConfig), C.POINTER(StepWeights), C.POINTER(BlockWeights), _i32, _i32, _i32,
                          _f32, _f32, _f32, _vp, _vp, _vp, _vp, _vp, _sz, _stream], _i32),
    "dit_profile_begin": ([], _i32),
    "dit_teacache_init": ([C.POINTER(TeaCacheState), C.c_double, C.POINTER(C.c_double), _i32], _i32),
    "dit_teacache_gate": ([C.POINTER(TeaCacheState), C.c_double, _i32, C.POINTER(_i32)], _i32),
    "dit_teacache_cache_bytes": ([C.POINTER(BlockConfig), _i32], _sz),
    "dit_denoise_step_teacache": ([C.POINTER(BlockConfig), C.POINTER(StepWeights), C.POINTER(BlockWeights), _i32,
                                   _i32, _i32, _f32, _f32, _f32, _vp, _vp, _vp, _vp, C.POINTER(TeaCacheState), _i32,
                                   _vp, _sz, C.POINTER(_i32), C.POINTER(C.c_double), _vp, _sz, _stream], _i32),
    "dit_profile_end": ([C.POINTER(KernelStat), _i32, C.POINTER(_i32)], _i32),
    "packed_attention_workspace_bytes": ([C.POINTER(PackedConfig)], _sz),
    "packed_attention": ([C.POINTER(PackedConfig)] + [_vp] * 9 + [_sz, _stream], _i32),
    "packed_attention_backward_workspace_bytes": ([C.POINTER(PackedConfig)], _sz),
    "packed_attention_backward": ([C.POINTER(PackedConfig)] + [_vp] * 13 + [_sz, _stream], _i32),
    "gated_norm": ([C.POINTER(GatedNormConfig)] + [_vp] * 10 + [_stream], _i32),
    "gated_norm_backward_workspace_bytes": ([C.POINTER(GatedNormConfig)], _sz),
    "gated_norm_backward": ([C.POINTER(GatedNormConfig)] + [_vp] * 17 + [_sz, _stream], _i32),
    "flow_policy_loss_workspace_bytes": ([_i32, _i64], _sz),
    "flow_policy_loss": ([_vp, _vp, _vp, _vp, _i32, _i64] + [C.c_double] * 3 + [_vp, _vp] + [C.c_double] * 4 + [ _vp, _vp, _vp, _vp, _vp, _sz, _stream], _i32),
}
for _name, (_args, _res) in _sigs.items():
    _fn = getattr(_lib, _name)
    _fn.argtypes = _args
    _fn.restype = _res


def lib() -> C.CDLL:
    return _lib


def _check(status: int) -> None:
    if status != 0:
        raise DitError(status, _lib.dit_last_error_message().decode())


def _ptr(t) -> int | None:
    return None if t is None else t.data_ptr()


# the current device, and its current stream's handle without a Stream object around it (2.5 us of a call's host time)
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _s(stream) -> int | None:
    if stream is None:
        if _raw_stream is not None:
            return _raw_stream(_current_device())
        stream = torch.cuda.current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else stream


def _dtype_code(dtype) -> int:
    if dtype in ("bf16", torch.bfloat16, DIT_BF16):
        return DIT_BF16
    if dtype in ("f32", torch.float32, DIT_F32):
        return DIT_F32
    raise ValueError(f"dtype {dtype!r}")


# ---------------------------------------------------------------------------
# structures
# ---------------------------------------------------------------------------
def block_config(hidden, heads, head_dim, mlp_hidden, n_img, n_txt, grid_h, grid_w, rope=True,
                 ln_eps=1e-6, rope_theta=1e4, dtype="bf16") -> BlockConfig:
    return BlockConfig(hidden, heads, head_dim, mlp_hidden, n_img, n_txt, grid_h, grid_w, int(bool(rope)),
                       ln_eps, rope_theta, _dtype_code(dtype))


def block_weights(img: dict, txt: dict) -> BlockWeights:
    """img/txt: {tensor name: device tensor} for the two streams (image = index 0)."""
    w = BlockWeights()
    for n in _BLOCK_TENSORS:
        setattr(w, n, _P2(_ptr(img.get(n)), _ptr(txt.get(n))))
    w._keep = (dict(img), dict(txt))   # the struct holds raw device pointers: keep the tensors alive with it
    return w


def step_weights(sw: dict) -> StepWeights:
    w = StepWeights()
    for n in _STEP_TENSORS:
        setattr(w, n, _ptr(sw.get(n)))
    w._keep = dict(sw)
    return w


def workspace(nbytes: int, device="cuda") -> torch.Tensor:
    """A device byte buffer (torch's allocator returns >= 256-byte aligned blocks)."""
    return torch.empty(max(int(nbytes), 1), dtype=torch.uint8, device=device)


# ---------------------------------------------------------------------------
# entry points (same names as the C ABI)
# ---------------------------------------------------------------------------
def dit_abi_version() -> int:
    return _lib.dit_abi_version()


def dit_block_workspace_bytes(cfg: BlockConfig, batch: int) -> int:
    return _lib.dit_block_workspace_bytes(C.byref(cfg), batch)


def dit_block_forward(cfg, w, temb, x_img, x_txt, ws, stream=None):
    _check(_lib.dit_block_forward(C.byref(cfg), C.byref(w), temb.shape[0], _ptr(temb), _ptr(x_img), _ptr(x_txt),
                                  _ptr(ws), ws.numel() if ws is not None else 0, _s(stream)))


def dit_block_mlp(cfg, w, temb, x_img, x_txt, ws, stream=None):
    _check(_lib.dit_block_mlp(C.byref(cfg), C.byref(w), temb.shape[0], _ptr(temb), _ptr(x_img), _ptr(x_txt),
                              _ptr(ws), ws.numel() if ws is not None else 0, _s(stream)))


def joint_attention(q, k, v, o, batch, heads, seq, head_dim, qkv_strides, o_strides, scale=None, dtype="bf16",
                    stream=None):
    """q/k/v/o: device tensors (or views) whose element (b, s, h, e) sits at the given element strides."""
    if scale is None:
        scale = 1.0 / math.sqrt(head_dim)
    _check(_lib.joint_attention(_ptr(q), _ptr(k), _ptr(v), _ptr(o), batch, heads, seq, head_dim, *qkv_strides,
                                *o_strides, scale, _dtype_code(dtype), _s(stream)))


def flow_step(x, v, noise, t, t_next, noise_level, stream=None):
    _check(_lib.flow_step(_ptr(x), _ptr(v), _ptr(noise), x.numel(), t, t_next, noise_level, _s(stream)))


def flow_logprob(x, v, x_next, t, t_next, noise_level, logp, stream=None):
    """x, v, x_next: [batch][n] fp32 device tensors (any trailing shape, flattened per sample);
    logp: [batch] fp64 device tensor."""
    b = x.shape[0] if x.dim() > 0 else 0
    n = x.numel() // b if b else 0
    _check(_lib.flow_logprob(_ptr(x), _ptr(v), _ptr(x_next), b, n, t, t_next, noise_level, _ptr(logp), _s(stream)))


def group_reward_stats(rewards, adv_eps=1e-4, k_select=0, mean=None, std=None, adv=None, order=None, selected=None,
                       stream=None):
    g, n = rewards.shape
    _check(_lib.group_reward_stats(_ptr(rewards), g, n, adv_eps, k_select, _ptr(mean), _ptr(std), _ptr(adv),
                                   _ptr(order), _ptr(selected), _s(stream)))


def group_reward_stats_async(rewards, status, adv_eps=1e-4, k_select=0, mean=None, std=None, adv=None, order=None,
                             selected=None, stream=None):
    """status: one-element int32 device tensor; holds DIT_OK or DIT_ERR_NAN once the stream has run."""
    g, n = rewards.shape
    _check(_lib.group_reward_stats_async(_ptr(rewards), g, n, adv_eps, k_select, _ptr(mean), _ptr(std), _ptr(adv),
                                         _ptr(order), _ptr(selected), _ptr(status), _s(stream)))


def dit_timestep_embed(cfg, sw, t, temb, ws, stream=None):
    _check(_lib.dit_timestep_embed(C.byref(cfg), C.byref(sw), t.shape[0], _ptr(t), _ptr(temb), _ptr(ws),
                                   ws.numel(), _s(stream)))


def dit_timestep_embed_noalloc(cfg, sw, t, temb, stream=None):
    _check(_lib.dit_timestep_embed_noalloc(C.byref(cfg), C.byref(sw), t.shape[0], _ptr(t), _ptr(temb), _s(stream)))


def dit_patch_embed(cfg, sw, latent, x_img, ws, stream=None):
    _check(_lib.dit_patch_embed(C.byref(cfg), C.byref(sw), latent.shape[0], latent.shape[-1], _ptr(latent),
                                _ptr(x_img), _ptr(ws), ws.numel() if ws is not None else 0, _s(stream)))


def dit_final_layer(cfg, sw, temb, x_img, v, ws, stream=None):
    _check(_lib.dit_final_layer(C.byref(cfg), C.byref(sw), temb.shape[0], v.shape[-1], _ptr(temb), _ptr(x_img),
                                _ptr(v), _ptr(ws), ws.numel(), _s(stream)))


def dit_denoise_workspace_bytes(cfg, batch, latent_dim) -> int:
    return _lib.dit_denoise_workspace_bytes(C.byref(cfg), batch, latent_dim)


def dit_denoise_step(cfg, sw, blocks, t, t_next, noise_level, latent, x_txt, noise, v_out, ws, stream=None):
    arr = (BlockWeights * max(len(blocks), 1))(*blocks)
    _check(_lib.dit_denoise_step(C.byref(cfg), C.byref(sw), arr, len(blocks), latent.shape[0], latent.shape[-1],
                                 t, t_next, noise_level, _ptr(latent), _ptr(x_txt), _ptr(noise), _ptr(v_out),
                                 _ptr(ws), ws.numel(), _s(stream)))


def teacache_state(threshold, coef=()):
    st = TeaCacheState()
    c = (C.c_double * max(len(coef), 1))(*[float(x) for x in coef])
    _check(_lib.dit_teacache_init(C.byref(st), float(threshold), c, len(coef)))
    return st


def dit_teacache_gate(state, rel, force=False):
    run = _i32()
    _check(_lib.dit_teacache_gate(C.byref(state), float(rel), int(bool(force)), C.byref(run)))
    return bool(run.value)


def dit_teacache_cache_bytes(cfg, batch):
    return _lib.dit_teacache_cache_bytes(C.byref(cfg), batch)


def dit_denoise_step_teacache(cfg, sw, blocks, t, t_next, noise_level, latent, x_txt, noise, v_out, state, cache, ws,
                              force=False, stream=None):
    """Returns (ran_blocks, rel)."""
    arr = (BlockWeights * max(len(blocks), 1))(*blocks)
    ran, rel = _i32(), C.c_double()
    _check(_lib.dit_denoise_step_teacache(C.byref(cfg), C.byref(sw), arr, len(blocks), latent.shape[0],
                                          latent.shape[-1], t, t_next, noise_level, _ptr(latent), _ptr(x_txt),
                                          _ptr(noise), _ptr(v_out), C.byref(state), int(bool(force)), _ptr(cache),
                                          cache.numel(), C.byref(ran), C.byref(rel), _ptr(ws), ws.numel(),
                                          _s(stream)))
    return bool(ran.value), rel.value


# ---------------------------------------------------------------------------
# policy update (include/ditpolicy.h)
# ---------------------------------------------------------------------------
NORM_KINDS = {"none": 0, "layer": 1, "rms": 2}
_ROW_TYPES = {DIT_BF16: torch.bfloat16, DIT_F32: torch.float32}


def _at(t, layout):
    """The device pointer of a tensor (or None) whose (type, shape, strides, device) has to be `layout`: the device is the current one, whose
    stream runs the call."""
    if t is None:
        return None
    if (t.dtype, t.shape, t.stride(), t.get_device()) != layout:
        _check_layout(t, *layout)
    return t.data_ptr()


def _dense(t, dev, dtype, n):
    """The same of n elements without gaps (or more)."""
    if t is None:
        return None
    if t.dtype is not dtype or t.numel() < n or not t.is_contiguous() or t.get_device() != dev:
        _check_layout(t, dtype, (n,), (1,), dev)
    return t.data_ptr()


def _check_layout(t, dtype, shape, strides, dev):
    """What else may be read and written as `shape` at `strides`: more rows, any stride of an index that has one value, and, where the
    elements lie without gaps, as many of them in any contiguous shape."""
    if dtype is not None and t.dtype is not dtype:   # (None: a config of an unknown type, which the library refuses)
        raise ValueError(f"a tensor of {t.dtype} where {dtype} is wanted")
    if t.get_device() != dev:
        raise ValueError(f"a tensor on {t.device} in a call on cuda:{dev}")
    if 0 in shape:
        return
    dense = [math.prod(shape[i + 1:]) for i in range(len(shape))]
    if t.is_contiguous() and t.numel() >= math.prod(shape) and all(n == 1 or a == b for n, a, b in zip(shape, strides, dense)):
        return
    if t.dim() != len(shape) or t.shape[0] < shape[0] or t.shape[1:] != shape[1:]:
        raise ValueError(f"a tensor of shape {tuple(t.shape)} where the call has {shape}")
    if any(n > 1 and a != b for n, a, b in zip(shape, t.stride(), strides)):
        raise ValueError(f"a tensor of strides {t.stride()} where the call has {strides}")


def _ws_args(ws, dev):
    if ws is None:
        return None, 0
    if ws.get_device() != dev:
        _check_layout(ws, ws.dtype, (), (), dev)
    return ws.data_ptr(), ws.numel()


def packed_config(q, k, v, o, sequences, causal=False, scale=None, max_q=0) -> PackedConfig:
    """Shapes and strides of q, o [rows][heads][d] and k, v [rows][kv_heads][d] (views are fine, e contiguous).
    max_q: no sequence has more queries (0: not known)."""
    for t in (q, k, v, o):
        if t.dim() != 3 or (t.numel() and t.stride(2) != 1):
            raise ValueError("q, k, v and o are [rows][heads][head_dim] with the last index contiguous")
        if t.dtype != q.dtype or t.shape[2] != q.shape[2]:
            raise ValueError("q, k, v and o have one type and one head_dim")
    if k.shape != v.shape or o.shape != q.shape:
        raise ValueError("k and v, and q and o, have one shape")
    d = q.shape[2]
    if scale is None:
        scale = 1.0 / math.sqrt(d)
    strides = [s for t in (q, k, v, o) for s in (t.stride(0), t.stride(1))]
    return PackedConfig(sequences, q.shape[1], k.shape[1], d, q.shape[0], k.shape[0], max_q, int(bool(causal)),
                        _dtype_code(q.dtype), scale, *strides)


def _attention_layouts(cfg, dev):
    """Of q, k, v, o and their gradients."""
    dt, d = _ROW_TYPES.get(cfg.dtype), cfg.head_dim
    q, k = (cfg.total_q, cfg.heads, d), (cfg.total_k, cfg.kv_heads, d)
    return (dt, q, (cfg.q_row, cfg.q_head, 1), dev), (dt, k, (cfg.k_row, cfg.k_head, 1), dev), (dt, k, (cfg.v_row, cfg.v_head, 1), dev), (
        dt, q, (cfg.o_row, cfg.o_head, 1), dev)


def packed_attention_workspace_bytes(cfg) -> int:
    return _lib.packed_attention_workspace_bytes(C.byref(cfg))


def packed_attention(cfg, q, k, v, o, lse=None, q_offsets=None, k_offsets=None, k_lengths=None, ws=None, stream=None):
    """Tensors laid out as those cfg was made from; lse: fp32 [rows][heads]; offsets (one more than sequences) and lengths: device
    int32, or None (equal lengths)."""
    dev, s, i32 = _current_device(), cfg.sequences, torch.int32
    lq, lk, lv, lo = _attention_layouts(cfg, dev)
    qo, ko, kl = _dense(q_offsets, dev, i32, s + 1), _dense(k_offsets, dev, i32, s + 1), _dense(k_lengths, dev, i32, s)
    _check(_lib.packed_attention(C.byref(cfg), _at(q, lq), _at(k, lk), _at(v, lv), qo, ko, kl, _at(o, lo),
                                 _dense(lse, dev, torch.float32, cfg.total_q * cfg.heads), *_ws_args(ws, dev), _s(stream)))


def packed_attention_backward_workspace_bytes(cfg) -> int:
    return _lib.packed_attention_backward_workspace_bytes(C.byref(cfg))


def packed_attention_backward(cfg, q, k, v, o, lse, d_o, dq, dk, dv, q_offsets=None, k_offsets=None, k_lengths=None,
                              ws=None, stream=None):
    """d_o laid out like o, dq, dk, dv like q, k, v."""
    dev, s, i32 = _current_device(), cfg.sequences, torch.int32
    lq, lk, lv, lo = _attention_layouts(cfg, dev)
    qo, ko, kl = _dense(q_offsets, dev, i32, s + 1), _dense(k_offsets, dev, i32, s + 1), _dense(k_lengths, dev, i32, s)
    _check(_lib.packed_attention_backward(
        C.byref(cfg), _at(q, lq), _at(k, lk), _at(v, lv), _at(o, lo),
        _dense(lse, dev, torch.float32, cfg.total_q * cfg.heads), _at(d_o, lo), qo, ko, kl, _at(dq, lq), _at(dk, lk),
        _at(dv, lv), *_ws_args(ws, dev), _s(stream)))


def gated_norm_config(x, sequences, post="none", pre="layer", eps=1e-6, residual_scale=1.0, y_row=None, h_row=None,
                      mod_row=None) -> GatedNormConfig:
    """x [rows][hidden] (a row stride is fine); row strides of y and h are x's, that of gate, scale and shift is hidden, unless given."""
    if x.dim() != 2 or (x.numel() and x.stride(1) != 1):
        raise ValueError("x is [rows][hidden] with the last index contiguous")
    rows, hidden = x.shape
    row = x.stride(0) if rows > 1 else max(x.stride(0), hidden)
    return GatedNormConfig(sequences, rows, hidden, _dtype_code(x.dtype), NORM_KINDS[post], NORM_KINDS[pre], eps,
                           residual_scale, row, row if y_row is None else y_row, row if h_row is None else h_row,
                           hidden if mod_row is None else mod_row)


def gated_norm(cfg, x, y, x_out, h, gate=None, scale=None, shift=None, post_w=None, pre_w=None, offsets=None,
               stream=None):
    """x, x_out, y, h: cfg's type, at its x_row, y_row, h_row; post_w, pre_w: [hidden], cfg's type; gate, scale, shift: fp32
    [sequences][hidden] at its mod_row; offsets: device int32 (one more than sequences), or None (equal lengths)."""
    dev, dt, f32, hidden, s = _current_device(), _ROW_TYPES.get(cfg.dtype), torch.float32, cfg.hidden, cfg.sequences
    rows = (cfg.rows, hidden)
    lx, lm = (dt, rows, (cfg.x_row, 1), dev), (f32, (s, hidden), (cfg.mod_row, 1), dev)
    off, g, sc, sh = _dense(offsets, dev, torch.int32, s + 1), _at(gate, lm), _at(scale, lm), _at(shift, lm)
    _check(_lib.gated_norm(C.byref(cfg), _at(x, lx), _at(y, (dt, rows, (cfg.y_row, 1), dev)), _dense(post_w, dev, dt, hidden),
                           _dense(pre_w, dev, dt, hidden), g, sc, sh, off, _at(x_out, lx), _at(h, (dt, rows, (cfg.h_row, 1), dev)), _s(stream)))


def gated_norm_backward_workspace_bytes(cfg) -> int:
    return _lib.gated_norm_backward_workspace_bytes(C.byref(cfg))


def gated_norm_backward(cfg, x_out, y, dx_out, dh, dx, dy, gate=None, scale=None, post_w=None, pre_w=None, offsets=None,
                        dgate=None, dscale=None, dshift=None, dpost_w=None, dpre_w=None, ws=None, stream=None):
    """x_out: the forward call's output. Any gradient may be None; those of vectors and weights are fp32."""
    dev, dt, f32, hidden, s = _current_device(), _ROW_TYPES.get(cfg.dtype), torch.float32, cfg.hidden, cfg.sequences
    rows = (cfg.rows, hidden)
    lx, ly, lh = (dt, rows, (cfg.x_row, 1), dev), (dt, rows, (cfg.y_row, 1), dev), (dt, rows, (cfg.h_row, 1), dev)
    lm = (f32, (s, hidden), (cfg.mod_row, 1), dev)
    off, g, sc = _dense(offsets, dev, torch.int32, s + 1), _at(gate, lm), _at(scale, lm)
    _check(_lib.gated_norm_backward(
        C.byref(cfg), _at(x_out, lx), _at(y, ly), _dense(post_w, dev, dt, hidden), _dense(pre_w, dev, dt, hidden), g, sc, off,
        _at(dx_out, lx), _at(dh, lh), _at(dx, lx), _at(dy, ly), _at(dgate, lm), _at(dscale, lm),
        _at(dshift, lm), _dense(dpost_w, dev, f32, hidden), _dense(dpre_w, dev, f32, hidden), *_ws_args(ws, dev), _s(stream)))


def flow_policy_loss_workspace_bytes(batch, n_per_sample) -> int:
    return _lib.flow_policy_loss_workspace_bytes(batch, n_per_sample)


def flow_policy_loss(x, v, x_next, logp_old, adv, t, t_next, noise_level, loss, dv=None, logp=None, ratio=None,
                     v_ref=None, logp_scale=None, clip_low=0.2, clip_high=0.2, kl_weight=0.0, ws=None, stream=None):
    """x, v, x_next, v_ref, dv: [batch][n] fp32 (any trailing shape, contiguous); logp_old, logp, ratio: [batch] fp64; adv: [batch]
    fp32; loss: one fp64. logp_scale None: 1 / n."""
    b = x.shape[0] if x.dim() > 0 else 0
    n = x.numel() // b if b else 0
    if logp_scale is None:
        logp_scale = 1.0 / max(n, 1)
    dev, f32, f64, bn = _current_device(), torch.float32, torch.float64, b * n
    old, pa = _dense(logp_old, dev, f64, b), _dense(adv, dev, f32, b)
    px, pv, pn, pr, dvp = (_dense(u, dev, f32, bn) for u in (x, v, x_next, v_ref, dv))
    _check(_lib.flow_policy_loss(px, pv, pn, pr, b, n, t, t_next, noise_level, old, pa, logp_scale, clip_low, clip_high, kl_weight,
                                 _dense(loss, dev, f64, 1), _dense(logp, dev, f64, b), _dense(ratio, dev, f64, b), dvp,
                                 *_ws_args(ws, dev), _s(stream)))


def dit_profile_begin():
    _check(_lib.dit_profile_begin())


def dit_profile_end() -> list:
    """Per-kernel-class totals since dit_profile_begin: list of dicts (name, launches, total_ms, flops, bytes)."""
    cap = 64
    arr = (KernelStat * cap)()
    n = _i32(0)
    _check(_lib.dit_profile_end(arr, cap, C.byref(n)))
    return [{"name": arr[i].name.decode(), "launches": arr[i].launches, "total_ms": arr[i].total_ms,
             "flops": arr[i].flops, "bytes": arr[i].bytes} for i in range(min(n.value, cap))]
