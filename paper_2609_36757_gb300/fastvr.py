"""Python binding of libfastvr_attn.so (the C ABI in include/fastvr_attn.h and
include/fastvr_block.h).

The functions below carry the C names and only marshal arguments: pointers are
passed as integers (device addresses), streams as cudaStream_t handles.  Every
step of the computation runs in the library's CUDA kernels; there is no
fallback of any kind, and importing this module raises when the library has
not been built.

`StreamingAttention` is a convenience wrapper for torch tensors: it allocates
the KV cache with torch (device memory is the caller's in the C ABI) and
passes data pointers and the current CUDA stream through;
`StreamingAttention4` is the same over a cache held in 4 bits.  `rotary`,
`gated_norm` and their gradients cover what runs before and after the
attention in a block, `cross_attention` (queries over an encoder's states) and
`gated_ffn` (the feed-forward's projections and activation) with their
gradients the block's other operators.
"""
from __future__ import annotations

import ctypes
import functools
import os
from typing import NamedTuple, Optional, Tuple

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libfastvr_attn.so")
# The same library with device-side index checks (FASTVR_BOUNDS_CHECK).
DEBUG_LIB_PATH = os.path.join(_HERE, "libfastvr_attn_debug.so")

FASTVR_OK = 0
FASTVR_ERR_INVALID_ARG = 1
FASTVR_ERR_UNSUPPORTED = 2
FASTVR_ERR_CAPACITY = 3
FASTVR_ERR_SEQUENCE = 4
FASTVR_ERR_CUDA = 5
FASTVR_ERR_TIMEOUT = 6
FASTVR_ERR_BOUNDS = 7


class fastvr_attn_config_t(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32),
                ("tokens_per_frame", ctypes.c_int32),
                ("frames_per_chunk", ctypes.c_int32),
                ("window_chunks", ctypes.c_int32),
                ("max_chunks", ctypes.c_int32),
                ("softmax_scale", ctypes.c_float)]


# Element types, rotary layouts and scalings, norms (include/fastvr_block.h).
FASTVR_BF16, FASTVR_F32 = 0, 1
ROTARY_LAYOUTS = {"interleaved": 0, "half": 1}
ROTARY_SCALINGS = {"none": 0, "linear": 1, "ntk": 2, "yarn": 3}
NORMS = {"none": 0, "rms": 1, "layer": 2}
ACTIVATIONS = {"silu": 0, "gelu": 1, "gelu_tanh": 2}


class fastvr_strides_t(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int64), ("token", ctypes.c_int64),
                ("head", ctypes.c_int64)]


class fastvr_rotary_config_t(ctypes.Structure):
    _fields_ = [("head_dim", ctypes.c_int32), ("rotary_dim", ctypes.c_int32),
                ("layout", ctypes.c_int32), ("axes", ctypes.c_int32),
                ("section", ctypes.c_int32 * 3), ("scaling", ctypes.c_int32),
                ("base", ctypes.c_double), ("factor", ctypes.c_double * 3),
                ("original_context", ctypes.c_double * 3),
                ("beta_fast", ctypes.c_double),
                ("beta_slow", ctypes.c_double),
                ("magnitude", ctypes.c_double)]


class fastvr_norm_config_t(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("tokens", ctypes.c_int32),
                ("dim", ctypes.c_int32), ("groups", ctypes.c_int32),
                ("pre", ctypes.c_int32), ("post", ctypes.c_int32),
                ("residual_dtype", ctypes.c_int32),
                ("block_dtype", ctypes.c_int32), ("eps", ctypes.c_float),
                ("residual_scale", ctypes.c_float)]


class fastvr_cross_config_t(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("q_tokens", ctypes.c_int32),
                ("kv_tokens", ctypes.c_int32), ("heads", ctypes.c_int32),
                ("kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("softmax_scale", ctypes.c_float)]


class fastvr_ffn_config_t(ctypes.Structure):
    _fields_ = [("tokens", ctypes.c_int32), ("dim", ctypes.c_int32),
                ("hidden", ctypes.c_int32), ("activation", ctypes.c_int32)]


# Every symbol the headers declare, with (restype, argtypes).
_VP, _I32, _I64, _SZ = (ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64,
                        ctypes.c_size_t)
_CFGP = ctypes.POINTER(fastvr_attn_config_t)
_STRP = ctypes.POINTER(fastvr_strides_t)
_ROTP = ctypes.POINTER(fastvr_rotary_config_t)
_NRMP = ctypes.POINTER(fastvr_norm_config_t)
_CRSP = ctypes.POINTER(fastvr_cross_config_t)
_FFNP = ctypes.POINTER(fastvr_ffn_config_t)
SIGNATURES = {
    "fastvr_kv_cache_bytes": (_I32, [_CFGP, ctypes.POINTER(_SZ)]),
    "fastvr_attn_plan": (_I32, [_CFGP, _VP, _SZ, ctypes.POINTER(_VP)]),
    "fastvr_kv_append": (_I32, [_VP, _VP, _VP, _I32, _VP]),
    "fastvr_chunk_attn_fwd": (_I32, [_VP, _VP, _VP, _VP, _VP]),
    "fastvr_plan_reset": (_I32, [_VP]),
    "fastvr_get_status": (_I32, [_VP]),
    "fastvr_plan_get_state": (_I32, [_VP, ctypes.POINTER(_I64),
                                     ctypes.POINTER(_I32)]),
    "fastvr_plan_set_state": (_I32, [_VP, _I64, _I32]),
    "fastvr_plan_visible": (_I32, [_VP, ctypes.POINTER(_I32),
                                   ctypes.POINTER(_I64),
                                   ctypes.POINTER(_I64),
                                   ctypes.POINTER(_I64)]),
    "fastvr_plan_launch_count": (_I32, [_VP, ctypes.POINTER(_I64)]),
    "fastvr_one_step_update": (_I32, [_VP, _VP, _VP, _I64, ctypes.c_float,
                                      _I32, _VP]),
    "fastvr_blockcausal_bwd_scratch_bytes": (_I32, [_CFGP, _I32,
                                                    ctypes.POINTER(_SZ)]),
    "fastvr_blockcausal_attn_bwd": (_I32, [_CFGP, _I32] + [_VP] * 10 +
                                    [_SZ, _VP]),
    "fastvr_blockcausal_attn_fwd": (_I32, [_CFGP, _I32, _VP, _VP, _VP, _VP,
                                           _VP, _VP]),
    "fastvr_chunk_attn_fwd_static": (_I32, [_CFGP, _VP, _I32, _VP, _VP, _I64,
                                            _I32, ctypes.POINTER(_I64),
                                            ctypes.POINTER(_I64), _VP, _VP,
                                            _VP]),
    "fastvr_debug_inject_stall": (_I32, [_VP, _I32, ctypes.c_uint64]),
    "fastvr_debug_shift_next_append": (_I32, [_VP, _I64]),
    "fastvr_get_device_status": (_I32, []),
    "fastvr_debug_inject_stall_noplan": (_I32, [_I32, ctypes.c_uint64]),
    "fastvr_plan_destroy": (None, [_VP]),
    "fastvr_status_string": (ctypes.c_char_p, [_I32]),
    "fastvr_rotary_frequencies": (_I32, [_ROTP,
                                         ctypes.POINTER(ctypes.c_double),
                                         ctypes.POINTER(ctypes.c_double)]),
    "fastvr_rotary": (_I32, [_ROTP] + [_I32] * 5 + [_VP, _STRP, _VP, _STRP,
                                                    _VP, _I64, _VP, _STRP,
                                                    _VP, _STRP, _I32, _VP]),
    "fastvr_gated_norm_fwd": (_I32, [_NRMP] + [_VP] * 10),
    "fastvr_gated_norm_bwd_scratch_bytes": (_I32, [_NRMP,
                                                   ctypes.POINTER(_SZ)]),
    "fastvr_gated_norm_bwd": (_I32, [_NRMP] + [_VP] * 16 + [_SZ, _VP]),
    "fastvr_q4_cache_bytes": (_I32, [_CFGP, _I32, ctypes.POINTER(_SZ)]),
    "fastvr_q4_workspace_bytes": (_I32, [_CFGP, _I32, ctypes.POINTER(_SZ)]),
    "fastvr_q4_plan": (_I32, [_CFGP, _I32, _VP, _SZ, _VP, _SZ,
                              ctypes.POINTER(_VP)]),
    "fastvr_q4_append": (_I32, [_VP, _VP, _STRP, _VP, _STRP, _I32, _VP]),
    "fastvr_q4_attn_fwd": (_I32, [_VP] * 6),
    "fastvr_q4_read": (_I32, [_VP, _I64, _VP, _VP, _VP]),
    "fastvr_cross_attn_fwd": (_I32, [_CRSP] + [_VP, _STRP] * 3 +
                              [_VP, _VP, _STRP, _VP, _VP]),
    "fastvr_cross_attn_bwd_scratch_bytes": (_I32, [_CRSP,
                                                   ctypes.POINTER(_SZ)]),
    "fastvr_cross_attn_bwd": (_I32, [_CRSP] + [_VP, _STRP] * 3 + [_VP] +
                              [_VP, _STRP] * 2 + [_VP] + [_VP, _STRP] * 3 +
                              [_VP, _SZ, _VP]),
    "fastvr_gated_ffn_fwd": (_I32, [_FFNP, _VP, _I64] + [_VP] * 6),
    "fastvr_gated_ffn_bwd_scratch_bytes": (_I32, [_FFNP,
                                                  ctypes.POINTER(_SZ)]),
    "fastvr_gated_ffn_bwd": (_I32, [_FFNP, _VP, _VP, _I64] + [_VP] * 8 +
                             [_SZ, _VP]),
}


def _load(path: str = LIB_PATH) -> ctypes.CDLL:
    if not os.path.exists(path):
        raise ImportError(
            f"{path} is missing: build it with "
            "`python -m paper_2609_36757_gb300.build` (there is no fallback)")
    lib = ctypes.CDLL(path)
    for name, (res, args) in SIGNATURES.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    return lib


lib = _load()


def use_library(path: str) -> ctypes.CDLL:
    """Route every call of this module to the library at path (e.g.
    DEBUG_LIB_PATH) and return the one used before."""
    global lib
    previous, lib = lib, _load(path)
    return previous


class FastVRError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {fastvr_status_string(status)}")


def _check(status: int, where: str) -> None:
    if status != FASTVR_OK:
        raise FastVRError(status, where)


# ------------------------------------------------------------ C-named calls
def fastvr_status_string(status: int) -> str:
    return lib.fastvr_status_string(status).decode()


def fastvr_kv_cache_bytes(cfg: fastvr_attn_config_t) -> int:
    n = _SZ(0)
    _check(lib.fastvr_kv_cache_bytes(ctypes.byref(cfg), ctypes.byref(n)),
           "fastvr_kv_cache_bytes")
    return n.value


def fastvr_attn_plan(cfg: fastvr_attn_config_t, kv_cache: int,
                     nbytes: int) -> int:
    plan = _VP()
    _check(lib.fastvr_attn_plan(ctypes.byref(cfg), kv_cache, nbytes,
                                ctypes.byref(plan)), "fastvr_attn_plan")
    return plan.value


def fastvr_kv_append(plan: int, k_new: int, v_new: int, frames: int,
                     stream: int) -> None:
    _check(lib.fastvr_kv_append(plan, k_new, v_new, frames, stream),
           "fastvr_kv_append")


def fastvr_chunk_attn_fwd(plan: int, q: int, out: int, lse: int,
                          stream: int) -> None:
    _check(lib.fastvr_chunk_attn_fwd(plan, q, out, lse, stream),
           "fastvr_chunk_attn_fwd")


def fastvr_plan_reset(plan: int) -> None:
    _check(lib.fastvr_plan_reset(plan), "fastvr_plan_reset")


def fastvr_get_status(plan: int) -> int:
    return lib.fastvr_get_status(plan)


def fastvr_plan_get_state(plan: int) -> Tuple[int, int]:
    c, f = _I64(0), _I32(0)
    _check(lib.fastvr_plan_get_state(plan, ctypes.byref(c), ctypes.byref(f)),
           "fastvr_plan_get_state")
    return c.value, f.value


def fastvr_plan_set_state(plan: int, chunks: int, last_frames: int) -> None:
    _check(lib.fastvr_plan_set_state(plan, chunks, last_frames),
           "fastvr_plan_set_state")


def fastvr_plan_visible(plan: int):
    """[(start, len), ...] token ranges of a head's cache, and their total."""
    n = _I32(0)
    st, ln = (_I64 * 2)(), (_I64 * 2)()
    tot = _I64(0)
    _check(lib.fastvr_plan_visible(plan, ctypes.byref(n), st, ln,
                                   ctypes.byref(tot)), "fastvr_plan_visible")
    return [(st[i], ln[i]) for i in range(n.value)], tot.value


def fastvr_chunk_attn_fwd_static(cfg: fastvr_attn_config_t, q: int,
                                 q_frames: int, k_cache: int, v_cache: int,
                                 cache_tokens: int, segments, out: int,
                                 lse: int, stream: int) -> None:
    """The allocation-free attention entry point; `segments` is a list of
    (start, len) key ranges of one head's cache."""
    n = len(segments)
    st = (_I64 * max(2, n))(*[s for s, _ in segments])
    ln = (_I64 * max(2, n))(*[l for _, l in segments])
    _check(lib.fastvr_chunk_attn_fwd_static(
        ctypes.byref(cfg), q, q_frames, k_cache, v_cache, cache_tokens, n, st,
        ln, out, lse, stream), "fastvr_chunk_attn_fwd_static")


def fastvr_blockcausal_attn_fwd(cfg: fastvr_attn_config_t, num_frames: int,
                                q: int, k: int, v: int, out: int, lse: int,
                                stream: int) -> None:
    _check(lib.fastvr_blockcausal_attn_fwd(ctypes.byref(cfg), num_frames, q,
                                           k, v, out, lse, stream),
           "fastvr_blockcausal_attn_fwd")


def blockcausal_attention(cfg: fastvr_attn_config_t, q, k, v,
                          want_lse: bool = False):
    """Torch convenience for fastvr_blockcausal_attn_fwd: q, k, v contiguous
    bfloat16 CUDA tensors [B, L, H, d]; runs on the current stream."""
    import torch
    for t in (q, k, v):
        if t.dtype != torch.bfloat16 or not t.is_cuda or not t.is_contiguous():
            raise ValueError("q, k, v must be contiguous bfloat16 CUDA tensors")
    if not (q.shape == k.shape == v.shape):
        raise ValueError("q, k, v differ in shape")
    B, L, H, d = q.shape
    if (B, H, d) != (cfg.batch, cfg.heads, cfg.head_dim) or \
            L % cfg.tokens_per_frame:
        raise ValueError(f"q has shape {tuple(q.shape)}")
    out = torch.empty_like(q)
    lse = (torch.empty((B, H, L), dtype=torch.float32, device=q.device)
           if want_lse else None)
    fastvr_blockcausal_attn_fwd(cfg, L // cfg.tokens_per_frame, q.data_ptr(),
                                k.data_ptr(), v.data_ptr(), out.data_ptr(),
                                0 if lse is None else lse.data_ptr(),
                                torch.cuda.current_stream().cuda_stream)
    return (out, lse) if want_lse else out


def fastvr_blockcausal_bwd_scratch_bytes(cfg: fastvr_attn_config_t,
                                         num_frames: int) -> int:
    n = _SZ(0)
    _check(lib.fastvr_blockcausal_bwd_scratch_bytes(ctypes.byref(cfg),
                                                    num_frames, ctypes.byref(n)),
           "fastvr_blockcausal_bwd_scratch_bytes")
    return n.value


def fastvr_blockcausal_attn_bwd(cfg, num_frames, q, k, v, out, dout, lse, dq,
                                dk, dv, scratch, scratch_bytes, stream) -> None:
    _check(lib.fastvr_blockcausal_attn_bwd(
        ctypes.byref(cfg), num_frames, q, k, v, out, dout, lse, dq, dk, dv,
        scratch, scratch_bytes, stream), "fastvr_blockcausal_attn_bwd")


def blockcausal_attention_bwd(cfg: fastvr_attn_config_t, q, k, v, out, dout,
                              lse):
    """Torch convenience for fastvr_blockcausal_attn_bwd: bfloat16 CUDA
    tensors [B, L, H, d] and the forward's float32 lse [B, H, L]; returns
    (dq, dk, dv).  The scratch is allocated with torch."""
    import torch
    L = q.shape[1]
    frames = L // cfg.tokens_per_frame
    nbytes = fastvr_blockcausal_bwd_scratch_bytes(cfg, frames)
    scratch = torch.empty(nbytes // 4, dtype=torch.float32, device=q.device)
    dq, dk, dv = (torch.empty_like(q) for _ in range(3))
    fastvr_blockcausal_attn_bwd(
        cfg, frames, q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(),
        dout.data_ptr(), lse.data_ptr(), dq.data_ptr(), dk.data_ptr(),
        dv.data_ptr(), scratch.data_ptr(), nbytes,
        torch.cuda.current_stream().cuda_stream)
    return dq, dk, dv


def fastvr_one_step_update(z_lq: int, v: int, z_hat: int, n: int,
                           sigma: float, dtype: int, stream: int) -> None:
    _check(lib.fastvr_one_step_update(z_lq, v, z_hat, n, sigma, dtype, stream),
           "fastvr_one_step_update")


def one_step_update(z_lq, v, sigma: float, out=None):
    """Torch convenience: z_lq bfloat16 or float32, v bfloat16, same shape,
    contiguous CUDA tensors; returns z_lq - sigma * v (in place when
    out is z_lq)."""
    import torch
    if v.dtype != torch.bfloat16 or z_lq.dtype not in (torch.bfloat16,
                                                       torch.float32):
        raise ValueError("z_lq must be bfloat16 or float32 and v bfloat16")
    if z_lq.shape != v.shape or not (z_lq.is_contiguous() and v.is_contiguous()):
        raise ValueError("z_lq and v must be contiguous and of one shape")
    if out is None:
        out = torch.empty_like(z_lq)
    fastvr_one_step_update(z_lq.data_ptr(), v.data_ptr(), out.data_ptr(),
                           z_lq.numel(), sigma,
                           0 if z_lq.dtype == torch.bfloat16 else 1,
                           torch.cuda.current_stream().cuda_stream)
    return out


def fastvr_plan_launch_count(plan: int) -> int:
    n = _I64(0)
    _check(lib.fastvr_plan_launch_count(plan, ctypes.byref(n)),
           "fastvr_plan_launch_count")
    return n.value


def fastvr_debug_inject_stall(plan: int, stall: int,
                              wait_limit_ns: int) -> None:
    _check(lib.fastvr_debug_inject_stall(plan, stall, wait_limit_ns),
           "fastvr_debug_inject_stall")


def fastvr_debug_shift_next_append(plan: int, tokens: int) -> None:
    _check(lib.fastvr_debug_shift_next_append(plan, tokens),
           "fastvr_debug_shift_next_append")


def fastvr_get_device_status() -> int:
    """Status of the calls without a plan on the current device (synchronises;
    a recorded failure is cleared once returned)."""
    return lib.fastvr_get_device_status()


def fastvr_debug_inject_stall_noplan(stall: int, wait_limit_ns: int) -> None:
    _check(lib.fastvr_debug_inject_stall_noplan(stall, wait_limit_ns),
           "fastvr_debug_inject_stall_noplan")


def fastvr_plan_destroy(plan: int) -> None:
    lib.fastvr_plan_destroy(plan)


def fastvr_rotary_frequencies(cfg: fastvr_rotary_config_t):
    """The rotary_dim / 2 angles per position (radians) in pair order, and
    the magnitude."""
    theta = (ctypes.c_double * max(1, cfg.rotary_dim // 2))()
    mag = ctypes.c_double(0)
    _check(lib.fastvr_rotary_frequencies(ctypes.byref(cfg), theta,
                                         ctypes.byref(mag)),
           "fastvr_rotary_frequencies")
    return list(theta), mag.value


def fastvr_rotary(cfg, batch, tokens, heads, kv_heads, dtype, q, q_str, k,
                  k_str, positions, pos_batch, q_out, q_out_str, k_out,
                  k_out_str, transpose, stream) -> None:
    """Strides are fastvr_strides_t or None (contiguous)."""
    _check(lib.fastvr_rotary(cfg, batch, tokens, heads, kv_heads, dtype, q,
                             q_str, k, k_str, positions, pos_batch, q_out,
                             q_out_str, k_out, k_out_str, transpose, stream),
           "fastvr_rotary")


def fastvr_gated_norm_fwd(cfg, x, y, gate, scale, shift, pre_weight,
                          post_weight, r, h, stream) -> None:
    _check(lib.fastvr_gated_norm_fwd(cfg, x, y, gate, scale, shift,
                                     pre_weight, post_weight, r, h, stream),
           "fastvr_gated_norm_fwd")


def fastvr_gated_norm_bwd_scratch_bytes(cfg: fastvr_norm_config_t) -> int:
    n = _SZ(0)
    _check(lib.fastvr_gated_norm_bwd_scratch_bytes(cfg, ctypes.byref(n)),
           "fastvr_gated_norm_bwd_scratch_bytes")
    return n.value


def fastvr_gated_norm_bwd(cfg, dr, dh, r, y, gate, scale, pre_weight,
                          post_weight, dx, dy, dgate, dscale, dshift,
                          dpre_weight, dpost_weight, scratch, scratch_bytes,
                          stream) -> None:
    _check(lib.fastvr_gated_norm_bwd(
        cfg, dr, dh, r, y, gate, scale, pre_weight, post_weight, dx, dy,
        dgate, dscale, dshift, dpre_weight, dpost_weight, scratch,
        scratch_bytes, stream), "fastvr_gated_norm_bwd")


def fastvr_q4_cache_bytes(cfg: fastvr_attn_config_t, kv_heads: int) -> int:
    n = _SZ(0)
    _check(lib.fastvr_q4_cache_bytes(ctypes.byref(cfg), kv_heads,
                                     ctypes.byref(n)), "fastvr_q4_cache_bytes")
    return n.value


def fastvr_q4_workspace_bytes(cfg: fastvr_attn_config_t,
                              kv_heads: int) -> int:
    n = _SZ(0)
    _check(lib.fastvr_q4_workspace_bytes(ctypes.byref(cfg), kv_heads,
                                         ctypes.byref(n)),
           "fastvr_q4_workspace_bytes")
    return n.value


def fastvr_q4_plan(cfg: fastvr_attn_config_t, kv_heads: int, cache: int,
                   cache_bytes: int, workspace: int,
                   workspace_bytes: int) -> int:
    plan = _VP()
    _check(lib.fastvr_q4_plan(ctypes.byref(cfg), kv_heads, cache, cache_bytes,
                              workspace, workspace_bytes, ctypes.byref(plan)),
           "fastvr_q4_plan")
    return plan.value


def fastvr_q4_append(plan: int, k: int, k_str, v: int, v_str, frames: int,
                     stream: int) -> None:
    """Strides are fastvr_strides_t or None (contiguous)."""
    _check(lib.fastvr_q4_append(plan, k, k_str, v, v_str, frames, stream),
           "fastvr_q4_append")


def fastvr_q4_attn_fwd(plan: int, q: int, first_chunk: int, out: int,
                       lse: int, stream: int) -> None:
    _check(lib.fastvr_q4_attn_fwd(plan, q, first_chunk, out, lse, stream),
           "fastvr_q4_attn_fwd")


def fastvr_q4_read(plan: int, chunk: int, k: int, v: int,
                   stream: int) -> None:
    _check(lib.fastvr_q4_read(plan, chunk, k, v, stream), "fastvr_q4_read")


def fastvr_cross_attn_fwd(cfg, q, q_str, k, k_str, v, v_str, kv_len, out,
                          out_str, lse, stream) -> None:
    """Strides are fastvr_strides_t or None (contiguous)."""
    _check(lib.fastvr_cross_attn_fwd(cfg, q, q_str, k, k_str, v, v_str, kv_len,
                                     out, out_str, lse, stream),
           "fastvr_cross_attn_fwd")


def fastvr_cross_attn_bwd_scratch_bytes(cfg: fastvr_cross_config_t) -> int:
    n = _SZ(0)
    _check(lib.fastvr_cross_attn_bwd_scratch_bytes(cfg, ctypes.byref(n)),
           "fastvr_cross_attn_bwd_scratch_bytes")
    return n.value


def fastvr_cross_attn_bwd(cfg, q, q_str, k, k_str, v, v_str, kv_len, out,
                          out_str, dout, dout_str, lse, dq, dq_str, dk, dk_str,
                          dv, dv_str, scratch, scratch_bytes, stream) -> None:
    """Strides are fastvr_strides_t or None (contiguous)."""
    _check(lib.fastvr_cross_attn_bwd(
        cfg, q, q_str, k, k_str, v, v_str, kv_len, out, out_str, dout,
        dout_str, lse, dq, dq_str, dk, dk_str, dv, dv_str, scratch,
        scratch_bytes, stream), "fastvr_cross_attn_bwd")


def fastvr_gated_ffn_fwd(cfg, x, x_row, w_gate, w_up, h, g, u,
                         stream) -> None:
    _check(lib.fastvr_gated_ffn_fwd(cfg, x, x_row, w_gate, w_up, h, g, u,
                                    stream), "fastvr_gated_ffn_fwd")


def fastvr_gated_ffn_bwd_scratch_bytes(cfg: fastvr_ffn_config_t) -> int:
    n = _SZ(0)
    _check(lib.fastvr_gated_ffn_bwd_scratch_bytes(cfg, ctypes.byref(n)),
           "fastvr_gated_ffn_bwd_scratch_bytes")
    return n.value


def fastvr_gated_ffn_bwd(cfg, dh, x, x_row, w_gate, w_up, g, u, dx, dw_gate,
                         dw_up, scratch, scratch_bytes, stream) -> None:
    _check(lib.fastvr_gated_ffn_bwd(cfg, dh, x, x_row, w_gate, w_up, g, u, dx,
                                    dw_gate, dw_up, scratch, scratch_bytes,
                                    stream), "fastvr_gated_ffn_bwd")


def make_config(batch: int, heads: int, head_dim: int, tokens_per_frame: int,
                frames_per_chunk: int, window_chunks: int = -1,
                max_chunks: int = 0, softmax_scale: float = 0.0
                ) -> fastvr_attn_config_t:
    return fastvr_attn_config_t(batch, heads, head_dim, tokens_per_frame,
                                frames_per_chunk, window_chunks, max_chunks,
                                softmax_scale)


# ------------------------------------------------------- torch convenience
class StreamingAttention:
    """One video stream: a caller-side KV cache tensor plus a plan.

    append(k, v) and forward(q) take bfloat16 CUDA tensors [B, f*N, H, d]
    (contiguous, token-major) and enqueue on the current CUDA stream."""

    def __init__(self, cfg: fastvr_attn_config_t, device=None):
        import torch
        self.cfg = cfg
        self.nbytes = fastvr_kv_cache_bytes(cfg)
        self.cache = torch.empty(self.nbytes, dtype=torch.uint8,
                                 device=device or "cuda")
        self.plan = fastvr_attn_plan(cfg, self.cache.data_ptr(), self.nbytes)

    def __del__(self):
        plan = getattr(self, "plan", None)
        if plan:
            fastvr_plan_destroy(plan)
            self.plan = None

    def _check_chunk(self, t, name: str) -> int:
        import torch
        c = self.cfg
        if t.dtype != torch.bfloat16 or not t.is_cuda or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous bfloat16 CUDA tensor")
        B, L, H, d = t.shape
        if (B, H, d) != (c.batch, c.heads, c.head_dim) or L % c.tokens_per_frame:
            raise ValueError(f"{name} has shape {tuple(t.shape)}")
        return L // c.tokens_per_frame

    @staticmethod
    def _stream() -> int:
        import torch
        return torch.cuda.current_stream().cuda_stream

    def append(self, k, v) -> None:
        frames = self._check_chunk(k, "k")
        if self._check_chunk(v, "v") != frames:
            raise ValueError("k and v differ in length")
        fastvr_kv_append(self.plan, k.data_ptr(), v.data_ptr(), frames,
                         self._stream())

    def forward(self, q, out=None, lse: Optional[object] = None,
                want_lse: bool = False):
        import torch
        self._check_chunk(q, "q")
        if out is None:
            out = torch.empty_like(q)
        if lse is None and want_lse:
            B, L, H, _ = q.shape
            lse = torch.empty((B, H, L), dtype=torch.float32, device=q.device)
        fastvr_chunk_attn_fwd(self.plan, q.data_ptr(), out.data_ptr(),
                              0 if lse is None else lse.data_ptr(),
                              self._stream())
        return (out, lse) if want_lse or lse is not None else out

    def reset(self) -> None:
        fastvr_plan_reset(self.plan)

    def launch_count(self) -> int:
        return fastvr_plan_launch_count(self.plan)

    def status(self) -> int:
        return fastvr_get_status(self.plan)

    def visible(self):
        return fastvr_plan_visible(self.plan)

    def state(self) -> Tuple[int, int]:
        return fastvr_plan_get_state(self.plan)

    def set_state(self, chunks: int, last_frames: int) -> None:
        fastvr_plan_set_state(self.plan, chunks, last_frames)


# ------------------------------------------- operators around the attention
# These wrappers are on the path of a decode step, where the host's time is
# what a call costs: they look torch up once, and ask for the stream's handle
# directly (torch.cuda.current_stream() builds a stream object, 2.9 us on the
# measured host against 0.1).
_CODES: dict = {}
_torch = _raw_stream = _current_device = None


def _setup():
    """torch, with the tables that need it filled in."""
    global _current_device, _raw_stream, _torch
    import torch
    _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
        lambda i: torch.cuda.current_stream(i).cuda_stream)
    _current_device = getattr(torch._C, "_cuda_getDevice",
                              torch.cuda.current_device)
    _CODES[torch.bfloat16] = FASTVR_BF16
    _CODES[torch.float32] = FASTVR_F32
    _torch = torch
    return torch


def _stream_of(*tensors) -> int:
    """Handle of the current device's current stream, where all tensors of a
    call lie (None: absent)."""
    device = _current_device()
    for t in tensors:
        if t is not None and t.get_device() != device:
            raise ValueError("a call's tensors must lie on the current CUDA "
                             "device")
    return _raw_stream(device)


def _dtype_code(dtype) -> int:
    code = _CODES.get(dtype)
    if code is None:
        raise ValueError("tensors must be bfloat16 or float32")
    return code


@functools.lru_cache(maxsize=64)
def _strides_ref(batch: int, token: int, head: int):
    return ctypes.byref(fastvr_strides_t(batch, token, head))


def _head_strides(t, name: str):
    """fastvr_strides_t of a [B, L, H, d] tensor whose heads are contiguous,
    None when the whole tensor is."""
    strides = t.stride()
    if len(strides) != 4:
        raise ValueError(f"{name} must be a CUDA tensor [B, L, H, d]")
    if t.is_contiguous():
        return None
    if strides[3] != 1:
        raise ValueError(f"the elements of a head of {name} must be contiguous")
    return _strides_ref(*strides[:3])


def make_rotary_config(head_dim: int, rotary_dim: Optional[int] = None,
                       layout: str = "interleaved", sections=None,
                       base: float = 10000.0, scaling: str = "none",
                       factors=None, original_contexts=None,
                       beta_fast: float = 32.0, beta_slow: float = 1.0,
                       magnitude: float = 0.0) -> fastvr_rotary_config_t:
    """Rotary positions of heads of head_dim elements, the first rotary_dim
    of them rotated.  sections: pairs per axis (default: one axis); factors
    and original_contexts: per axis, for the scalings that use them."""
    rot = head_dim if rotary_dim is None else rotary_dim
    sections = [rot // 2] if sections is None else list(sections)
    n = len(sections)
    if n > 3:
        raise ValueError("at most three axes")
    three = lambda v, fill: (list(v) if v is not None else [fill] * n) + \
        [fill] * (3 - n)
    return fastvr_rotary_config_t(
        head_dim, rot, ROTARY_LAYOUTS[layout], n,
        (ctypes.c_int32 * 3)(*three(sections, 0)), ROTARY_SCALINGS[scaling],
        base, (ctypes.c_double * 3)(*three(factors, 1.0)),
        (ctypes.c_double * 3)(*three(original_contexts, 0.0)), beta_fast,
        beta_slow, magnitude)


def rotary(cfg: fastvr_rotary_config_t, q, k, positions, out=None,
           transpose: bool = False):
    """Torch convenience for fastvr_rotary: q [B, L, H, d] and k [B, L, Hkv,
    d] (or None), bfloat16 or float32, heads contiguous, any other strides
    (slices of a fused projection); positions int32 [L, axes] or [B or 1, L,
    axes].  Returns (q', k'), contiguous unless `out` gives the two outputs
    (out=(q, k) works in place)."""
    torch = _torch or _setup()
    code = _dtype_code(q.dtype)
    q_str = _head_strides(q, "q")
    B, L, H, d = q.shape
    Hk, k_str = 0, None
    if d != cfg.head_dim:
        raise ValueError(f"q has shape {tuple(q.shape)}")
    if k is not None:
        k_str = _head_strides(k, "k")
        shape = k.shape
        Hk = shape[2]
        if shape != (B, L, Hk, d) or k.dtype != q.dtype:
            raise ValueError("q and k differ in type or shape")
    if positions.dtype != torch.int32 or not positions.is_contiguous():
        raise ValueError("positions must be a contiguous int32 CUDA tensor")
    axes, shape = cfg.axes, positions.shape
    rows = shape[0] if len(shape) == 3 else 1
    if shape != ((rows, L, axes) if len(shape) == 3 else (L, axes)) or \
            rows != 1 and rows != B:
        raise ValueError(f"positions have shape {tuple(shape)}")
    if out is None:
        q_out = torch.empty_like(q, memory_format=torch.contiguous_format)
        k_out = None if k is None else torch.empty_like(
            k, memory_format=torch.contiguous_format)
        q_out_str = k_out_str = None
    else:
        q_out, k_out = out
        for o, i in ((q_out, q), (k_out, k)):
            if (o is None) != (i is None) or o is not None and \
                    (o.shape != i.shape or o.dtype != i.dtype):
                raise ValueError("outputs differ from the inputs")
        q_out_str = _head_strides(q_out, "the output for q")
        k_out_str = None if k is None else _head_strides(
            k_out, "the output for k")
    fastvr_rotary(cfg, B, L, H, Hk, code, q.data_ptr(), q_str,
                  0 if k is None else k.data_ptr(), k_str,
                  positions.data_ptr(), L * axes if rows > 1 else 0,
                  q_out.data_ptr(), q_out_str,
                  0 if k is None else k_out.data_ptr(), k_out_str,
                  int(transpose), _stream_of(q, k, positions, *(out or ())))
    return q_out, k_out


def rotary_bwd(cfg: fastvr_rotary_config_t, dq, dk, positions, out=None):
    """Gradients of rotary's inputs from those of its outputs."""
    return rotary(cfg, dq, dk, positions, out, transpose=True)


def make_norm_config(pre: str = "rms", post: str = "none", eps: float = 1e-6,
                     residual_scale: float = 1.0) -> fastvr_norm_config_t:
    """The norms of gated_norm; the shapes are taken from its tensors."""
    return fastvr_norm_config_t(0, 0, 0, 0, NORMS[pre], NORMS[post], 0, 0,
                                eps, residual_scale)


def _norm_call(cfg, x, y, mods, weights):
    """cfg for the tensors of a call, after the checks of their types and
    shapes."""
    torch = _torch or _setup()
    shape = x.shape
    if len(shape) != 3 or not x.is_contiguous():
        raise ValueError("x must be a contiguous CUDA tensor [B, L, D]")
    B, L, D = shape
    code = _dtype_code(x.dtype)
    block = FASTVR_BF16
    for t in y:
        if t is not None:
            if t.shape != shape or not t.is_contiguous():
                raise ValueError(
                    "block tensors must be contiguous and of x's shape")
            block = _dtype_code(t.dtype)
    f32, groups = torch.float32, 0
    for t in mods:
        if t is not None:
            s = t.shape
            if t.dtype != f32 or not t.is_contiguous() or \
                    len(s) != 3 or s[0] != B or s[2] != D:
                raise ValueError("gate, scale and shift must be contiguous "
                                 "float32 CUDA tensors [B, G, D]")
            if groups and s[1] != groups:
                raise ValueError("gate, scale and shift differ in groups")
            groups = s[1]
    for t in weights:
        if t is not None and (t.dtype != f32 or
                              t.shape != (D,) or not t.is_contiguous()):
            raise ValueError("weights must be contiguous float32 CUDA "
                             "tensors [D]")
    return fastvr_norm_config_t(B, L, D, groups or 1, cfg.pre, cfg.post, code,
                                block, cfg.eps, cfg.residual_scale)


def _ptr(t) -> int:
    return 0 if t is None else t.data_ptr()


def gated_norm(cfg: fastvr_norm_config_t, x, y, gate=None, scale=None,
               shift=None, pre_weight=None, post_weight=None, block_dtype=None,
               want_r: bool = True, want_h: bool = True):
    """Torch convenience for fastvr_gated_norm_fwd: x [B, L, D] (bfloat16 or
    float32) and y the same shape (or None: no block output), gate, scale and
    shift float32 [B, G, D], weights float32 [D].  Returns (r, h), None for
    the one not wanted; h has y's type (block_dtype without y)."""
    torch = _torch or _setup()
    c = _norm_call(cfg, x, (y,), (gate, scale, shift),
                   (pre_weight, post_weight))
    block = (block_dtype or torch.bfloat16) if y is None else y.dtype
    if y is None:
        c.block_dtype = _dtype_code(block)
    r = torch.empty_like(x) if want_r else None
    h = torch.empty_like(x, dtype=block) if want_h else None
    fastvr_gated_norm_fwd(c, x.data_ptr(), _ptr(y), _ptr(gate), _ptr(scale),
                          _ptr(shift), _ptr(pre_weight), _ptr(post_weight),
                          _ptr(r), _ptr(h),
                          _stream_of(x, y, gate, scale, shift, pre_weight,
                                     post_weight))
    return r, h


class NormGrads(NamedTuple):
    """Gradients of gated_norm; None where the forward had no such input."""
    dx: object
    dy: object
    dgate: object
    dscale: object
    dshift: object
    dpre_weight: object
    dpost_weight: object


def gated_norm_bwd(cfg: fastvr_norm_config_t, dr, dh, r, y, gate=None,
                   scale=None, pre_weight=None, post_weight=None,
                   want_dshift: Optional[bool] = None) -> NormGrads:
    """Torch convenience for fastvr_gated_norm_bwd: dr, dh the gradients of r
    and h (either may be None), r the forward's r.  dshift is formed when
    scale is given, or as want_dshift says (the groups are then gate's or
    scale's, or one)."""
    torch = _torch or _setup()
    if dr is not None and (dr.shape != r.shape or dr.dtype != r.dtype or
                           not dr.is_contiguous()):
        raise ValueError("dr must be contiguous and of r's type and shape")
    c = _norm_call(cfg, r, (dh, y), (gate, scale), (pre_weight, post_weight))
    if dh is not None and y is not None and dh.dtype != y.dtype:
        raise ValueError("dh and y differ in type")
    new = lambda *s: torch.empty(s, dtype=torch.float32, device=r.device)
    like = lambda t: None if t is None else torch.empty_like(t)
    B, L, D = r.shape
    if want_dshift is None:
        want_dshift = scale is not None
    dshift = new(B, c.groups, D) if want_dshift else None
    g = NormGrads(torch.empty_like(r), like(y),
                  None if y is None else like(gate), like(scale), dshift,
                  like(pre_weight), None if y is None else like(post_weight))
    nbytes = fastvr_gated_norm_bwd_scratch_bytes(c)
    scratch = new((nbytes + 3) // 4)
    fastvr_gated_norm_bwd(c, _ptr(dr), _ptr(dh), r.data_ptr(), _ptr(y),
                          _ptr(gate), _ptr(scale), _ptr(pre_weight),
                          _ptr(post_weight), *(_ptr(t) for t in g),
                          scratch.data_ptr(), nbytes,
                          _stream_of(r, y, dr, dh, gate, scale, pre_weight,
                                     post_weight))
    return g


def make_cross_config(softmax_scale: float = 0.0) -> fastvr_cross_config_t:
    """Cross attention with a softmax scale (0: 1 / sqrt(d)); the shapes are
    taken from its tensors."""
    return fastvr_cross_config_t(0, 0, 0, 0, 0, 0, softmax_scale)


def _check_32_bits(*sizes) -> None:
    """ctypes keeps the low 32 bits of a size without a word."""
    if max(sizes) >> 31:
        raise ValueError("a call's sizes must be below 2^31")


def _cross_call(cfg, q, k, v, kv_len):
    """cfg for the tensors of a call and the strides of q, k and v, after the
    checks of their types and shapes."""
    torch = _torch or _setup()
    bf16 = torch.bfloat16
    if q.dtype != bf16 or k.dtype != bf16 or v.dtype != bf16:
        raise ValueError("q, k and v must be bfloat16")
    q_str = _head_strides(q, "q")
    k_str, v_str = _head_strides(k, "k"), _head_strides(v, "v")
    B, L, H, d = q.shape
    _, T, K, _ = shape = k.shape
    if shape != (B, T, K, d) or v.shape != shape:
        raise ValueError("q, k and v differ in batch or head size, or k and v "
                         "in shape")
    if kv_len is not None and (kv_len.dtype != torch.int32 or
                               kv_len.shape != (B,) or
                               not kv_len.is_contiguous()):
        raise ValueError("kv_len must be a contiguous int32 CUDA tensor [B]")
    _check_32_bits(B, L, T, H, K, d)
    return (fastvr_cross_config_t(B, L, T, H, K, d, cfg.softmax_scale), q_str,
            k_str, v_str)


def cross_attention(cfg: fastvr_cross_config_t, q, k, v, kv_len=None,
                    want_lse: bool = False):
    """Torch convenience for fastvr_cross_attn_fwd: q [B, L, H, d] and k, v
    [B, T, Hkv, d] bfloat16, heads contiguous, any other strides (halves of a
    fused projection; one prompt expanded over the batch); kv_len int32 [B]:
    the keys that each batch entry sees (none: all).  Returns out [B, L, H, d],
    or (out, lse) with the float32 log-sum-exp [B, H, L]."""
    c, q_str, k_str, v_str = _cross_call(cfg, q, k, v, kv_len)
    torch = _torch
    out = torch.empty_like(q, memory_format=torch.contiguous_format)
    lse = (torch.empty((c.batch, c.heads, c.q_tokens), dtype=torch.float32,
                       device=q.device) if want_lse else None)
    fastvr_cross_attn_fwd(c, q.data_ptr(), q_str, k.data_ptr(), k_str,
                          v.data_ptr(), v_str, _ptr(kv_len), out.data_ptr(),
                          None, _ptr(lse), _stream_of(q, k, v, kv_len))
    return (out, lse) if want_lse else out


class CrossGrads(NamedTuple):
    """Gradients of cross_attention."""
    dq: object
    dk: object
    dv: object


def cross_attention_bwd(cfg: fastvr_cross_config_t, q, k, v, out, dout, lse,
                        kv_len=None) -> CrossGrads:
    """Torch convenience for fastvr_cross_attn_bwd: out and lse are
    cross_attention's, dout out's gradient (heads contiguous, any other
    strides).  The gradients are contiguous, with q's, k's and v's shapes: of
    a prompt expanded over the batch, a gradient for each entry."""
    c, q_str, k_str, v_str = _cross_call(cfg, q, k, v, kv_len)
    torch = _torch
    for t, name in ((out, "out"), (dout, "dout")):
        if t.dtype != torch.bfloat16 or t.shape != q.shape:
            raise ValueError(f"{name} must be bfloat16 and of q's shape")
    if lse.dtype != torch.float32 or not lse.is_contiguous() or \
            lse.shape != (c.batch, c.heads, c.q_tokens):
        raise ValueError("lse must be contiguous float32 [B, H, L]")
    like = lambda t: torch.empty_like(t, memory_format=torch.contiguous_format)
    g = CrossGrads(like(q), like(k), like(v))
    nbytes = fastvr_cross_attn_bwd_scratch_bytes(c)
    scratch = torch.empty((nbytes + 3) // 4, dtype=torch.float32,
                          device=q.device)
    fastvr_cross_attn_bwd(
        c, q.data_ptr(), q_str, k.data_ptr(), k_str, v.data_ptr(), v_str,
        _ptr(kv_len), out.data_ptr(), _head_strides(out, "out"),
        dout.data_ptr(), _head_strides(dout, "dout"), lse.data_ptr(),
        g.dq.data_ptr(), None, g.dk.data_ptr(), None, g.dv.data_ptr(), None,
        scratch.data_ptr(), nbytes,
        _stream_of(q, k, v, kv_len, out, dout, lse))
    return g


def make_ffn_config(activation: str = "silu") -> fastvr_ffn_config_t:
    """A gated feed-forward with the activation "silu", "gelu" or "gelu_tanh";
    the shapes are taken from its tensors."""
    return fastvr_ffn_config_t(0, 0, 0, ACTIVATIONS[activation])


def _ffn_call(cfg, x, w_gate, w_up, hidden):
    """cfg for the tensors of a call and x's row stride, after the checks of
    their types and shapes; hidden: tensors [..., hidden]."""
    torch = _torch or _setup()
    bf16 = torch.bfloat16
    if x.dtype != bf16 or w_gate.dtype != bf16 or w_up.dtype != bf16:
        raise ValueError("x and the weights must be bfloat16")
    shape = w_gate.shape
    if len(shape) != 2 or w_up.shape != shape or \
            not w_gate.is_contiguous() or not w_up.is_contiguous():
        raise ValueError("w_gate and w_up must be contiguous [F, D]")
    F, D = shape
    lead = x.shape[:-1]
    if not lead or x.shape[-1] != D:
        raise ValueError("x must be [..., D]")
    row = D
    if not x.is_contiguous():
        try:
            row = x.view(-1, D).stride(0)
        except RuntimeError:
            row = 0
        if row < D or x.stride(-1) != 1:
            raise ValueError("x's rows must be contiguous and evenly spaced")
    for t in hidden:
        if t.dtype != bf16 or t.shape != lead + (F,) or not t.is_contiguous():
            raise ValueError("dh and the saved projections must be contiguous "
                             "bfloat16 [..., F]")
    tokens = x.numel() // D if D else 0
    _check_32_bits(tokens, F, D)
    return fastvr_ffn_config_t(tokens, D, F, cfg.activation), row


def gated_ffn(cfg: fastvr_ffn_config_t, x, w_gate, w_up,
              want_saved: bool = False):
    """Torch convenience for fastvr_gated_ffn_fwd: x [..., D] (rows evenly
    spaced), w_gate and w_up [F, D], bfloat16.  Returns h [..., F], or
    (h, (g, u)) with the projections that gated_ffn_bwd takes."""
    c, row = _ffn_call(cfg, x, w_gate, w_up, ())
    empty, shape, kind = _torch.empty, x.shape[:-1] + (c.hidden,), x.dtype
    h = empty(shape, dtype=kind, device=x.device)
    g = u = None
    if want_saved:
        g, u = (empty(shape, dtype=kind, device=x.device) for _ in "gu")
    fastvr_gated_ffn_fwd(c, x.data_ptr(), row, w_gate.data_ptr(),
                         w_up.data_ptr(), h.data_ptr(), _ptr(g), _ptr(u),
                         _stream_of(x, w_gate, w_up))
    return (h, (g, u)) if want_saved else h


class FfnGrads(NamedTuple):
    """Gradients of gated_ffn; None for frozen weights."""
    dx: object
    dw_gate: object
    dw_up: object


def gated_ffn_bwd(cfg: fastvr_ffn_config_t, dh, x, w_gate, w_up, saved,
                  want_dw: bool = True) -> FfnGrads:
    """Torch convenience for fastvr_gated_ffn_bwd: dh [..., F] the gradient of
    h, saved the forward's (g, u).  The scratch is allocated with torch."""
    g, u = saved
    c, row = _ffn_call(cfg, x, w_gate, w_up, (dh, g, u))
    torch = _torch
    dx = torch.empty_like(x, memory_format=torch.contiguous_format)
    dw = [torch.empty_like(w) if want_dw else None for w in (w_gate, w_up)]
    nbytes = fastvr_gated_ffn_bwd_scratch_bytes(c)
    scratch = torch.empty(nbytes, dtype=torch.uint8, device=x.device)
    fastvr_gated_ffn_bwd(c, dh.data_ptr(), x.data_ptr(), row,
                         w_gate.data_ptr(), w_up.data_ptr(), g.data_ptr(),
                         u.data_ptr(), dx.data_ptr(), _ptr(dw[0]),
                         _ptr(dw[1]), scratch.data_ptr(), nbytes,
                         _stream_of(x, dh, w_gate, w_up, g, u))
    return FfnGrads(dx, *dw)


class StreamingAttention4:
    """One video stream, or a batch of them, over a KV cache held in 4 bits.

    append(k, v) takes bfloat16 CUDA tensors [B, f*N, kv_heads, d] (heads
    contiguous, any other strides; f up to k, or several whole chunks at
    once), forward(q) contiguous [B, f*N, heads, d]; both enqueue on the
    current CUDA stream.  `workspace` (a uint8 CUDA tensor of at least
    fastvr_q4_workspace_bytes) may be shared by streams whose calls do not
    overlap on the GPU, as the layers of a model should: with long chunks it is
    as large as a bfloat16 cache.  By default one is allocated for the stream.
    A stream's first call that launches work cannot be captured into a CUDA
    graph (FASTVR_ERR_SEQUENCE); a captured call is replayed on the chunks of
    its capture."""

    def __init__(self, cfg: fastvr_attn_config_t,
                 kv_heads: Optional[int] = None, device=None, workspace=None):
        torch = _torch or _setup()
        self.cfg = cfg
        self.kv_heads = cfg.heads if kv_heads is None else kv_heads
        device = device or "cuda"
        self.nbytes = fastvr_q4_cache_bytes(cfg, self.kv_heads)
        need = fastvr_q4_workspace_bytes(cfg, self.kv_heads)
        if workspace is None:
            workspace = torch.empty(need, dtype=torch.uint8, device=device)
        elif not workspace.is_cuda or not workspace.is_contiguous():
            raise ValueError("workspace must be a contiguous CUDA tensor")
        self.workspace = workspace
        self.cache = torch.empty(self.nbytes, dtype=torch.uint8, device=device)
        self.plan = fastvr_q4_plan(cfg, self.kv_heads, self.cache.data_ptr(),
                                   self.nbytes, workspace.data_ptr(),
                                   workspace.numel() *
                                   workspace.element_size())
        self._state = _I64(0), _I32(0)
        self._state_refs = tuple(map(ctypes.byref, self._state))

    def __del__(self):
        plan = getattr(self, "plan", None)
        if plan:
            fastvr_plan_destroy(plan)
            self.plan = None

    def append(self, k, v) -> None:
        torch = _torch or _setup()
        c = self.cfg
        if k.dtype != torch.bfloat16 or v.dtype != torch.bfloat16:
            raise ValueError("k and v must be bfloat16")
        k_str, v_str = _head_strides(k, "k"), _head_strides(v, "v")
        B, L, H, d = k.shape
        if v.shape != k.shape:
            raise ValueError("k and v differ in shape")
        if (B, H, d) != (c.batch, self.kv_heads, c.head_dim) or \
                L % c.tokens_per_frame:
            raise ValueError(f"k has shape {tuple(k.shape)}")
        fastvr_q4_append(self.plan, k.data_ptr(), k_str, v.data_ptr(), v_str,
                         L // c.tokens_per_frame,
                         _stream_of(k, v, self.cache))

    def forward(self, q, first_chunk=None, out=None, lse=None,
                want_lse: bool = False):
        """Attention of the newest chunk's queries; first_chunk, int32 [B]:
        the first chunk that each batch entry sees."""
        torch = _torch or _setup()
        c = self.cfg
        if q.dtype != torch.bfloat16 or not q.is_contiguous() or q.dim() != 4:
            raise ValueError("q must be a contiguous bfloat16 CUDA tensor "
                             "[B, L, H, d]")
        B, L, H, d = q.shape
        frames = self.state()[1]
        if (B, H, d) != (c.batch, c.heads, c.head_dim) or \
                frames and L != frames * c.tokens_per_frame:
            raise ValueError(f"q has shape {tuple(q.shape)}")
        if first_chunk is not None and (
                first_chunk.dtype != torch.int32 or
                first_chunk.shape != (B,) or not first_chunk.is_contiguous()):
            raise ValueError("first_chunk must be a contiguous int32 CUDA "
                             "tensor [B]")
        if out is None:
            out = torch.empty_like(q)
        elif out.shape != q.shape or out.dtype != q.dtype or \
                out.device != q.device or not out.is_contiguous() or \
                out.data_ptr() == q.data_ptr():
            raise ValueError("out must be contiguous, like q and not q")
        if lse is None and want_lse:
            lse = torch.empty((B, H, L), dtype=torch.float32, device=q.device)
        elif lse is not None and (lse.shape != (B, H, L) or
                                  lse.dtype != torch.float32 or
                                  lse.device != q.device or
                                  not lse.is_contiguous()):
            raise ValueError("lse must be contiguous float32 [B, H, L], where "
                             "q is")
        fastvr_q4_attn_fwd(self.plan, q.data_ptr(), _ptr(first_chunk),
                           out.data_ptr(), _ptr(lse),
                           _stream_of(q, first_chunk, self.cache))
        return (out, lse) if lse is not None else out

    def read(self, chunk: Optional[int] = None):
        """(k, v) bfloat16 [B, f*N, kv_heads, d]: the values held for a chunk
        (default: the newest)."""
        torch = _torch or _setup()
        c = self.cfg
        chunks, frames = self.state()
        chunk = chunks - 1 if chunk is None else chunk
        if chunk != chunks - 1:
            frames = c.frames_per_chunk
        shape = (c.batch, frames * c.tokens_per_frame, self.kv_heads,
                 c.head_dim)
        k, v = (torch.empty(shape, dtype=torch.bfloat16,
                            device=self.cache.device) for _ in range(2))
        fastvr_q4_read(self.plan, chunk, k.data_ptr(), v.data_ptr(),
                       _stream_of(k))
        return k, v

    def reset(self) -> None:
        fastvr_plan_reset(self.plan)

    def launch_count(self) -> int:
        return fastvr_plan_launch_count(self.plan)

    def status(self) -> int:
        return fastvr_get_status(self.plan)

    def visible(self):
        return fastvr_plan_visible(self.plan)

    def state(self) -> Tuple[int, int]:
        _check(lib.fastvr_plan_get_state(self.plan, *self._state_refs),
               "fastvr_plan_get_state")
        return self._state[0].value, self._state[1].value

    def set_state(self, chunks: int, last_frames: int) -> None:
        fastvr_plan_set_state(self.plan, chunks, last_frames)


def config_from_workload(w) -> fastvr_attn_config_t:
    return make_config(w.batch, w.heads, w.head_dim, w.tokens_per_frame,
                       w.frames_per_chunk, w.window_chunks,
                       w.max_chunks, w.softmax_scale)
