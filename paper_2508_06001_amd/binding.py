"""ctypes binding of libknapattn.so: the same names as include/knapattn.h (and the benchmark hooks of
include/knapattn_bench.h).

Argument marshalling only.  Every step of the attention path runs in the HIP
kernels of the shared library; PyTorch supplies device memory and the stream.
There is no fallback: if the library has not been built the import fails.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import List, Optional, Sequence, Tuple

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libknapattn.so")

KNAP_OK = 0
KNAP_ERR_INVALID_ARG = -1
KNAP_ERR_WORKSPACE_TOO_SMALL = -2
KNAP_ERR_LAUNCH_FAILED = -3
KNAP_ERR_TOO_MANY_SEQS = -4
KNAP_ERR_CAPACITY = -5
KNAP_ERR_PARSE = -6
KNAP_ERR_SCRATCH_TOO_SMALL = -7
KNAP_NOALLOC_MAX_ROWS = 4 * 1024 * 1024
KNAP_MAX_SEQS = 2048
KNAP_ULYSSES_MAX_GPUS = 64
KNAP_ROPE_HALF = 0
KNAP_ROPE_INTERLEAVED = 1
KNAP_ROPE_MAX_AXES = 4
KNAP_ROPE_MAX_DIM = 1024
KNAP_ROPE_PLAIN = 0
KNAP_ROPE_LINEAR = 1
KNAP_ROPE_BASE = 2
KNAP_ROPE_PARTS = 3
KNAP_BF16 = 0
KNAP_F32 = 1
KNAP_LAYER_NORM_MAX_WIDTH = 16384

if not os.path.exists(LIB_PATH):
    raise ImportError(
        f"{LIB_PATH} is missing: build it first with `python paper_2508_06001_amd/build.py` "
        "(there is no CPU or PyTorch fallback for the attention path)")

# PyTorch ships its own HIP runtime (same SONAME as the system one).  It must be
# in the process before this library is loaded, so that both resolve to ONE
# runtime: streams and device pointers handed over by PyTorch are only valid in
# the runtime that created them.
import torch  # noqa: E402,F401

lib = C.CDLL(LIB_PATH)

_vp, _i, _f, _d, _i64, _sz = C.c_void_p, C.c_int, C.c_float, C.c_double, C.c_int64, C.c_size_t
_pd, _pi, _pi64, _pi32 = C.POINTER(C.c_double), C.POINTER(C.c_int), C.POINTER(C.c_int64), C.POINTER(C.c_int32)

_SIGNATURES = {
    "knap_varlen_attn_fwd": (_i, [_vp, _vp, _vp, _vp, _i, _i, _i, _f, _vp, _vp, _vp]),
    "knap_varlen_attn_bwd": (_i, [_vp, _vp, _vp, _vp, _i, _i, _i, _f, _vp, _vp, _vp, _vp, _vp, _vp, _i64, _vp, _sz, _vp]),
    "knap_varlen_attn_bwd_workspace_bytes": (_sz, [_i64, _i, _i, _i]),
    "knap_varlen_attn_bwd_noalloc": (_i, [_vp, _vp, _vp, _vp, _i, _i, _i, _f, _vp, _vp, _vp, _vp, _vp, _vp, _i64, _vp]),
    "knap_varlen_attn_causal_fwd": (_i, [_vp, _vp, _vp, _vp, _i, _i, _i, _f, _vp, _vp, _vp]),
    "knap_varlen_attn_causal_bwd": (_i, [_vp, _vp, _vp, _vp, _i, _i, _i, _f, _vp, _vp, _vp, _vp, _vp, _vp, _i64, _vp, _sz, _vp]),
    "knap_varlen_diff_attn_fwd": (_i, [_vp, _vp, _vp, _vp, _i, _i, _i, _f, _vp, _vp, _vp, _vp, _vp]),
    "knap_varlen_diff_attn_causal_fwd": (_i, [_vp, _vp, _vp, _vp, _i, _i, _i, _f, _vp, _vp, _vp, _vp, _vp]),
    "knap_varlen_diff_attn_bwd": (_i, [_vp, _vp, _vp, _vp, _i, _i, _i, _f] + [_vp] * 9 + [_i64, _vp, _sz, _vp]),
    "knap_varlen_diff_attn_causal_bwd": (_i, [_vp, _vp, _vp, _vp, _i, _i, _i, _f] + [_vp] * 9 + [_i64, _vp, _sz, _vp]),
    "knap_varlen_diff_attn_bwd_workspace_bytes": (_sz, [_i64, _i, _i, _i]),
    "knap_ulysses_pack_heads": (_i, [_vp, _i64, _i, _i, _i, _vp, _vp]),
    "knap_ulysses_unpack_heads": (_i, [_vp, _i64, _i, _i, _i, _vp, _vp]),
    "knap_ulysses_plan_workspace_bytes": (_sz, [_i, _i]),
    "knap_ulysses_plan": (_i, [_vp, _i, _i64, _i, _vp, _vp, _sz, _vp]),
    "knap_ulysses_gather_chunks": (_i, [_vp, _vp, _i64, _i, _i, _vp, _vp]),
    "knap_ulysses_scatter_chunks": (_i, [_vp, _vp, _i64, _i, _i, _vp, _vp]),
    "knap_ulysses_local_tokens": (_i, [_pi64, _i, _i, _pi64]),
    "knap_rope_fwd": (_i, [_vp, _vp, _i64, _i, _i, _i, _vp, _i, _i, _vp, _i, _vp, _vp, _i, _vp, _f, _vp, _vp, _vp]),
    "knap_rope_bwd": (_i, [_vp, _vp, _i64, _i, _i, _i, _vp, _i, _i, _vp, _i, _vp, _vp, _i, _vp, _f, _vp, _vp, _vp]),
    "knap_rope_frequencies": (_i, [_i, _d, _i, _d, _i64, _d, _d, _pd, _pd]),
    "knap_layer_norm_fwd": (_i, [_vp, _i, _i64, _i64, _i, _vp, _vp, _i, _f, _vp, _i, _i64, _vp, _vp, _vp]),
    "knap_layer_norm_bwd": (_i, [_vp, _i, _i64, _i64, _i, _vp, _i, _vp, _vp, _vp, _i, _i64, _vp, _i64, _vp, _vp, _vp, _sz, _vp]),
    "knap_layer_norm_bwd_workspace_bytes": (_sz, [_i64, _i]),
    "knap_strerror": (C.c_char_p, [_i]),
    "knap_last_hip_error": (_i, []),
    "knap_launch_workgroups": (_i, [_i]),
    "knap_fwd_queue_counters": (_vp, [C.POINTER(_i)]),
    "knap_bwd_profile_events": (None, [_vp, _vp]),
    "knap_seq_cost": (_d, [_i64, _d, _d]),
    "knap_flux_workload": (_d, [_i64, _i64, _d]),
    "knap_fit_cost_model": (_i, [_pd, _pd, _pd, _i, _pd, _pd, _pd]),
    "knap_parse_topology": (_i, [C.c_char_p, _pi, _i, _pi]),
    "knap_greedy_assign": (_i, [_pi64, _i, _pi, _i, _d, _d, _pi, _pd]),
    "knap_greedy_assign_weights": (_i, [_pd, _i, _pi, _i, _pi, _pd]),
    "knap_chunk_lengths": (_i, [_i64, _i, _pi64]),
    "knap_wir": (_d, [_pd, _pi, _i]),
    "knap_bag_cu_seqlens": (_i, [_pi64, _pi, _i, _i, _pi64, _i, _pi, _pi32]),
}
EXPORTS = tuple(_SIGNATURES)

for _name, (_res, _args) in _SIGNATURES.items():
    _fn = getattr(lib, _name)      # AttributeError here = the library does not export the symbol
    _fn.restype = _res
    _fn.argtypes = _args


class KnapError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        hip = int(lib.knap_last_hip_error()) if code == KNAP_ERR_LAUNCH_FAILED else 0
        extra = f", hipError_t {hip}" if hip else ""
        super().__init__(f"{where}: {knap_strerror(code)} (code {code}{extra})")


def knap_strerror(code: int) -> str:
    return lib.knap_strerror(int(code)).decode()


def _check(code: int, where: str) -> None:
    if code != KNAP_OK:
        raise KnapError(code, where)


def _ptr(t) -> int:
    """Device (or host) address of a tensor; None -> NULL."""
    return 0 if t is None else t.data_ptr()


# The current stream's handle without a Stream object around it, which costs more than the rest of a call's marshalling: 2.8 us
# against 0.2, of 7.7 us of host time for a forward and 11.4 for a backward, which is what bounds the smallest calls.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_current_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream_handle(stream) -> int:
    if stream is None:
        if _raw_stream is None or _current_device is None or not torch.cuda.is_initialized():
            return int(torch.cuda.current_stream().cuda_stream)
        return _raw_stream(_current_device())
    if isinstance(stream, int):
        return stream
    return int(stream.cuda_stream)


# --------------------------------------------------------------------------- attention

def knap_varlen_attn_fwd(q, k, v, cu_seqlens, n_seq: int, H: int, d: int, scale: float, out, lse,
                         stream=None, check: bool = True) -> int:
    """Enqueue the forward kernel.  q, k, v, out: bf16 (T, H, d) CUDA tensors; cu_seqlens: int32
    (n_seq + 1,) CUDA tensor; lse: fp32 (H, T).  Returns the library's status code."""
    rc = lib.knap_varlen_attn_fwd(_ptr(q), _ptr(k), _ptr(v), _ptr(cu_seqlens), n_seq, H, d, scale,
                                  _ptr(out), _ptr(lse), _stream_handle(stream))
    if check:
        _check(rc, "knap_varlen_attn_fwd")
    return rc


def knap_varlen_attn_bwd_workspace_bytes(total_tokens: int, n_seq: int, H: int, d: int) -> int:
    return int(lib.knap_varlen_attn_bwd_workspace_bytes(total_tokens, n_seq, H, d))


def knap_varlen_attn_bwd(q, k, v, cu_seqlens, n_seq: int, H: int, d: int, scale: float, out, lse, dout,
                         dq, dk, dv, total_tokens: int, workspace, workspace_bytes: Optional[int] = None,
                         stream=None, check: bool = True) -> int:
    """Enqueue the backward kernels.  `workspace` is a CUDA uint8 tensor of at least
    knap_varlen_attn_bwd_workspace_bytes(...) bytes."""
    if workspace_bytes is None:
        workspace_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    rc = lib.knap_varlen_attn_bwd(_ptr(q), _ptr(k), _ptr(v), _ptr(cu_seqlens), n_seq, H, d, scale,
                                  _ptr(out), _ptr(lse), _ptr(dout), _ptr(dq), _ptr(dk), _ptr(dv),
                                  total_tokens, _ptr(workspace), workspace_bytes, _stream_handle(stream))
    if check:
        _check(rc, "knap_varlen_attn_bwd")
    return rc


def knap_varlen_attn_bwd_noalloc(q, k, v, cu_seqlens, n_seq: int, H: int, d: int, scale: float, out, lse, dout,
                                 dq, dk, dv, total_tokens: int, stream=None, check: bool = True) -> int:
    """knap_varlen_attn_bwd without a workspace argument: the scratch is an array in the library's device
    image (total_tokens * H <= KNAP_NOALLOC_MAX_ROWS)."""
    rc = lib.knap_varlen_attn_bwd_noalloc(_ptr(q), _ptr(k), _ptr(v), _ptr(cu_seqlens), n_seq, H, d, scale,
                                          _ptr(out), _ptr(lse), _ptr(dout), _ptr(dq), _ptr(dk), _ptr(dv),
                                          total_tokens, _stream_handle(stream))
    if check:
        _check(rc, "knap_varlen_attn_bwd_noalloc")
    return rc


def knap_varlen_attn_causal_fwd(q, k, v, cu_seqlens, n_seq: int, H: int, d: int, scale: float, out, lse,
                                stream=None, check: bool = True) -> int:
    """knap_varlen_attn_fwd with the causal mask inside every sequence."""
    rc = lib.knap_varlen_attn_causal_fwd(_ptr(q), _ptr(k), _ptr(v), _ptr(cu_seqlens), n_seq, H, d, scale,
                                         _ptr(out), _ptr(lse), _stream_handle(stream))
    if check:
        _check(rc, "knap_varlen_attn_causal_fwd")
    return rc


def knap_varlen_attn_causal_bwd(q, k, v, cu_seqlens, n_seq: int, H: int, d: int, scale: float, out, lse, dout,
                                dq, dk, dv, total_tokens: int, workspace, workspace_bytes: Optional[int] = None,
                                stream=None, check: bool = True) -> int:
    """knap_varlen_attn_bwd with the causal mask inside every sequence."""
    if workspace_bytes is None:
        workspace_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    rc = lib.knap_varlen_attn_causal_bwd(_ptr(q), _ptr(k), _ptr(v), _ptr(cu_seqlens), n_seq, H, d, scale,
                                         _ptr(out), _ptr(lse), _ptr(dout), _ptr(dq), _ptr(dk), _ptr(dv),
                                         total_tokens, _ptr(workspace), workspace_bytes, _stream_handle(stream))
    if check:
        _check(rc, "knap_varlen_attn_causal_bwd")
    return rc


def knap_last_hip_error() -> int:
    return int(lib.knap_last_hip_error())


def knap_bwd_profile_events(start: Optional[int], stop: Optional[int]) -> None:
    """Raw hipEvent_t handles (ints) recorded around the main backward kernel; None switches it off."""
    lib.knap_bwd_profile_events(start or 0, stop or 0)


def knap_launch_workgroups(which: int) -> int:
    return int(lib.knap_launch_workgroups(which))


# --------------------------------------------------------------------------- Ulysses layout switch (local part)

def knap_ulysses_pack_heads(x, local_tokens: int, H: int, d: int, g: int, y, stream=None, check: bool = True) -> int:
    """x (T_r, H, d) -> y (g, T_r, H/g, d); CUDA tensors of a two-byte type."""
    rc = lib.knap_ulysses_pack_heads(_ptr(x), local_tokens, H, d, g, _ptr(y), _stream_handle(stream))
    if check:
        _check(rc, "knap_ulysses_pack_heads")
    return rc


def knap_ulysses_unpack_heads(y, local_tokens: int, H: int, d: int, g: int, x, stream=None, check: bool = True) -> int:
    rc = lib.knap_ulysses_unpack_heads(_ptr(y), local_tokens, H, d, g, _ptr(x), _stream_handle(stream))
    if check:
        _check(rc, "knap_ulysses_unpack_heads")
    return rc


def knap_ulysses_plan_workspace_bytes(n_seq: int, g: int) -> int:
    return int(lib.knap_ulysses_plan_workspace_bytes(n_seq, g))


def knap_ulysses_plan(cu_seqlens, n_seq: int, total_tokens: int, g: int, row_map, workspace,
                      workspace_bytes: Optional[int] = None, stream=None, check: bool = True) -> int:
    """Fills row_map (int32 CUDA tensor of total_tokens entries) for a g-GPU bag."""
    if workspace_bytes is None:
        workspace_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    rc = lib.knap_ulysses_plan(_ptr(cu_seqlens), n_seq, total_tokens, g, _ptr(row_map), _ptr(workspace),
                               workspace_bytes, _stream_handle(stream))
    if check:
        _check(rc, "knap_ulysses_plan")
    return rc


def knap_ulysses_gather_chunks(recv, row_map, total_tokens: int, heads_local: int, d: int, z,
                               stream=None, check: bool = True) -> int:
    rc = lib.knap_ulysses_gather_chunks(_ptr(recv), _ptr(row_map), total_tokens, heads_local, d, _ptr(z),
                                        _stream_handle(stream))
    if check:
        _check(rc, "knap_ulysses_gather_chunks")
    return rc


def knap_ulysses_scatter_chunks(z, row_map, total_tokens: int, heads_local: int, d: int, send,
                                stream=None, check: bool = True) -> int:
    rc = lib.knap_ulysses_scatter_chunks(_ptr(z), _ptr(row_map), total_tokens, heads_local, d, _ptr(send),
                                         _stream_handle(stream))
    if check:
        _check(rc, "knap_ulysses_scatter_chunks")
    return rc


def knap_ulysses_local_tokens(seq_lens, g: int):
    """T_r for r = 0..g-1: tokens every GPU of a g-GPU bag holds after the second pass."""
    n = len(seq_lens)
    arr = (C.c_int64 * max(n, 1))(*[int(x) for x in seq_lens])
    out = (C.c_int64 * g)()
    _check(lib.knap_ulysses_local_tokens(arr, n, g, out), "knap_ulysses_local_tokens")
    return [int(v) for v in out]


def _refuse(where: str, what: str) -> None:
    err = KnapError(KNAP_ERR_INVALID_ARG, where)
    err.args = (f"{err.args[0]}: {what}",)
    raise err


def _here(where: str, *tensors) -> None:
    """Tensors that are not on the current device, whose stream the call would go to, are refused."""
    dev = _current_device() if _current_device is not None else torch.cuda.current_device()
    for t in tensors:
        if t is not None and t.get_device() != dev:
            _refuse(where, f"a tensor on device {t.get_device()} while device {dev} is current")


_KNAP_TYPES = {torch.bfloat16: KNAP_BF16, torch.float32: KNAP_F32}


# --------------------------------------------------------------------------- differential attention

def _diff_tensors(where: str, cu_seqlens, n_seq, H, d, rows, f32) -> int:
    """How many rows the tensors have, q first among them, checked; f32: vectors and the least that each holds."""
    if cu_seqlens is not None and (cu_seqlens.dtype is not torch.int32 or cu_seqlens.numel() <= n_seq or not cu_seqlens.is_contiguous()):
        _refuse(where, "cu_seqlens is a contiguous int32 tensor of n_seq + 1 entries")
    shape = () if rows[0] is None else rows[0].shape
    T, bf16 = shape[0] if shape else -1, torch.bfloat16
    shapes = ((T, H, d), (T, H * d))
    if shape not in shapes:
        _refuse(where, "q is a (T, H, d) tensor")
    for t in rows:
        if t is not None and (t.dtype is not bf16 or not t.is_contiguous() or (t.shape != shape and t.shape not in shapes)):
            _refuse(where, "q, k, v, the outputs and their gradients are contiguous bf16 (T, H, d) tensors")
    for t, n in f32:
        if t is not None and (t.dtype is not torch.float32 or t.numel() < n or not t.is_contiguous()):
            _refuse(where, "lambda and dlambda are contiguous fp32 (H,) tensors, lse is an fp32 (2, H, T) one")
    return T


def _diff_fwd(fn, where: str, q, k, v, cu_seqlens, n_seq, H, d, scale, lam, out, out2, lse, stream, check) -> int:
    _here(where, q, k, v, cu_seqlens, lam, out, out2, lse)
    T = _diff_tensors(where, cu_seqlens, n_seq, H, d, (q, k, v, out, out2), ((lam, H), (lse, 0)))
    # the kernel writes 2 H log-sums for each token of the bag, whose number the host cannot see: room for all rows, or the shape that a
    # padded bag's has
    if lse is not None and lse.numel() < 2 * H * T and (lse.dim() != 3 or lse.shape[0] != 2 or lse.shape[1] != H):
        _refuse(where, "lse is an fp32 (2, H, T) tensor")
    rc = fn(_ptr(q), _ptr(k), _ptr(v), _ptr(cu_seqlens), n_seq, H, d, scale, _ptr(lam), _ptr(out), _ptr(out2), _ptr(lse), _stream_handle(stream))
    if check:
        _check(rc, where)
    return rc


def knap_varlen_diff_attn_fwd(q, k, v, cu_seqlens, n_seq: int, H: int, d: int, scale: float, lam, out, out2, lse, stream=None,
                              check: bool = True) -> int:
    """Enqueue the forward of differential attention.  q, k, v, out, out2 (or None): bf16 (T, H, d); lam: fp32 (H,); lse: fp32 (2, H, T), where
    the tensors may have more rows than T = cu_seqlens[n_seq] (a padded bag), or any contiguous fp32 tensor of 2 H values a row."""
    return _diff_fwd(lib.knap_varlen_diff_attn_fwd, "knap_varlen_diff_attn_fwd", q, k, v, cu_seqlens, n_seq, H, d, scale, lam, out, out2, lse,
                     stream, check)


def knap_varlen_diff_attn_causal_fwd(q, k, v, cu_seqlens, n_seq: int, H: int, d: int, scale: float, lam, out, out2, lse, stream=None,
                                     check: bool = True) -> int:
    """knap_varlen_diff_attn_fwd with the causal mask inside every sequence."""
    return _diff_fwd(lib.knap_varlen_diff_attn_causal_fwd, "knap_varlen_diff_attn_causal_fwd", q, k, v, cu_seqlens, n_seq, H, d, scale, lam, out,
                     out2, lse, stream, check)


def knap_varlen_diff_attn_bwd_workspace_bytes(total_tokens: int, n_seq: int, H: int, d: int) -> int:
    return int(lib.knap_varlen_diff_attn_bwd_workspace_bytes(total_tokens, n_seq, H, d))


def _diff_bwd(fn, where: str, q, k, v, cu_seqlens, n_seq, H, d, scale, lam, out, out2, lse, dout, dq, dk, dv, dlam, total_tokens, workspace,
              workspace_bytes, stream, check) -> int:
    _here(where, q, k, v, cu_seqlens, lam, out, out2, lse, dout, dq, dk, dv, dlam, workspace)
    T = _diff_tensors(where, cu_seqlens, n_seq, H, d, (q, k, v, out, out2, dout, dq, dk, dv), ((lam, H), (dlam, H), (lse, 2 * H * total_tokens)))
    if total_tokens > T:
        _refuse(where, "total_tokens is more than the tensors hold")
    if workspace_bytes is None:
        workspace_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    rc = fn(_ptr(q), _ptr(k), _ptr(v), _ptr(cu_seqlens), n_seq, H, d, scale, _ptr(lam), _ptr(out), _ptr(out2), _ptr(lse), _ptr(dout), _ptr(dq),
            _ptr(dk), _ptr(dv), _ptr(dlam), total_tokens, _ptr(workspace), workspace_bytes, _stream_handle(stream))
    if check:
        _check(rc, where)
    return rc


def knap_varlen_diff_attn_bwd(q, k, v, cu_seqlens, n_seq: int, H: int, d: int, scale: float, lam, out, out2, lse, dout, dq, dk, dv, dlam,
                              total_tokens: int, workspace, workspace_bytes: Optional[int] = None, stream=None, check: bool = True) -> int:
    """Enqueue the backward of differential attention; dlam: fp32 (H,)."""
    return _diff_bwd(lib.knap_varlen_diff_attn_bwd, "knap_varlen_diff_attn_bwd", q, k, v, cu_seqlens, n_seq, H, d, scale, lam, out, out2, lse,
                     dout, dq, dk, dv, dlam, total_tokens, workspace, workspace_bytes, stream, check)


def knap_varlen_diff_attn_causal_bwd(q, k, v, cu_seqlens, n_seq: int, H: int, d: int, scale: float, lam, out, out2, lse, dout, dq, dk, dv, dlam,
                                     total_tokens: int, workspace, workspace_bytes: Optional[int] = None, stream=None,
                                     check: bool = True) -> int:
    """knap_varlen_diff_attn_bwd with the causal mask inside every sequence."""
    return _diff_bwd(lib.knap_varlen_diff_attn_causal_bwd, "knap_varlen_diff_attn_causal_bwd", q, k, v, cu_seqlens, n_seq, H, d, scale, lam, out,
                     out2, lse, dout, dq, dk, dv, dlam, total_tokens, workspace, workspace_bytes, stream, check)


# --------------------------------------------------------------------------- rotary positions, layer norm

def _rope(fn, where: str, q, k, rot, layout, freq, factor, q_out, k_out, positions, axis_pairs, cu_seqlens, stream, check) -> int:
    # the host's time bounds the smallest calls: each property is asked for once, strides only where something is not contiguous
    _here(where, q, k, q_out, k_out, freq, positions, cu_seqlens)
    bf16 = torch.bfloat16
    q_shape, k_shape = q.shape, None if k is None else k.shape
    if len(q_shape) != 3 or q.dtype is not bf16 or q_out.dtype is not bf16 or q_out.shape != q_shape:
        _refuse(where, "q, k and their outputs are bf16 (tokens, heads, d) tensors of the same tokens and d")
    T, H, d = q_shape
    plain, H_k, k_at, k_out_at = q.is_contiguous() and q_out.is_contiguous(), 0, 0, 0
    if k is not None:
        if (len(k_shape) != 3 or k.dtype is not bf16 or k_out is None or k_out.dtype is not bf16 or k_out.shape != k_shape or k_shape[0] != T
                or k_shape[2] != d):
            _refuse(where, "q, k and their outputs are bf16 (tokens, heads, d) tensors of the same tokens and d")
        plain = plain and k.is_contiguous() and k_out.is_contiguous()
        H_k, k_at, k_out_at = k_shape[1], k.data_ptr(), k_out.data_ptr()
    strides = None
    if not plain:
        qs, qos = q.stride(), q_out.stride()
        ks, kos = (k.stride(), k_out.stride()) if k is not None else ((0, 0, 1), (0, 0, 1))
        if d > 1 and (qs[2] != 1 or qos[2] != 1 or ks[2] != 1 or kos[2] != 1):
            _refuse(where, "the columns of a head are contiguous")
        strides = (C.c_int64 * 8)(qs[0], qs[1], ks[0], ks[1], qos[0], qos[1], kos[0], kos[1])
    if freq.dtype is not torch.float64 or freq.numel() != rot // 2 or not freq.is_contiguous():
        _refuse(where, "freq is a contiguous float64 tensor of rot / 2 entries")
    n_axes, pairs, n_seq, pos_at, cu_at = 0, None, 0, 0, 0
    if positions is not None:
        n_axes = 1 if positions.dim() == 1 else positions.shape[-1] if positions.dim() else 0
        # (none: no address, which the library takes for no positions given)
        if n_axes < 1 or positions.dtype is not torch.int32 or positions.numel() != T * n_axes or positions.shape[0] != T or not positions.is_contiguous():
            _refuse(where, "positions is a contiguous int32 (tokens,) or (tokens, axes) tensor")
        pos_at = positions.data_ptr()
        if axis_pairs:
            if len(axis_pairs) != n_axes:
                _refuse(where, "axis_pairs has an entry for each axis")
            pairs = (C.c_int * n_axes)(*axis_pairs)
    elif cu_seqlens is not None:
        if cu_seqlens.dtype is not torch.int32 or not cu_seqlens.is_contiguous():
            _refuse(where, "cu_seqlens is a contiguous int32 tensor")
        n_seq, cu_at = cu_seqlens.numel() - 1, cu_seqlens.data_ptr()
    else:
        _refuse(where, "positions or cu_seqlens")
    rc = fn(q.data_ptr(), k_at, T, H, H_k, d, strides, rot, layout, pos_at, n_axes, pairs, cu_at, n_seq, freq.data_ptr(), factor,
            q_out.data_ptr(), k_out_at, _stream_handle(stream))
    if check:
        _check(rc, where)
    return rc


def knap_rope_fwd(q, k, rot: int, layout: int, freq, factor: float, q_out, k_out, positions=None, axis_pairs=None, cu_seqlens=None,
                  stream=None, check: bool = True) -> int:
    """Rotary positions of q (T, H, d) and k (T, H_k, d) or None; any strides of tokens and heads.  positions: int32 (T,) or
    (T, axes), else the position in the own sequence of cu_seqlens.  freq: float64 CUDA tensor of rot / 2 entries."""
    return _rope(lib.knap_rope_fwd, "knap_rope_fwd", q, k, rot, layout, freq, factor, q_out, k_out, positions, axis_pairs, cu_seqlens,
                 stream, check)


def knap_rope_bwd(dq_out, dk_out, rot: int, layout: int, freq, factor: float, dq, dk, positions=None, axis_pairs=None, cu_seqlens=None,
                  stream=None, check: bool = True) -> int:
    """Gradients back through knap_rope_fwd: the same arguments, turned the other way."""
    return _rope(lib.knap_rope_bwd, "knap_rope_bwd", dq_out, dk_out, rot, layout, freq, factor, dq, dk, positions, axis_pairs, cu_seqlens,
                 stream, check)


def knap_rope_frequencies(rot: int, base: float = 10000.0, kind: int = KNAP_ROPE_PLAIN, scale: float = 1.0, trained_len: int = 1,
                          low: float = 1.0, high: float = 32.0) -> Tuple[List[float], float]:
    """Frequencies of rot / 2 pairs (radians per position) and the factor that goes with them."""
    freq, factor = (C.c_double * max(1, rot // 2))(), C.c_double()
    _check(lib.knap_rope_frequencies(rot, base, kind, scale, trained_len, low, high, freq, C.byref(factor)), "knap_rope_frequencies")
    return list(freq), factor.value


def _rows(where: str, name: str, t, shape, dtype=None) -> int:
    """The row stride of a (rows, width) tensor with contiguous rows, checked."""
    if t.dtype not in _KNAP_TYPES or (dtype is not None and t.dtype is not dtype):
        _refuse(where, f"the type of {name}")
    if len(shape) != 2 or t.shape != shape:
        _refuse(where, f"{name} is a (rows, width) tensor")
    if t.is_contiguous():
        return shape[1]
    if shape[1] > 1 and t.stride(1) != 1:
        _refuse(where, f"the rows of {name} are contiguous")
    return t.stride(0)


def _vector(where: str, name: str, t, n: int, dtype) -> int:
    """The address of a vector of n values, checked."""
    if t.dtype is not dtype or t.numel() != n or not t.is_contiguous():
        _refuse(where, f"{name} is a contiguous vector of {n} values of its type")
    return t.data_ptr()


def knap_layer_norm_fwd(x, weight, bias, eps: float, y, mean=None, rstd=None, stream=None, check: bool = True) -> int:
    """y = (x - mean) rstd weight + bias of every row of x (rows, width); weight and bias (of one type) may be None."""
    where = "knap_layer_norm_fwd"
    _here(where, x, weight, bias, y, mean, rstd)
    shape, types, f32 = x.shape, _KNAP_TYPES, torch.float32
    xs, ys = _rows(where, "x", x, shape), _rows(where, "y", y, shape)
    rows, width = shape
    w_type = f32 if weight is None and bias is None else (bias if weight is None else weight).dtype
    if w_type not in types:
        _refuse(where, "the type of weight and bias")
    w_at = 0 if weight is None else _vector(where, "weight", weight, width, w_type)
    b_at = 0 if bias is None else _vector(where, "bias", bias, width, w_type)
    mean_at = 0 if mean is None else _vector(where, "mean", mean, rows, f32)
    rstd_at = 0 if rstd is None else _vector(where, "rstd", rstd, rows, f32)
    rc = lib.knap_layer_norm_fwd(x.data_ptr(), types[x.dtype], xs, rows, width, w_at, b_at, types[w_type], eps, y.data_ptr(), types[y.dtype], ys,
                                 mean_at, rstd_at, _stream_handle(stream))
    if check:
        _check(rc, where)
    return rc


def knap_layer_norm_bwd_workspace_bytes(rows: int, width: int) -> int:
    return int(lib.knap_layer_norm_bwd_workspace_bytes(rows, width))


def knap_layer_norm_bwd(x, weight, mean, rstd, dy, dx, dweight, dbias, workspace, workspace_bytes: Optional[int] = None, stream=None,
                        check: bool = True) -> int:
    """dx (of x's type), dweight and dbias (fp32, or None) of knap_layer_norm_fwd, whose mean and rstd it takes."""
    where = "knap_layer_norm_bwd"
    _here(where, x, weight, mean, rstd, dy, dx, dweight, dbias, workspace)
    shape, types, f32 = x.shape, _KNAP_TYPES, torch.float32
    xs, dys, dxs = _rows(where, "x", x, shape), _rows(where, "dy", dy, shape), _rows(where, "dx", dx, shape, x.dtype)
    rows, width = shape
    w_type = f32 if weight is None else weight.dtype
    if w_type not in types:
        _refuse(where, "the type of weight")
    w_at = 0 if weight is None else _vector(where, "weight", weight, width, w_type)
    dw_at = 0 if dweight is None else _vector(where, "dweight", dweight, width, f32)
    db_at = 0 if dbias is None else _vector(where, "dbias", dbias, width, f32)
    mean_at = 0 if mean is None else _vector(where, "mean", mean, rows, f32)
    rstd_at = 0 if rstd is None else _vector(where, "rstd", rstd, rows, f32)
    if workspace_bytes is None:
        workspace_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    rc = lib.knap_layer_norm_bwd(x.data_ptr(), types[x.dtype], xs, rows, width, w_at, types[w_type], mean_at, rstd_at, dy.data_ptr(), types[dy.dtype],
                                 dys, dx.data_ptr(), dxs, dw_at, db_at, 0 if workspace is None else workspace.data_ptr(), workspace_bytes,
                                 _stream_handle(stream))
    if check:
        _check(rc, where)
    return rc


# --------------------------------------------------------------------------- host model / balancer

def knap_seq_cost(L: int, a: float, b: float) -> float:
    return float(lib.knap_seq_cost(L, a, b))


def knap_flux_workload(l: int, d_model: int, gamma: float) -> float:
    return float(lib.knap_flux_workload(l, d_model, gamma))


def _darr(xs: Sequence[float]):
    return (C.c_double * len(xs))(*[float(x) for x in xs])


def _iarr(xs: Sequence[int]):
    return (C.c_int * len(xs))(*[int(x) for x in xs])


def _i64arr(xs: Sequence[int]):
    return (C.c_int64 * len(xs))(*[int(x) for x in xs])


def knap_fit_cost_model(sum_l2: Sequence[float], sum_l: Sequence[float], t: Sequence[float]) -> Tuple[float, float, float]:
    a, b, r = C.c_double(), C.c_double(), C.c_double()
    _check(lib.knap_fit_cost_model(_darr(sum_l2), _darr(sum_l), _darr(t), len(t), C.byref(a), C.byref(b), C.byref(r)),
           "knap_fit_cost_model")
    return a.value, b.value, r.value


def knap_parse_topology(spec: str, cap: int = 4096) -> List[int]:
    bags = (C.c_int * cap)()
    n = C.c_int()
    _check(lib.knap_parse_topology(spec.encode(), bags, cap, C.byref(n)), "knap_parse_topology")
    return list(bags[: n.value])


def knap_greedy_assign(seq_len: Sequence[int], bag_gpus: Sequence[int], a: float, b: float) -> Tuple[List[int], List[float]]:
    bag_of = (C.c_int * max(1, len(seq_len)))()
    load = (C.c_double * len(bag_gpus))()
    _check(lib.knap_greedy_assign(_i64arr(seq_len), len(seq_len), _iarr(bag_gpus), len(bag_gpus), a, b, bag_of, load),
           "knap_greedy_assign")
    return list(bag_of[: len(seq_len)]), list(load)


def knap_greedy_assign_weights(weight: Sequence[float], bag_gpus: Sequence[int]) -> Tuple[List[int], List[float]]:
    bag_of = (C.c_int * max(1, len(weight)))()
    load = (C.c_double * len(bag_gpus))()
    _check(lib.knap_greedy_assign_weights(_darr(weight), len(weight), _iarr(bag_gpus), len(bag_gpus), bag_of, load),
           "knap_greedy_assign_weights")
    return list(bag_of[: len(weight)]), list(load)


def knap_chunk_lengths(L: int, g: int) -> List[int]:
    out = (C.c_int64 * max(1, g))()
    _check(lib.knap_chunk_lengths(L, g, out), "knap_chunk_lengths")
    return list(out[:g])


def knap_wir(bag_load: Sequence[float], bag_gpus: Sequence[int]) -> float:
    return float(lib.knap_wir(_darr(bag_load), _iarr(bag_gpus), len(bag_gpus)))


def knap_bag_cu_seqlens(seq_len: Sequence[int], bag_of_seq: Sequence[int], bag: int) -> Tuple[List[int], List[int]]:
    n = len(seq_len)
    out_len = (C.c_int64 * max(1, n))()
    cu = (C.c_int32 * (n + 1))()
    cnt = C.c_int()
    _check(lib.knap_bag_cu_seqlens(_i64arr(seq_len), _iarr(bag_of_seq), n, bag, out_len, n, C.byref(cnt), cu),
           "knap_bag_cu_seqlens")
    return list(out_len[: cnt.value]), list(cu[: cnt.value + 1])
