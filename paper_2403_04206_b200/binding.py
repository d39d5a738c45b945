"""ctypes binding of libgrawa.so: argument marshalling only.

Each function has the name of the C entry point it calls (see ``include/grawa.h`` for the
meaning of every argument).  Device buffers are passed as torch CUDA tensors (float32,
contiguous, 1-D) or as raw integer device addresses; torch is used for device memory and
streams only.  Every step of the update runs in the library's CUDA kernels.
"""
from __future__ import annotations

import ctypes
from typing import Optional, Sequence

import numpy as np

from . import build as _build

GRAWA_MAX_WORKERS = 64
_VARIANTS = {"grawa": 0, "mgrawa": 1, "lgrawa": 2}


class GrawaError(RuntimeError):
    """A libgrawa entry point returned a negative status."""

    def __init__(self, status: int, where: str):
        self.status = status
        text = library().grawa_status_string(status).decode()
        detail = library().grawa_last_cuda_error().decode() if status == -2 else ""
        super().__init__(f"{where}: {text} ({status})" + (f": {detail}" if detail else ""))


class _Options(ctypes.Structure):
    _fields_ = [("weights_out", ctypes.c_void_p), ("scores_out", ctypes.c_void_p), ("sumsq_out", ctypes.c_void_p),
                ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t), ("status_word", ctypes.c_void_p)]


_lib = None


def library() -> ctypes.CDLL:
    """Loads (building first when missing or stale) libgrawa.so.  Raises if that is impossible."""
    global _lib
    if _lib is not None:
        return _lib
    import os
    path = _build.build(debug_bounds=os.environ.get("GRAWA_DEBUG_BOUNDS", "0") == "1",
                        trace=os.environ.get("GRAWA_TRACE", "0") == "1")
    lib = ctypes.CDLL(path)
    vp, i64, ci, cf = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_float
    step_args = [vp, vp, i64, ci, cf, vp, ci, vp, vp, vp]
    for name in ("grawa_mgrawa_step", "grawa_grawa_step", "grawa_lgrawa_step"):
        getattr(lib, name).argtypes = step_args
        getattr(lib, name).restype = ci
    lib.grawa_step_typed.argtypes = [ci, ci, vp, vp, i64, ci, cf, vp, ci, vp, vp, vp]
    lib.grawa_step_typed.restype = ci
    lib.grawa_step_host.argtypes = [ci, vp, vp, i64, ci, cf, vp, ci, vp, vp]
    lib.grawa_step_host.restype = ci
    lib.grawa_prox_step.argtypes = [vp, vp, i64, ci, cf, vp]
    lib.grawa_prox_step.restype = ci
    lib.grawa_workspace_bytes.argtypes = [i64, ci, vp, ci]
    lib.grawa_workspace_bytes.restype = ctypes.c_size_t
    lib.grawa_last_step_status.argtypes = [vp]
    lib.grawa_last_step_status.restype = ci
    lib.grawa_status_string.argtypes = [ci]
    lib.grawa_status_string.restype = ctypes.c_char_p
    lib.grawa_last_cuda_error.argtypes = []
    lib.grawa_last_cuda_error.restype = ctypes.c_char_p
    lib.grawa_version.restype = ci
    lib.grawa_set_option.argtypes = [ctypes.c_char_p, i64]
    lib.grawa_set_option.restype = ci
    lib.grawa_get_option.argtypes = [ctypes.c_char_p]
    lib.grawa_get_option.restype = i64
    lib.grawa_launch_count.restype = i64
    lib.grawa_clear_plans.restype = None
    lib.grawa_layer_norms.argtypes = [vp, i64, vp, ci, vp, vp]
    lib.grawa_layer_norms.restype = ci
    lib.grawa_norm_ema.argtypes = [vp, vp, ci, ctypes.c_double, i64, vp, vp]
    lib.grawa_norm_ema.restype = ci
    lib.grawa_step_from_layer_norms.argtypes = [ci, vp, vp, i64, ci, cf, vp, ci, vp, vp, vp]
    lib.grawa_step_from_layer_norms.restype = ci
    lib.grawa_layer_sumsq.argtypes = [vp, i64, ci, vp, ci, vp, vp]
    lib.grawa_layer_sumsq.restype = ci
    lib.grawa_step_from_layer_sums.argtypes = [ci, vp, vp, ci, i64, ci, cf, vp, ci, vp, vp, vp]
    lib.grawa_step_from_layer_sums.restype = ci
    lib.grawa_prox_step_typed.argtypes = [ci, vp, vp, i64, ci, cf, vp]
    lib.grawa_prox_step_typed.restype = ci
    lib.grawa_layer_norms_typed.argtypes = [ci, vp, i64, vp, ci, vp, vp]
    lib.grawa_layer_norms_typed.restype = ci
    lib.grawa_layer_sumsq_typed.argtypes = [ci, vp, i64, ci, vp, ci, vp, vp]
    lib.grawa_layer_sumsq_typed.restype = ci
    lib.grawa_step_from_layer_norms_typed.argtypes = [ci, ci, vp, vp, i64, ci, cf, vp, ci, vp, vp, vp]
    lib.grawa_step_from_layer_norms_typed.restype = ci
    lib.grawa_step_from_layer_sums_typed.argtypes = [ci, ci, vp, vp, ci, i64, ci, cf, vp, ci, vp, vp, vp]
    lib.grawa_step_from_layer_sums_typed.restype = ci
    lib.grawa_step_host_typed.argtypes = [ci, ci, vp, vp, i64, ci, cf, vp, ci, vp, vp]
    lib.grawa_step_host_typed.restype = ci
    lib.grawa_sumsq_static.argtypes = [vp, i64, ci, vp, vp]
    lib.grawa_sumsq_static.restype = ci
    lib.grawa_debug_bounds_violations.argtypes = [ci]
    lib.grawa_debug_bounds_violations.restype = i64
    lib.grawa_trace_read.argtypes = [vp, ci]
    lib.grawa_trace_read.restype = ci
    lib.grawa_selftest_bounded_wait.argtypes = [i64, vp]
    lib.grawa_selftest_bounded_wait.restype = ci
    lib.grawa_collect_kernel_times.argtypes = [vp, vp, vp, vp]
    lib.grawa_collect_kernel_times.restype = ci
    u64 = ctypes.c_uint64
    lib.grawa_dropout_forward.argtypes = [ci, vp, vp, vp, i64, ci, cf, u64, u64, vp, vp]
    lib.grawa_dropout_forward.restype = ci
    lib.grawa_dropout_backward.argtypes = [ci, vp, vp, i64, ci, cf, u64, u64, vp, vp]
    lib.grawa_dropout_backward.restype = ci
    lib.grawa_layernorm_forward.argtypes = [ci] + [vp] * 6 + [i64] * 4 + [ci, cf, vp]
    lib.grawa_layernorm_forward.restype = ci
    lib.grawa_layernorm_backward.argtypes = [ci] + [vp] * 8 + [i64] * 4 + [ci, ci, vp, ctypes.c_size_t, vp]
    lib.grawa_layernorm_backward.restype = ci
    lib.grawa_layernorm_backward_workspace_bytes.argtypes = [i64, i64, ci, ci]
    lib.grawa_layernorm_backward_workspace_bytes.restype = ctypes.c_size_t
    sz = ctypes.c_size_t
    lib.grawa_gated_ffn_forward.argtypes = [ci, ci] + [vp] * 6 + [i64] * 3 + [ci, vp, sz, vp]
    lib.grawa_gated_ffn_forward.restype = ci
    lib.grawa_gated_ffn_backward.argtypes = [ci, ci] + [vp] * 9 + [i64] * 3 + [ci, ci, vp, sz, vp]
    lib.grawa_gated_ffn_backward.restype = ci
    lib.grawa_gated_ffn_workspace_bytes.argtypes = [i64] * 3 + [ci] * 3
    lib.grawa_gated_ffn_workspace_bytes.restype = sz
    lib.grawa_gated_ffn_status.argtypes = [vp]
    lib.grawa_gated_ffn_status.restype = ci
    lib.grawa_selftest_gated_ffn_wait.argtypes = [vp]
    lib.grawa_selftest_gated_ffn_wait.restype = ci
    lib.grawa_head_rotary_forward.argtypes = [ci, ci] + [vp] * 8 + [i64] * 10 + [ci, cf, vp]
    lib.grawa_head_rotary_forward.restype = ci
    lib.grawa_head_rotary_backward.argtypes = [ci, ci] + [vp] * 12 + [i64] * 10 + [ci, cf, ci, vp, sz, vp]
    lib.grawa_head_rotary_backward.restype = ci
    lib.grawa_head_rotary_backward_workspace_bytes.argtypes = [i64, ci]
    lib.grawa_head_rotary_backward_workspace_bytes.restype = sz
    lib.grawa_window_attention_forward.argtypes = [ci] + [vp] * 6 + [i64] * 13 + [ci, cf, vp]
    lib.grawa_window_attention_forward.restype = ci
    lib.grawa_window_attention_backward.argtypes = [ci] + [vp] * 10 + [i64] * 13 + [ci, cf, vp, sz, vp]
    lib.grawa_window_attention_backward.restype = ci
    lib.grawa_window_attention_backward_workspace_bytes.argtypes = [i64] * 5 + [ci]
    lib.grawa_window_attention_backward_workspace_bytes.restype = sz
    lib.grawa_window_attention_status.argtypes = [vp]
    lib.grawa_window_attention_status.restype = ci
    lib.grawa_selftest_window_attention_wait.argtypes = [vp]
    lib.grawa_selftest_window_attention_wait.restype = ci
    _lib = lib
    return lib


# ------------------------------------------------------------------ marshalling helpers

def _addr(buf) -> int:
    """Device (or host) address of a torch tensor / numpy array / integer / None."""
    if buf is None:
        return 0
    if isinstance(buf, int):
        return buf
    if isinstance(buf, np.ndarray):
        if not buf.flags["C_CONTIGUOUS"]:
            raise ValueError("numpy buffers must be C-contiguous")
        return buf.ctypes.data
    if hasattr(buf, "data_ptr"):
        if not buf.is_contiguous():
            raise ValueError("tensors must be contiguous")
        return buf.data_ptr()
    raise TypeError(f"cannot take the address of {type(buf)!r}")


def _numel(buf) -> int:
    if isinstance(buf, np.ndarray):
        return buf.size
    return buf.numel()


def _check_f32(bufs):
    for b in bufs:
        if hasattr(b, "dtype") and str(b.dtype) not in ("torch.float32", "float32"):
            raise TypeError(f"expected float32 buffers, got {b.dtype}")


def _ptr_array(bufs: Sequence) -> ctypes.Array:
    return (ctypes.c_void_p * len(bufs))(*[_addr(b) for b in bufs])


def _stream(stream) -> int:
    if stream is None:
        import torch
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _offsets(layer_offsets):
    if layer_offsets is None:
        return None, 0
    off = np.ascontiguousarray(np.asarray(layer_offsets), dtype=np.int64)
    return off, off.size - 1


def _raise(status: int, where: str):
    if status < 0:
        raise GrawaError(status, where)


def _options(weights_out=None, scores_out=None, sumsq_out=None, workspace=None, status_word=None):
    """The optional-arguments struct, or None when every option is at its default."""
    if all(b is None for b in (weights_out, scores_out, sumsq_out, workspace, status_word)):
        return None
    ws_bytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    return _Options(_addr(weights_out), _addr(scores_out), _addr(sumsq_out), _addr(workspace), ws_bytes, _addr(status_word))


def _byref(opt):
    return ctypes.byref(opt) if opt is not None else None


_DTYPES = {"torch.float32": 0, "torch.bfloat16": 1, "torch.float16": 2, "float32": 0, "float16": 2}


def _dtype_of(bufs) -> int:
    """Storage type code of a list of buffers (all of one type)."""
    key = str(bufs[0].dtype)
    if key not in _DTYPES:
        raise TypeError(f"unsupported storage dtype {key}")
    for b in bufs:
        if str(b.dtype) != key:
            raise TypeError(f"all buffers must be {key}, got {b.dtype}")
    return _DTYPES[key]


def _step(name, params, grads, pull, layer_offsets, center_out, weights_out, scores_out, sumsq_out,
          workspace, stream, n, status_word=None):
    lib = library()
    if len(params) != len(grads):
        raise ValueError("params and grads must have one entry per worker")
    _check_f32(list(params) + list(grads) + ([center_out] if center_out is not None else []))
    M = len(params)
    if n is None:
        n = _numel(params[0]) if M else 0
    off, K = _offsets(layer_offsets)
    opt = _options(weights_out, scores_out, sumsq_out, workspace, status_word)
    status = getattr(lib, name)(_ptr_array(params), _ptr_array(grads), n, M, float(pull),
                                off.ctypes.data if off is not None else None, K, _addr(center_out),
                                _byref(opt), _stream(stream))
    _raise(status, name)


# ------------------------------------------------------------------ entry points (same names as the C ABI)

def grawa_mgrawa_step(params, grads, pull, layer_offsets=None, center_out=None, *, weights_out=None,
                      scores_out=None, sumsq_out=None, workspace=None, stream=None, n=None, status_word=None) -> None:
    """MGRAWA step (Eq. 3-4, centre, pull) in place on ``params``; see grawa_mgrawa_step in grawa.h."""
    _step("grawa_mgrawa_step", params, grads, pull, layer_offsets, center_out, weights_out, scores_out,
          sumsq_out, workspace, stream, n, status_word)


def grawa_grawa_step(params, grads, pull, layer_offsets=None, center_out=None, *, weights_out=None,
                     scores_out=None, sumsq_out=None, workspace=None, stream=None, n=None, status_word=None) -> None:
    """Vanilla GRAWA step (Eq. 2: flat gradient norm); see grawa_grawa_step in grawa.h."""
    _step("grawa_grawa_step", params, grads, pull, layer_offsets, center_out, weights_out, scores_out,
          sumsq_out, workspace, stream, n, status_word)


def grawa_lgrawa_step(params, grads, pull, layer_offsets, center_out=None, *, weights_out=None,
                      scores_out=None, sumsq_out=None, workspace=None, stream=None, n=None, status_word=None) -> None:
    """LGRAWA step (Eq. 5-7: per-layer weights); see grawa_lgrawa_step in grawa.h."""
    _step("grawa_lgrawa_step", params, grads, pull, layer_offsets, center_out, weights_out, scores_out,
          sumsq_out, workspace, stream, n, status_word)


def grawa_step_typed(variant, params, grads, pull, layer_offsets=None, center_out=None, *, weights_out=None,
                     scores_out=None, sumsq_out=None, workspace=None, stream=None, n=None, status_word=None) -> None:
    """The step on parameters / gradients / centre stored as float32, bfloat16 or float16 device tensors
    (all of one dtype, taken from ``params[0]``); arithmetic in fp32/fp64, one rounding per stored value."""
    M = len(params)
    if len(grads) != M or M == 0:
        raise ValueError("params and grads must have one entry per worker")
    dt = _dtype_of(list(params) + list(grads) + ([center_out] if center_out is not None else []))
    v = _VARIANTS[variant] if isinstance(variant, str) else int(variant)
    if n is None:
        n = _numel(params[0])
    off, K = _offsets(layer_offsets)
    opt = _options(weights_out, scores_out, sumsq_out, workspace, status_word)
    _raise(library().grawa_step_typed(dt, v, _ptr_array(params), _ptr_array(grads), n, M, float(pull),
                                      off.ctypes.data if off is not None else None, K, _addr(center_out),
                                      _byref(opt), _stream(stream)), "grawa_step_typed")


def grawa_step_host_typed(variant, params, grads, pull, layer_offsets=None, center_out=None, *, stream=None, n=None) -> None:
    """Whole step with HOST buffers (numpy arrays or pinned CPU tensors) of float32, float16 or bfloat16;
    synchronises before returning."""
    v = _VARIANTS[variant] if isinstance(variant, str) else int(variant)
    M = len(params)
    dt = _dtype_of(list(params) + list(grads) + ([center_out] if center_out is not None else []))
    if n is None:
        n = _numel(params[0]) if M else 0
    off, K = _offsets(layer_offsets)
    _raise(library().grawa_step_host_typed(dt, v, _ptr_array(params), _ptr_array(grads), n, M, float(pull),
                                           off.ctypes.data if off is not None else None, K, _addr(center_out),
                                           _stream(stream)), "grawa_step_host_typed")


def grawa_step_host(variant, params, grads, pull, layer_offsets=None, center_out=None, *, stream=None, n=None) -> None:
    """Whole step with HOST float32 buffers (numpy arrays or pinned CPU tensors); synchronises before returning."""
    lib = library()
    v = _VARIANTS[variant] if isinstance(variant, str) else int(variant)
    _check_f32(list(params) + list(grads) + ([center_out] if center_out is not None else []))
    M = len(params)
    if n is None:
        n = _numel(params[0]) if M else 0
    off, K = _offsets(layer_offsets)
    status = lib.grawa_step_host(v, _ptr_array(params), _ptr_array(grads), n, M, float(pull),
                                 off.ctypes.data if off is not None else None, K, _addr(center_out), _stream(stream))
    _raise(status, "grawa_step_host")


def grawa_prox_step_typed(params, center, mu_over_tau, *, stream=None, n=None) -> None:
    """Proximity step on float32, bfloat16 or float16 device tensors (dtype taken from the buffers)."""
    dt = _dtype_of(list(params) + [center])
    if n is None:
        n = _numel(center)
    _raise(library().grawa_prox_step_typed(dt, _ptr_array(params), _addr(center), n, len(params), float(mu_over_tau),
                                           _stream(stream)), "grawa_prox_step_typed")


def grawa_prox_step(params, center, mu_over_tau, *, stream=None, n=None) -> None:
    """Proximity step x_m <- (1 - mu/tau) x_m + (mu/tau) x_C for all workers in one pass."""
    lib = library()
    _check_f32(list(params) + [center])
    M = len(params)
    if n is None:
        n = _numel(center)
    _raise(lib.grawa_prox_step(_ptr_array(params), _addr(center), n, M, float(mu_over_tau), _stream(stream)),
           "grawa_prox_step")


def grawa_layer_norms_typed(grad, layer_offsets, norms_out, *, stream=None, n=None) -> None:
    """Per-layer L2 norms of one worker's gradient (float32, bfloat16 or float16) into ``norms_out`` (K float64)."""
    dt = _dtype_of([grad])
    if n is None:
        n = _numel(grad)
    off, K = _offsets(layer_offsets)
    _raise(library().grawa_layer_norms_typed(dt, _addr(grad), n, off.ctypes.data if off is not None else None, K,
                                             _addr(norms_out), _stream(stream)), "grawa_layer_norms_typed")


def grawa_layer_norms(grad, layer_offsets, norms_out, *, stream=None, n=None) -> None:
    """Per-layer L2 norms of one worker's gradient into ``norms_out`` (device, K float64)."""
    _check_f32([grad])
    if n is None:
        n = _numel(grad)
    off, K = _offsets(layer_offsets)
    _raise(library().grawa_layer_norms(_addr(grad), n, off.ctypes.data if off is not None else None, K,
                                       _addr(norms_out), _stream(stream)), "grawa_layer_norms")


def grawa_norm_ema(g_mvg, g_cur, gamma, t, g_est, *, stream=None) -> None:
    """Running norm estimate of the Local variants on device float64 vectors (g_mvg updated in place)."""
    _raise(library().grawa_norm_ema(_addr(g_mvg), _addr(g_cur), _numel(g_mvg), float(gamma), int(t), _addr(g_est),
                                    _stream(stream)), "grawa_norm_ema")


def _from_given(name, typed, variant, params, table, parts, pull, layer_offsets, center_out, weights_out, scores_out,
                sumsq_out, workspace, stream, n, status_word):
    v = _VARIANTS[variant] if isinstance(variant, str) else int(variant)
    bufs = list(params) + ([center_out] if center_out is not None else [])
    M = len(params)
    if n is None:
        n = _numel(params[0]) if M else 0
    off, K = _offsets(layer_offsets)
    opt = _options(weights_out, scores_out, sumsq_out, workspace, status_word)
    head = [_dtype_of(bufs), v] if typed else [v]
    if not typed:
        _check_f32(bufs)
    mid = [_ptr_array(params), _addr(table)] + ([int(parts)] if parts is not None else [])
    tail = [n, M, float(pull), off.ctypes.data if off is not None else None, K, _addr(center_out), _byref(opt), _stream(stream)]
    _raise(getattr(library(), name)(*(head + mid + tail)), name)


def grawa_step_from_layer_norms(variant, params, layer_norms, pull, layer_offsets=None, center_out=None, *,
                                weights_out=None, scores_out=None, sumsq_out=None, workspace=None, stream=None,
                                n=None, status_word=None) -> None:
    """Averaging step with scores from given per-layer norms ([K, M] device float64) instead of gradients."""
    _from_given("grawa_step_from_layer_norms", False, variant, params, layer_norms, None, pull, layer_offsets, center_out,
                weights_out, scores_out, sumsq_out, workspace, stream, n, status_word)


def grawa_step_from_layer_norms_typed(variant, params, layer_norms, pull, layer_offsets=None, center_out=None, *,
                                      weights_out=None, scores_out=None, sumsq_out=None, workspace=None, stream=None,
                                      n=None, status_word=None) -> None:
    """The same on float32, bfloat16 or float16 parameters and centre."""
    _from_given("grawa_step_from_layer_norms_typed", True, variant, params, layer_norms, None, pull, layer_offsets,
                center_out, weights_out, scores_out, sumsq_out, workspace, stream, n, status_word)


def grawa_layer_sumsq(grads, layer_offsets, sumsq_out, *, stream=None, n=None) -> None:
    """Per-layer sums of squares of the M workers' local gradients into ``sumsq_out`` ([K, M] device float64)."""
    _check_f32(list(grads))
    M = len(grads)
    if n is None:
        n = _numel(grads[0]) if M else 0
    off, K = _offsets(layer_offsets)
    _raise(library().grawa_layer_sumsq(_ptr_array(grads), n, M, off.ctypes.data if off is not None else None, K,
                                       _addr(sumsq_out), _stream(stream)), "grawa_layer_sumsq")


def grawa_layer_sumsq_typed(grads, layer_offsets, sumsq_out, *, stream=None, n=None) -> None:
    """The same from float32, bfloat16 or float16 gradients."""
    M = len(grads)
    dt = _dtype_of(list(grads))
    if n is None:
        n = _numel(grads[0]) if M else 0
    off, K = _offsets(layer_offsets)
    _raise(library().grawa_layer_sumsq_typed(dt, _ptr_array(grads), n, M, off.ctypes.data if off is not None else None, K,
                                             _addr(sumsq_out), _stream(stream)), "grawa_layer_sumsq_typed")


def grawa_step_from_layer_sums(variant, params, layer_sums, parts, pull, layer_offsets=None, center_out=None, *,
                               weights_out=None, scores_out=None, sumsq_out=None, workspace=None, stream=None,
                               n=None, status_word=None) -> None:
    """Averaging step on local elements with S = sum over ``parts`` tables of ``layer_sums`` ([parts, K, M])."""
    _from_given("grawa_step_from_layer_sums", False, variant, params, layer_sums, parts, pull, layer_offsets, center_out,
                weights_out, scores_out, sumsq_out, workspace, stream, n, status_word)


def grawa_step_from_layer_sums_typed(variant, params, layer_sums, parts, pull, layer_offsets=None, center_out=None, *,
                                     weights_out=None, scores_out=None, sumsq_out=None, workspace=None, stream=None,
                                     n=None, status_word=None) -> None:
    """The same on float32, bfloat16 or float16 parameters and centre."""
    _from_given("grawa_step_from_layer_sums_typed", True, variant, params, layer_sums, parts, pull, layer_offsets,
                center_out, weights_out, scores_out, sumsq_out, workspace, stream, n, status_word)


class PreparedStep:
    """A device-buffer step with its arguments marshalled once: calling the object makes the same C call
    (grawa_step_typed) again on the stream that is current at that moment.  For loops over small models,
    where building the pointer tables in Python costs as much as the update.  Holds references to the
    buffers; marshals only, like every function of this module."""

    def __init__(self, variant, params, grads, pull, layer_offsets=None, center_out=None, *, status_word=None):
        self._keep = (list(params), list(grads), center_out, status_word)
        self._dt = _dtype_of(list(params) + list(grads) + ([center_out] if center_out is not None else []))
        self._v = _VARIANTS[variant] if isinstance(variant, str) else int(variant)
        self._params, self._grads = _ptr_array(params), _ptr_array(grads)
        self._n, self._M, self._pull = _numel(params[0]), len(params), float(pull)
        self._off, self._K = _offsets(layer_offsets)
        self._off_ptr = self._off.ctypes.data if self._off is not None else None
        self._center = _addr(center_out)
        self._opt = _options(status_word=status_word)
        self._fn = library().grawa_step_typed

    def __call__(self, stream=None) -> None:
        status = self._fn(self._dt, self._v, self._params, self._grads, self._n, self._M, self._pull, self._off_ptr, self._K,
                          self._center, _byref(self._opt), _stream(stream))
        if status < 0:
            raise GrawaError(status, "grawa_step_typed")


def grawa_sumsq_static(grads, sumsq_out, *, stream=None, n=None) -> None:
    """Squared gradient norms of the M workers into ``sumsq_out`` (device, M float64) using only
    the scratch array built into the library: for callers whose device memory belongs to another
    allocator, or who cannot afford the synchronisation an allocation implies.  Calls that may
    overlap on the GPU share that array and race; keep them on one stream."""
    _check_f32(list(grads))
    M = len(grads)
    if n is None:
        n = _numel(grads[0]) if M else 0
    _raise(library().grawa_sumsq_static(_ptr_array(grads), n, M, _addr(sumsq_out), _stream(stream)),
           "grawa_sumsq_static")


# ------------------------------------------------------------------ replica operators

_marshal = None
_addresses = {}                               # of entry points
_ROWS, _OPTIONAL, _FLOAT32, _INT64 = 1, 2, 4, 8          # modes of a table, as in csrc/marshal.cpp; << 8: the head dimension
_ACTIVATIONS = {"silu": 0, "gelu": 1, "relu": 2}
_PAIRINGS = {"halves": 0, "neighbours": 1}


def _tables(first, specs):
    """Storage type code, then pointer table (bytes, read by the C call, or 0) and layout (16 * row stride + the low 4 bits of
    the addresses; stride 0 for contiguous tensors) of each spec (name, tensors or None, rows, cols, mode), from the native
    marshaller, which checks types, sizes, shapes, contiguity and that all tensors are on the current device; last the device."""
    global _marshal
    import torch
    if _marshal is None:
        _build.build_marshal()
        from . import _marshal as native
        _marshal = native
        torch.cuda.init()
    device = torch._C._cuda_getDevice()
    return _marshal.tables(first, device, specs) + (device,)


def _call(name, *args) -> int:
    """Status of an entry point, called by way of the native marshaller (loaded by _tables)."""
    address = _addresses.get(name)
    if address is None:
        address = _addresses[name] = ctypes.cast(getattr(library(), name), ctypes.c_void_p).value
    return getattr(_marshal, name)(address, *args)


def _stream_on(stream, device) -> int:
    if stream is None:
        import torch
        return torch._C._cuda_getCurrentRawStream(device)
    return _stream(stream)


def _matrix_shape(t, name):
    shape = t.shape
    if len(shape) != 2:
        raise ValueError(f"{name}: expected 2-D tensors")
    return shape


def _scratch(workspace, need, stream):
    """The caller's workspace, or one from torch's allocator that is tied to the call's stream."""
    if workspace is not None or not need:
        return workspace
    import torch
    if stream is None:
        return torch.empty(need, dtype=torch.uint8, device="cuda")
    with torch.cuda.stream(torch.cuda.ExternalStream(_stream(stream))):
        return torch.empty(need, dtype=torch.uint8, device="cuda")


def _on_device(buf, device, name):
    if buf.get_device() != device:
        raise ValueError(f"{name}: expected a tensor on the current CUDA device ({device}), got {buf.device}")


def _scratch_args(workspace, device):
    if workspace is None:
        return None, 0
    _on_device(workspace, device, "workspace")
    return _addr(workspace), workspace.numel() * workspace.element_size()


def _counter(offset_counter, device):
    if offset_counter is None or isinstance(offset_counter, int):
        return offset_counter
    if offset_counter.element_size() != 8 or offset_counter.is_floating_point():
        raise TypeError("offset_counter: expected a 64-bit integer device tensor")
    _on_device(offset_counter, device, "offset_counter")
    if offset_counter.numel() < 1:
        raise ValueError("offset_counter: expected one element")
    return _addr(offset_counter)


def grawa_dropout_forward(x, y, p, seed, offset=0, *, residual=None, offset_counter=None, stream=None) -> None:
    """y = residual + dropout(x) for all workers (lists of device tensors of equal size); the mask is a function
    of (seed, offset + counter, worker, element) and never stored; see grawa_dropout_forward in grawa.h."""
    n = x[0].numel()
    code, xt, _, rt, _, yt, _, dev = _tables(x, (("x", x, n, 1, 0), ("residual", residual, n, 1, _OPTIONAL), ("y", y, n, 1, 0)))
    status = library().grawa_dropout_forward(code, xt, rt, yt, n, len(x), p, seed, offset, _counter(offset_counter, dev), _stream_on(stream, dev))
    _raise(status, "grawa_dropout_forward")


def grawa_dropout_backward(dy, dx, p, seed, offset=0, *, offset_counter=None, stream=None) -> None:
    """dx = dy where the forward call with these p, seed, offset and counter kept the element, scaled; else 0."""
    n = dy[0].numel()
    code, yt, _, xt, _, dev = _tables(dy, (("dy", dy, n, 1, 0), ("dx", dx, n, 1, 0)))
    status = library().grawa_dropout_backward(code, yt, xt, n, len(dy), p, seed, offset, _counter(offset_counter, dev), _stream_on(stream, dev))
    _raise(status, "grawa_dropout_backward")


def grawa_layernorm_forward(x, gamma, beta, y, eps=1e-5, *, mean=None, rstd=None, stream=None) -> None:
    """Layer norm of the rows of each worker's x ([rows, cols], rows may be padded) into y; gamma and beta ([cols])
    may be None; mean and rstd ([rows] float32) are filled for the backward pass when given."""
    rows, cols = _matrix_shape(x[0], "x")
    code, xt, xs, gt, _, bt, _, yt, ys, mt, _, rt, _, dev = _tables(x, (
        ("x", x, rows, cols, _ROWS), ("gamma", gamma, cols, 1, _OPTIONAL), ("beta", beta, cols, 1, _OPTIONAL), ("y", y, rows, cols, _ROWS),
        ("mean", mean, rows, 1, _OPTIONAL | _FLOAT32), ("rstd", rstd, rows, 1, _OPTIONAL | _FLOAT32)))
    status = library().grawa_layernorm_forward(code, xt, gt, bt, yt, mt, rt, rows, cols, xs >> 4, ys >> 4, len(x), eps, _stream_on(stream, dev))
    _raise(status, "grawa_layernorm_forward")


def grawa_layernorm_backward(dy, x, gamma, mean, rstd, dx, dgamma, dbeta, *, accumulate=False, workspace=None, stream=None) -> None:
    """Gradients of grawa_layernorm_forward; dx, dgamma and dbeta may each be None.  accumulate adds dgamma and dbeta
    to what the buffers hold.  dx needs x's row stride.  Without a workspace the call takes one from torch's allocator."""
    lib, M = library(), len(x)
    rows, cols = _matrix_shape(x[0], "x")
    code, yt, ys, xt, xs, gt, _, mt, _, rt, _, dxt, dxs, dgt, _, dbt, _, dev = _tables(x, (
        ("dy", dy, rows, cols, _ROWS), ("x", x, rows, cols, _ROWS), ("gamma", gamma, cols, 1, _OPTIONAL), ("mean", mean, rows, 1, _FLOAT32),
        ("rstd", rstd, rows, 1, _FLOAT32), ("dx", dx, rows, cols, _ROWS | _OPTIONAL), ("dgamma", dgamma, cols, 1, _OPTIONAL),
        ("dbeta", dbeta, cols, 1, _OPTIONAL)))
    if dx is not None and dxs >> 4 != xs >> 4:
        raise ValueError("dx: expected the row stride of x")
    keep = workspace
    if keep is None and (dgamma is not None or dbeta is not None):
        size = 4 if code == 0 else 2                          # aligned: no address, stride or row end inside a 16-byte word
        inside = (xs | ys | (dxs if dx is not None else 0)) & 15 | (cols | xs >> 4 | ys >> 4) * size & 15
        keep = _scratch(None, lib.grawa_layernorm_backward_workspace_bytes(rows, cols, M, 0 if inside else 1), stream)
    status = lib.grawa_layernorm_backward(code, yt, xt, gt, mt, rt, dxt, dgt, dbt, rows, cols, xs >> 4, ys >> 4, M, 1 if accumulate else 0,
                                          *_scratch_args(keep, dev), _stream_on(stream, dev))
    _raise(status, "grawa_layernorm_backward")


def grawa_layernorm_backward_workspace_bytes(rows: int, cols: int, M: int, aligned: bool = False) -> int:
    return int(library().grawa_layernorm_backward_workspace_bytes(rows, cols, M, 1 if aligned else 0))


def _ffn_sizes(x, w_gate):
    rows, d_in = _matrix_shape(x[0], "x")
    d_hidden, of_weights = _matrix_shape(w_gate[0], "w_gate")
    if of_weights != d_in:
        raise ValueError(f"expected x [rows, d_in] and weights [d_hidden, d_in], got {d_in} and {of_weights} columns")
    return rows, d_in, d_hidden


def grawa_gated_ffn_forward(x, w_gate, w_up, h, *, activation="silu", gate_out=None, up_out=None, workspace=None, stream=None) -> None:
    """h = act(x w_gate^T) * (x w_up^T) for each worker's x [rows, d_in], weights [d_hidden, d_in] (views into the flat
    parameter vectors will do), bfloat16 or float16; gate_out and up_out receive the two products for the backward pass."""
    lib, M = library(), len(x)
    rows, d_in, d_hidden = _ffn_sizes(x, w_gate)
    act = _ACTIVATIONS[activation] if isinstance(activation, str) else int(activation)
    code, xt, xa, gt, ga, ut, ua, ht, _, got, _, uot, _, dev = _tables(x, (
        ("x", x, rows, d_in, 0), ("w_gate", w_gate, d_hidden, d_in, 0), ("w_up", w_up, d_hidden, d_in, 0), ("h", h, rows, d_hidden, 0),
        ("gate_out", gate_out, rows, d_hidden, _OPTIONAL), ("up_out", up_out, rows, d_hidden, _OPTIONAL)))
    keep = workspace
    if keep is None:
        keep = _scratch(None, lib.grawa_gated_ffn_workspace_bytes(rows, d_in, d_hidden, M, 0, 0 if (xa | ga | ua) & 15 else 1), stream)
    status = lib.grawa_gated_ffn_forward(code, act, xt, gt, ut, ht, got, uot, rows, d_in, d_hidden, M, *_scratch_args(keep, dev), _stream_on(stream, dev))
    _raise(status, "grawa_gated_ffn_forward")


def grawa_gated_ffn_backward(dh, x, w_gate, w_up, gate, up, dx, dw_gate, dw_up, *, activation="silu", accumulate=False, workspace=None,
                             stream=None) -> None:
    """Gradients of grawa_gated_ffn_forward from dh and its gate_out and up_out; dx may be None, dw_gate and dw_up both may be.
    accumulate adds the weights' gradients to what the buffers hold.  Without a workspace the call takes one from torch's allocator."""
    lib, M = library(), len(x)
    rows, d_in, d_hidden = _ffn_sizes(x, w_gate)
    act = _ACTIVATIONS[activation] if isinstance(activation, str) else int(activation)
    t = _tables(x, (
        ("dh", dh, rows, d_hidden, 0), ("x", x, rows, d_in, 0), ("w_gate", w_gate, d_hidden, d_in, 0), ("w_up", w_up, d_hidden, d_in, 0),
        ("gate", gate, rows, d_hidden, 0), ("up", up, rows, d_hidden, 0), ("dx", dx, rows, d_in, _OPTIONAL),
        ("dw_gate", dw_gate, d_hidden, d_in, _OPTIONAL), ("dw_up", dw_up, d_hidden, d_in, _OPTIONAL)))
    keep = workspace
    if keep is None:
        keep = _scratch(None, lib.grawa_gated_ffn_workspace_bytes(rows, d_in, d_hidden, M, 1, 0 if (t[4] | t[6] | t[8]) & 15 else 1), stream)
    status = lib.grawa_gated_ffn_backward(t[0], act, *t[1:-1:2], rows, d_in, d_hidden, M, 1 if accumulate else 0, *_scratch_args(keep, t[-1]),
                                          _stream_on(stream, t[-1]))
    _raise(status, "grawa_gated_ffn_backward")


def grawa_gated_ffn_workspace_bytes(rows: int, d_in: int, d_hidden: int, M: int, backward: bool = False, aligned: bool = True) -> int:
    return int(library().grawa_gated_ffn_workspace_bytes(rows, d_in, d_hidden, M, 1 if backward else 0, 1 if aligned else 0))


def grawa_gated_ffn_status(stream=None) -> int:
    """Synchronises the stream and returns 0, or -5 when a bounded wait of a gated feed-forward call ran out."""
    return int(library().grawa_gated_ffn_status(_stream(stream)))


def grawa_selftest_gated_ffn_wait(*, stream=None) -> None:
    """Launches the product kernel's bounded-wait self-test; grawa_gated_ffn_status then reports -5."""
    _raise(library().grawa_selftest_gated_ffn_wait(_stream(stream)), "grawa_selftest_gated_ffn_wait")


def _heads(t, name):
    shape = t[0].shape
    if len(shape) != 3:
        raise ValueError(f"{name}: expected 3-D tensors [rows, heads, head_dim]")
    return shape


def _frequencies(frequencies, device):
    """Address and number of the rotated elements."""
    if frequencies is None:
        return None, 0
    address, count = _marshal.vector("frequencies", frequencies, device)
    return address, 2 * count


def _head_specs(q, k):
    """Sizes (rows, query heads, key heads, head_dim) and the modes of tables of heads."""
    rows, heads, dim = _heads(q, "q")
    kv_heads = 0
    if k is not None:
        kv_heads = _heads(k, "k")[1]
        if kv_heads == 0:
            raise ValueError("k: expected at least one head")
    return rows, heads, kv_heads, dim, _ROWS | dim << 8


def grawa_head_rotary_forward(q, k, q_weight, k_weight, q_out, k_out, frequencies, *, positions=None, period=None, pairing="halves", eps=1e-6,
                              stream=None) -> None:
    """RMS norm of each head of q and k (lists of [rows, heads, head_dim], rows may be padded) with the weights ([head_dim], or
    None), then the rotation of the leading 2 * len(frequencies) elements (float64, device; None: none) by the rows' positions ([rows]
    int64; None: the row number, modulo ``period`` if given).  k, k_weight and k_out may be None; q_out may be q, k_out k."""
    rows, heads, kv_heads, dim, mode = _head_specs(q, k)
    code, qt, qs, kt, ks, qw, _, kw, _, qo, qos, ko, kos, pos, _, dev = _tables(q, (
        ("q", q, rows, heads * dim, mode), ("k", k, rows, kv_heads * dim, mode | _OPTIONAL), ("q_weight", q_weight, dim, 1, _OPTIONAL),
        ("k_weight", k_weight, dim, 1, _OPTIONAL), ("q_out", q_out, rows, heads * dim, mode),
        ("k_out", k_out, rows, kv_heads * dim, mode if kv_heads else mode | _OPTIONAL), ("positions", positions, rows, 1, _OPTIONAL | _INT64)))
    f, rotary = _frequencies(frequencies, dev)
    status = _call("grawa_head_rotary_forward", code, _PAIRINGS[pairing], qt, kt, qw, kw, qo, ko, pos, f, rows, heads, kv_heads, dim, rotary, qs >> 4, ks >> 4,
                                                 qos >> 4, kos >> 4, (rows or 1) if period is None else period, len(q), eps, _stream_on(stream, dev))
    _raise(status, "grawa_head_rotary_forward")


def grawa_head_rotary_backward(dq_out, dk_out, q, k, q_weight, k_weight, dq, dk, dq_weight, dk_weight, frequencies, *, positions=None, period=None,
                               pairing="halves", eps=1e-6, accumulate=False, workspace=None, stream=None) -> None:
    """Gradients of grawa_head_rotary_forward; dq, dk, dq_weight and dk_weight may each be None.  dq and dk need the row strides of q
    and k, and may be dq_out and dk_out where those have them too.  accumulate adds the weights' gradients to what the buffers hold."""
    lib, M = library(), len(q)
    rows, heads, kv_heads, dim, mode = _head_specs(q, k)
    optional = mode | _OPTIONAL
    code, qo, qos, ko, kos, qt, qs, kt, ks, qw, _, kw, _, dqt, dqs, dkt, dks, dqw, _, dkw, _, pos, _, dev = _tables(q, (
        ("dq_out", dq_out, rows, heads * dim, mode), ("dk_out", dk_out, rows, kv_heads * dim, mode if kv_heads else optional),
        ("q", q, rows, heads * dim, mode), ("k", k, rows, kv_heads * dim, optional), ("q_weight", q_weight, dim, 1, _OPTIONAL),
        ("k_weight", k_weight, dim, 1, _OPTIONAL), ("dq", dq, rows, heads * dim, optional), ("dk", dk, rows, kv_heads * dim, optional),
        ("dq_weight", dq_weight, dim, 1, _OPTIONAL), ("dk_weight", dk_weight, dim, 1, _OPTIONAL), ("positions", positions, rows, 1, _OPTIONAL | _INT64)))
    for name, t, s, of in (("dq", dq, dqs, qs), ("dk", dk, dks, ks)):
        if t is not None and s >> 4 != of >> 4:
            raise ValueError(f"{name}: expected the row stride of {name[1:]}")
    f, rotary = _frequencies(frequencies, dev)
    keep = workspace
    if keep is None and (dq_weight is not None or dk_weight is not None):
        keep = _scratch(None, lib.grawa_head_rotary_backward_workspace_bytes(rows, M), stream)
    status = _call("grawa_head_rotary_backward", code, _PAIRINGS[pairing], qo, ko, qt, kt, qw, kw, dqt, dkt, dqw, dkw, pos, f, rows, heads, kv_heads, dim, rotary,
                                            qs >> 4, ks >> 4, qos >> 4, kos >> 4, (rows or 1) if period is None else period, M, eps, 1 if accumulate else 0,
                                            *_scratch_args(keep, dev), _stream_on(stream, dev))
    _raise(status, "grawa_head_rotary_backward")


def grawa_head_rotary_backward_workspace_bytes(rows: int, M: int) -> int:
    return int(library().grawa_head_rotary_backward_workspace_bytes(rows, M))


def _window(rows, offsets, period, left, right, sinks):
    """offsets' length, then sequences, period, left, right and sinks as the C calls take them (None: no limit)."""
    length = offsets[0].numel() if offsets is not None else 0
    if offsets is not None and length < 1:
        raise ValueError("offsets: expected at least one element")
    every = rows or 1
    return length, (max(0, length - 1), every if period is None else period, every if left is None else left, every if right is None else right, sinks)


def grawa_window_attention_forward(q, k, v, out, *, lse=None, offsets=None, period=None, left=None, right=0, sinks=0, scale=None, stream=None) -> None:
    """Attention of q ([rows, heads, head_dim]) over k and v ([rows, kv_heads, head_dim]) of each worker, bfloat16 or float16, rows
    may be padded: a row sees the keys of its sequence from ``left`` rows in front of it (None: all) to ``right`` behind it (0:
    causal, None: all), and of the sequence's first ``sinks`` rows those up to there.  Sequences: offsets ([sequences + 1] int64) or
    ``period`` rows each (None: one).  lse ([heads, rows] float32) is filled for the backward pass when given."""
    rows, heads, kv_heads, dim, mode = _head_specs(q, k)
    length, window = _window(rows, offsets, period, left, right, sinks)
    code, qt, qs, kt, ks, vt, vs, ot, os, lt, _, off, _, dev = _tables(q, (
        ("q", q, rows, heads * dim, mode), ("k", k, rows, kv_heads * dim, mode), ("v", v, rows, kv_heads * dim, mode), ("out", out, rows, heads * dim, mode),
        ("lse", lse, heads, rows, _OPTIONAL | _FLOAT32), ("offsets", offsets, length, 1, _OPTIONAL | _INT64)))
    status = _call("grawa_window_attention_forward", code, qt, kt, vt, ot, lt, off, *window, rows, heads, kv_heads, dim, qs >> 4, ks >> 4, vs >> 4, os >> 4,
                                                      len(q), dim ** -0.5 if scale is None else scale, _stream_on(stream, dev))
    _raise(status, "grawa_window_attention_forward")


def grawa_window_attention_backward(dout, q, k, v, out, lse, dq, dk, dv, *, offsets=None, period=None, left=None, right=0, sinks=0, scale=None,
                                    workspace=None, stream=None) -> None:
    """Gradients of grawa_window_attention_forward from dout and its out and lse; dq may be None, dk and dv both may be.  dout needs
    the row stride of out, dq, dk and dv those of q, k and v.  Without a workspace the call takes one from torch's allocator."""
    lib, M = library(), len(q)
    rows, heads, kv_heads, dim, mode = _head_specs(q, k)
    length, window = _window(rows, offsets, period, left, right, sinks)
    wide, narrow, optional = heads * dim, kv_heads * dim, mode | _OPTIONAL
    code, gt, gs, qt, qs, kt, ks, vt, vs, ot, os, lt, _, dqt, dqs, dkt, dks, dvt, dvs, off, _, dev = _tables(q, (
        ("dout", dout, rows, wide, mode), ("q", q, rows, wide, mode), ("k", k, rows, narrow, mode), ("v", v, rows, narrow, mode),
        ("out", out, rows, wide, mode), ("lse", lse, heads, rows, _FLOAT32), ("dq", dq, rows, wide, optional), ("dk", dk, rows, narrow, optional),
        ("dv", dv, rows, narrow, optional), ("offsets", offsets, length, 1, _OPTIONAL | _INT64)))
    for name, t, s, of, other in (("dout", dout, gs, os, "out"), ("dq", dq, dqs, qs, "q"), ("dk", dk, dks, ks, "k"), ("dv", dv, dvs, vs, "v")):
        if t is not None and s >> 4 != of >> 4:
            raise ValueError(f"{name}: expected the row stride of {other}")
    keep = workspace
    if keep is None:
        keep = _scratch(None, lib.grawa_window_attention_backward_workspace_bytes(rows, heads, kv_heads, dim, sinks, M), stream)
    status = _call("grawa_window_attention_backward", code, gt, qt, kt, vt, ot, lt, dqt, dkt, dvt, off, *window, rows, heads, kv_heads, dim, qs >> 4, ks >> 4, vs >> 4,
                                                 os >> 4, M, dim ** -0.5 if scale is None else scale, *_scratch_args(keep, dev), _stream_on(stream, dev))
    _raise(status, "grawa_window_attention_backward")


def grawa_window_attention_backward_workspace_bytes(rows: int, q_heads: int, kv_heads: int, head_dim: int, sinks: int, M: int) -> int:
    return int(library().grawa_window_attention_backward_workspace_bytes(rows, q_heads, kv_heads, head_dim, sinks, M))


def grawa_window_attention_status(stream=None) -> int:
    """Synchronises the stream and returns 0, or -5 when a bounded wait of an attention call ran out."""
    return int(library().grawa_window_attention_status(_stream(stream)))


def grawa_selftest_window_attention_wait(*, stream=None) -> None:
    """Launches the attention kernel's bounded-wait self-test; grawa_window_attention_status then reports -5."""
    _raise(library().grawa_selftest_window_attention_wait(_stream(stream)), "grawa_selftest_window_attention_wait")


def grawa_workspace_bytes(n: int, M: int, layer_offsets=None) -> int:
    off, K = _offsets(layer_offsets)
    return int(library().grawa_workspace_bytes(n, M, off.ctypes.data if off is not None else None, K))


def grawa_last_step_status(stream=None) -> int:
    """Synchronises the stream and returns the status code of the last step enqueued on it."""
    return int(library().grawa_last_step_status(_stream(stream)))


def grawa_status_string(status: int) -> str:
    return library().grawa_status_string(int(status)).decode()


def grawa_last_cuda_error() -> str:
    return library().grawa_last_cuda_error().decode()


def grawa_version() -> int:
    return int(library().grawa_version())


def grawa_set_option(name: str, value: int) -> None:
    _raise(library().grawa_set_option(name.encode(), int(value)), f"grawa_set_option({name})")


def grawa_get_option(name: str) -> int:
    return int(library().grawa_get_option(name.encode()))


def grawa_launch_count() -> int:
    return int(library().grawa_launch_count())


def grawa_collect_kernel_times() -> dict:
    """Per-phase device time (ms, summed) of the steps run while option "kernel_timing" was 1."""
    a, b, c = ctypes.c_double(), ctypes.c_double(), ctypes.c_double()
    k = ctypes.c_int64()
    _raise(library().grawa_collect_kernel_times(ctypes.byref(a), ctypes.byref(b), ctypes.byref(c), ctypes.byref(k)),
           "grawa_collect_kernel_times")
    return {"sumsq_ms": a.value, "finalize_ms": b.value, "center_pull_ms": c.value, "steps": k.value}


def grawa_selftest_bounded_wait(limit_ns: int, *, stream=None) -> None:
    """Launches the bounded-wait self-test; read the outcome with grawa_last_step_status (expect -5)."""
    _raise(library().grawa_selftest_bounded_wait(int(limit_ns), _stream(stream)), "grawa_selftest_bounded_wait")


def grawa_debug_bounds_violations(selfcheck: bool = False) -> int:
    """Violations counted by a bounds-checking debug build since the last call (-1 in a normal build)."""
    return int(library().grawa_debug_bounds_violations(1 if selfcheck else 0))


def grawa_trace_read(max_rows: int = 64):
    """Trace build (GRAWA_TRACE=1 in the environment): the rows stamped since the last call as an
    array [rows, 3 kernels, 4 stamps] of uint64 nanoseconds, and a reset.  None in the normal build."""
    buf = np.zeros((max_rows, 3, 4), dtype=np.uint64)
    kept = int(library().grawa_trace_read(buf.ctypes.data, max_rows))
    if kept == -1:
        return None
    if kept < 0:
        raise GrawaError(-2, "grawa_trace_read")
    return buf


def grawa_clear_plans() -> None:
    library().grawa_clear_plans()
