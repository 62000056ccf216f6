"""Thin ctypes binding of liba2sgd (the C ABI declared in include/a2sgd.h).

Argument marshalling only: every step of the path runs in the library's CUDA
kernels.  Tensors are used for device memory and streams, nothing else.  There
is no fallback: if the shared library has not been built, or a call returns a
negative status, an exception is raised.

Layout conventions (same as the header): ``grad`` / ``err`` are float32 CUDA
tensors ``[P, >= n]`` with unit inner stride (row p = worker p); ``w`` is
``[>= n]`` (one shared vector) or ``[P, >= n]`` (one replica per worker).
"""
from __future__ import annotations

import ctypes
import os
import struct
from typing import Optional, Tuple

import torch

OK = 0
ERR_ARG, ERR_ALIGN, ERR_CUDA, ERR_TIMEOUT, ERR_NONFINITE, ERR_NOMEM, ERR_TOO_LARGE, ERR_BOUNDS = -1, -2, -3, -4, -5, -6, -7, -8
MODE_EF = 0
MODE_ALG1 = 1
FORCE_TWO_PASS = 1 << 4
FORCE_COOPERATIVE = 1 << 5
DEFERRED_RESIDUAL = 1 << 7
CHECK_POINTERS = 1 << 8
TEST_BARRIER_NEVER_OPENS = 1 << 9
DEBUG_CHECKS = 1 << 10
TEST_SHRINK_EXTENTS = 1 << 11
ROW_ALIGN_ELEMS = 32   # 128 bytes: rows that start on a cache-line boundary take the widest vector kernels

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "liba2sgd.so")
_lib = None

_vp = ctypes.c_void_p
_i64 = ctypes.c_int64


class A2SGDError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__(f"{what}: status {status} ({status_string(status)})")


def lib() -> ctypes.CDLL:
    """Loads liba2sgd.so; raises if it has not been built (no CPU fallback exists)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"{LIB_PATH} is missing: build it with `python -m paper_2006_07405_b200.build` "
                "(nvcc, sm_100a). This package has no CPU fallback.")
        l = ctypes.CDLL(LIB_PATH)
        l.a2sgd_create.restype = ctypes.c_int
        l.a2sgd_create.argtypes = [ctypes.POINTER(_vp), ctypes.c_uint64, ctypes.c_uint32, ctypes.c_int, ctypes.c_uint32]
        l.a2sgd_destroy.restype = ctypes.c_int
        l.a2sgd_destroy.argtypes = [_vp]
        l.a2sgd_encode.restype = ctypes.c_int
        l.a2sgd_encode.argtypes = [_vp, _vp, _i64, _vp, _i64, _vp, _vp, _vp, _vp]
        l.a2sgd_global_average.restype = ctypes.c_int
        l.a2sgd_global_average.argtypes = [_vp, _vp, _vp, _vp]
        l.a2sgd_decode_update.restype = ctypes.c_int
        l.a2sgd_decode_update.argtypes = [_vp, _vp, _i64, _vp, _i64, _vp, _i64, _vp, _vp, ctypes.c_float, _vp]
        l.a2sgd_step.restype = ctypes.c_int
        l.a2sgd_step.argtypes = [_vp, _vp, _i64, _vp, _i64, _vp, _i64, ctypes.c_float, _vp]
        l.a2sgd_decode_update_momentum.restype = ctypes.c_int
        l.a2sgd_decode_update_momentum.argtypes = [_vp, _vp, _i64, _vp, _i64, _vp, _i64, _vp, _i64, _vp, _vp,
                                                   ctypes.c_float, ctypes.c_float, ctypes.c_float, _vp]
        l.a2sgd_step_momentum.restype = ctypes.c_int
        l.a2sgd_step_momentum.argtypes = [_vp, _vp, _i64, _vp, _i64, _vp, _i64, _vp, _i64,
                                          ctypes.c_float, ctypes.c_float, ctypes.c_float, _vp]
        l.a2sgd_global_average_from_sums.restype = ctypes.c_int
        l.a2sgd_global_average_from_sums.argtypes = [_vp, _vp, ctypes.c_uint32, _vp, _vp]
        l.a2sgd_dense_sync_reduced.restype = ctypes.c_int
        l.a2sgd_dense_sync_reduced.argtypes = [_vp, _vp, _vp, ctypes.c_uint32, ctypes.c_float, _vp]
        l.a2sgd_step_host.restype = ctypes.c_int
        l.a2sgd_step_host.argtypes = [_vp, _vp, _i64, _vp, _i64, _vp, _i64, _vp, _i64, ctypes.c_float, _vp, _vp]
        l.a2sgd_read_stats.restype = ctypes.c_int
        l.a2sgd_read_stats.argtypes = [_vp, _vp, _vp, _vp, ctypes.POINTER(ctypes.c_int), _vp]
        l.a2sgd_launch_info.restype = ctypes.c_int
        l.a2sgd_launch_info.argtypes = [_vp, _i64, ctypes.POINTER(ctypes.c_uint32)]
        l.a2sgd_encode_noalloc.restype = ctypes.c_int
        l.a2sgd_encode_noalloc.argtypes = [ctypes.c_uint64, ctypes.c_uint32, ctypes.c_uint32, _vp, _i64, _vp, _i64,
                                           _vp, _vp, _vp]
        l.a2sgd_dense_sync.restype = ctypes.c_int
        l.a2sgd_dense_sync.argtypes = [_vp, _vp, _i64, _vp, _i64, ctypes.c_float, _vp]
        l.a2sgd_segments_create.restype = ctypes.c_int
        l.a2sgd_segments_create.argtypes = [_vp, ctypes.c_uint32, ctypes.POINTER(ctypes.c_uint64),
                                            ctypes.POINTER(_vp), ctypes.POINTER(_vp), ctypes.POINTER(_vp),
                                            ctypes.c_int, ctypes.POINTER(_vp)]
        l.a2sgd_segments_destroy.restype = ctypes.c_int
        l.a2sgd_segments_destroy.argtypes = [_vp]
        l.a2sgd_encode_segments.restype = ctypes.c_int
        l.a2sgd_encode_segments.argtypes = [_vp, _vp, _vp, _vp, _vp]
        l.a2sgd_decode_update_segments.restype = ctypes.c_int
        l.a2sgd_decode_update_segments.argtypes = [_vp, _vp, _vp, _vp, ctypes.c_float, _vp, _vp]
        l.a2sgd_step_segments_per_tensor.restype = ctypes.c_int
        l.a2sgd_step_segments_per_tensor.argtypes = [_vp, _vp, ctypes.c_float, _vp, _vp]
        l.a2sgd_read_segment_stats.restype = ctypes.c_int
        l.a2sgd_read_segment_stats.argtypes = [_vp, _vp, _vp, _vp, _vp, _vp]
        l.a2sgd_step_segments.restype = ctypes.c_int
        l.a2sgd_step_segments.argtypes = [_vp, _vp, ctypes.c_float, _vp]
        for fn in (l.a2sgd_step_bf16, l.a2sgd_step_f16):
            fn.restype = ctypes.c_int
            fn.argtypes = [_vp, _vp, _i64, _vp, _i64, _vp, _i64, ctypes.c_float, _vp]
        l.a2sgd_materialize_err.restype = ctypes.c_int
        l.a2sgd_materialize_err.argtypes = [_vp, _vp, _i64, _vp]
        l.a2sgd_step_segments_lr.restype = ctypes.c_int
        l.a2sgd_step_segments_lr.argtypes = [_vp, _vp, _vp, _vp]
        _dbl, _u64, _u32, _int = ctypes.c_double, ctypes.c_uint64, ctypes.c_uint32, ctypes.c_int
        l.a2sgd_adamw_state_elements.restype = _u64
        l.a2sgd_adamw_state_elements.argtypes = [_u32, ctypes.POINTER(_u64)]
        l.a2sgd_adamw_create.restype = _int
        l.a2sgd_adamw_create.argtypes = [ctypes.POINTER(_vp), _u32, ctypes.POINTER(_u64), ctypes.POINTER(_vp),
                                         ctypes.POINTER(_vp), _int, ctypes.POINTER(_vp), _int, _int, _vp, _vp, _vp,
                                         _vp, _int]
        l.a2sgd_adamw_destroy.restype = _int
        l.a2sgd_adamw_destroy.argtypes = [_vp]
        l.a2sgd_adamw_step.restype = _int
        l.a2sgd_adamw_step.argtypes = [_vp, _dbl, _dbl, _dbl, _dbl, _dbl, _u64, _vp, _vp]
        l.a2sgd_adamw_grad_norm.restype = _int
        l.a2sgd_adamw_grad_norm.argtypes = [_vp, ctypes.c_float, _vp, _vp]
        for fn in (l.a2sgd_adamw_read_state, l.a2sgd_adamw_write_state):
            fn.restype = _int
            fn.argtypes = [_vp, _vp, _vp, _vp]
        l.a2sgd_window_attention_workspace.restype = _u64
        l.a2sgd_window_attention_workspace.argtypes = [_vp, _u32]
        l.a2sgd_window_attention_forward.restype = _int
        l.a2sgd_window_attention_forward.argtypes = [_vp] * 7 + [_u64, _int, _vp]
        l.a2sgd_window_attention_backward.restype = _int
        l.a2sgd_window_attention_backward.argtypes = [_vp] * 11 + [_u64, _int, _vp]
        l.a2sgd_window_attention_status.restype = _int
        l.a2sgd_window_attention_status.argtypes = [_int, ctypes.POINTER(_int), _vp]
        l.a2sgd_rotary.restype = _int
        l.a2sgd_rotary.argtypes = [_vp] * 5 + [_u32, _vp, _dbl, _u32, _u64, _u32, _u32, _u32, _int, _int, _vp]
        l.a2sgd_residual_norm_forward.restype = _int
        l.a2sgd_residual_norm_forward.argtypes = [_vp] * 5 + [_int, _vp]
        l.a2sgd_residual_norm_workspace.restype = _u64
        l.a2sgd_residual_norm_workspace.argtypes = [_u64, _u32, _u64, _int]
        l.a2sgd_residual_norm_backward.restype = _int
        l.a2sgd_residual_norm_backward.argtypes = [_vp] * 9 + [_u64, _int, _vp]
        l.a2sgd_layer_norm_forward.restype = _int
        l.a2sgd_layer_norm_forward.argtypes = [_vp, _i64, _int, _vp, _vp, _int, _vp, _i64, _vp, _vp, _u64, _u32, _dbl,
                                               _int, _vp]
        l.a2sgd_layer_norm_workspace.restype = _u64
        l.a2sgd_layer_norm_workspace.argtypes = [_u64, _u32, _int]
        l.a2sgd_layer_norm_backward.restype = _int
        l.a2sgd_layer_norm_backward.argtypes = [_vp, _i64, _vp, _i64, _int, _vp, _int, _vp, _vp, _vp, _i64, _vp, _vp,
                                                _u64, _u32, _vp, _u64, _int, _vp]
        l.a2sgd_gated_ffn_workspace.restype = _u64
        l.a2sgd_gated_ffn_workspace.argtypes = [_u64, _u32, _u32, _u32]
        l.a2sgd_gated_ffn_forward.restype = _int
        l.a2sgd_gated_ffn_forward.argtypes = [_vp, _i64] * 8 + [_int, _int, _u64, _u32, _u32, _vp, _u64, _int, _vp]
        l.a2sgd_gated_ffn_backward.restype = _int
        l.a2sgd_gated_ffn_backward.argtypes = [_vp, _i64] * 12 + [_int, _int, _u64, _u32, _u32, _vp, _u64, _int, _vp]
        l.a2sgd_gated_ffn_status.restype = _int
        l.a2sgd_gated_ffn_status.argtypes = [_int, ctypes.POINTER(_int), _vp]
        l.a2sgd_status_string.restype = ctypes.c_char_p
        l.a2sgd_status_string.argtypes = [ctypes.c_int]
        _lib = l
    return _lib


def status_string(status: int) -> str:
    return lib().a2sgd_status_string(int(status)).decode()


def _check(status: int, what: str) -> None:
    if status != OK:
        raise A2SGDError(status, what)


def _stream(stream) -> Optional[int]:
    if stream is None:
        stream = torch.cuda.current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _rows(t: Optional[torch.Tensor], name: str) -> Tuple[Optional[int], int]:
    """float32 CUDA [P, n] with unit inner stride -> (address, worker stride in elements)."""
    if t is None:
        return None, 0
    if t.dtype != torch.float32 or not t.is_cuda or t.dim() != 2 or (t.shape[1] > 1 and t.stride(1) != 1):
        raise ValueError(f"{name}: need a float32 CUDA tensor [P, n] with unit inner stride")
    return t.data_ptr(), t.stride(0)


def _weights(w: torch.Tensor) -> Tuple[int, int]:
    if w.dtype != torch.float32 or not w.is_cuda:
        raise ValueError("w: need a float32 CUDA tensor")
    if w.dim() == 1:
        return w.data_ptr(), 0
    if w.dim() == 2:
        return w.data_ptr(), w.stride(0)
    raise ValueError("w: need [n] (shared) or [P, n] (replicated)")


def padded_rows(P: int, n: int, device, fill: Optional[float] = None) -> torch.Tensor:
    """A float32 [P, n] view whose rows start 128-byte aligned (row stride = n rounded up to 32
    elements).  Device memory only; the layout the fast kernels are measured with."""
    stride = (n + ROW_ALIGN_ELEMS - 1) // ROW_ALIGN_ELEMS * ROW_ALIGN_ELEMS
    buf = torch.empty((P, stride), dtype=torch.float32, device=device)
    if fill is not None:
        buf.fill_(fill)
    return buf[:, :n]


class Context:
    """Owns an ``a2sgd_ctx``.  ``n`` elements per worker, ``P`` workers."""

    def __init__(self, n: int, P: int, device: int = 0, flags: int = MODE_EF):
        self.n, self.P, self.device, self.flags = int(n), int(P), int(device), int(flags)
        self._h = _vp()
        _check(lib().a2sgd_create(ctypes.byref(self._h), self.n, self.P, self.device, self.flags), "a2sgd_create")

    @property
    def handle(self):
        if not self._h:
            raise RuntimeError("context destroyed")
        return self._h

    def destroy(self) -> None:
        if self._h:
            lib().a2sgd_destroy(self._h)
            self._h = _vp()

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


def a2sgd_create(n: int, P: int, device: int = 0, flags: int = MODE_EF) -> Context:
    return Context(n, P, device, flags)


def a2sgd_destroy(ctx: Context) -> None:
    ctx.destroy()


def a2sgd_encode(ctx: Context, grad: torch.Tensor, err: Optional[torch.Tensor], local_means: torch.Tensor,
                 pos_counts: Optional[torch.Tensor] = None, pos_mask: Optional[torch.Tensor] = None,
                 stream=None) -> None:
    """local_means: float32 CUDA [P, 2]; pos_counts: int64 CUDA [P]; pos_mask: int32 CUDA [P, ceil(n/32)]."""
    gp, gs = _rows(grad, "grad")
    ep, es = _rows(err, "err")
    _check(lib().a2sgd_encode(ctx.handle, gp, gs, ep, es, local_means.data_ptr(),
                              pos_counts.data_ptr() if pos_counts is not None else None,
                              pos_mask.data_ptr() if pos_mask is not None else None, _stream(stream)),
           "a2sgd_encode")


NOALLOC_MAX_P = 64


def a2sgd_encode_noalloc(grad: torch.Tensor, err: Optional[torch.Tensor], local_means: torch.Tensor,
                         pos_counts: Optional[torch.Tensor] = None, mode: int = MODE_EF, n: Optional[int] = None,
                         stream=None) -> None:
    """Encode without a context and without any allocation inside the library (its scratch is a
    fixed array in the library image).  For callers that may not call cudaMalloc; runs on the
    current device; calls that overlap on the GPU race on the shared scratch.  Output tensors are
    the caller's: local_means float32 CUDA [P, 2], pos_counts int64 CUDA [P]."""
    gp, gs = _rows(grad, "grad")
    ep, es = _rows(err, "err")
    P = grad.shape[0]
    n = grad.shape[1] if n is None else n
    _check(lib().a2sgd_encode_noalloc(int(n), int(P), int(mode), gp, gs, ep, es, local_means.data_ptr(),
                                      pos_counts.data_ptr() if pos_counts is not None else None,
                                      _stream(stream)), "a2sgd_encode_noalloc")


def a2sgd_global_average(ctx: Context, local_means: torch.Tensor, global_means: torch.Tensor, stream=None) -> None:
    _check(lib().a2sgd_global_average(ctx.handle, local_means.data_ptr(), global_means.data_ptr(), _stream(stream)),
           "a2sgd_global_average")


def a2sgd_global_average_from_sums(ctx: Context, sums: torch.Tensor, workers: int, global_means: torch.Tensor,
                                   stream=None) -> None:
    """sums: float64 CUDA [2], the all-reduced sums of the two local means over ``workers`` workers."""
    if sums.dtype != torch.float64 or not sums.is_cuda or sums.numel() < 2:
        raise ValueError("sums: need a float64 CUDA tensor of 2 elements")
    _check(lib().a2sgd_global_average_from_sums(ctx.handle, sums.data_ptr(), int(workers), global_means.data_ptr(),
                                                _stream(stream)), "a2sgd_global_average_from_sums")


def a2sgd_dense_sync_reduced(ctx: Context, w: torch.Tensor, grad_sum: torch.Tensor, workers: int, lr: float,
                             stream=None) -> None:
    """grad_sum: float32 CUDA [n], the all-reduced sum of the workers' gradients."""
    if grad_sum.dtype != torch.float32 or not grad_sum.is_cuda or not grad_sum.is_contiguous():
        raise ValueError("grad_sum: need a contiguous float32 CUDA tensor")
    wp, _ = _weights(w)
    _check(lib().a2sgd_dense_sync_reduced(ctx.handle, wp, grad_sum.data_ptr(), int(workers), float(lr),
                                          _stream(stream)), "a2sgd_dense_sync_reduced")


def a2sgd_decode_update(ctx: Context, w: torch.Tensor, grad: torch.Tensor, err: Optional[torch.Tensor],
                        local_means: Optional[torch.Tensor], global_means: torch.Tensor, lr: float,
                        stream=None) -> None:
    wp, ws = _weights(w)
    gp, gs = _rows(grad, "grad")
    ep, es = _rows(err, "err")
    _check(lib().a2sgd_decode_update(ctx.handle, wp, ws, gp, gs, ep, es,
                                     local_means.data_ptr() if local_means is not None else None,
                                     global_means.data_ptr(), float(lr), _stream(stream)),
           "a2sgd_decode_update")


def a2sgd_step(ctx: Context, w: torch.Tensor, grad: torch.Tensor, err: Optional[torch.Tensor], lr: float,
               stream=None) -> None:
    wp, ws = _weights(w)
    gp, gs = _rows(grad, "grad")
    ep, es = _rows(err, "err")
    _check(lib().a2sgd_step(ctx.handle, wp, ws, gp, gs, ep, es, float(lr), _stream(stream)), "a2sgd_step")


def a2sgd_decode_update_momentum(ctx: Context, w: torch.Tensor, mom: torch.Tensor, grad: torch.Tensor,
                                 err: Optional[torch.Tensor], local_means: Optional[torch.Tensor],
                                 global_means: torch.Tensor, lr: float, beta: float, weight_decay: float,
                                 stream=None) -> None:
    """mom: float32 CUDA tensor with the layout of w (zero before the first step)."""
    wp, ws = _weights(w)
    mp, ms = _weights(mom)
    gp, gs = _rows(grad, "grad")
    ep, es = _rows(err, "err")
    _check(lib().a2sgd_decode_update_momentum(ctx.handle, wp, ws, mp, ms, gp, gs, ep, es,
                                              local_means.data_ptr() if local_means is not None else None,
                                              global_means.data_ptr(), float(lr), float(beta), float(weight_decay),
                                              _stream(stream)), "a2sgd_decode_update_momentum")


def a2sgd_step_momentum(ctx: Context, w: torch.Tensor, mom: torch.Tensor, grad: torch.Tensor,
                        err: Optional[torch.Tensor], lr: float, beta: float, weight_decay: float, stream=None) -> None:
    wp, ws = _weights(w)
    mp, ms = _weights(mom)
    gp, gs = _rows(grad, "grad")
    ep, es = _rows(err, "err")
    _check(lib().a2sgd_step_momentum(ctx.handle, wp, ws, mp, ms, gp, gs, ep, es, float(lr), float(beta),
                                     float(weight_decay), _stream(stream)), "a2sgd_step_momentum")


def a2sgd_step_bf16(ctx: Context, w: torch.Tensor, grad: torch.Tensor, err: Optional[torch.Tensor], lr: float,
                    stream=None) -> None:
    """a2sgd_step with bfloat16 gradients: grad is a torch.bfloat16 CUDA tensor [P, >= n]."""
    if grad.dtype != torch.bfloat16 or not grad.is_cuda or grad.dim() != 2 or (grad.shape[1] > 1 and grad.stride(1) != 1):
        raise ValueError("grad: need a bfloat16 CUDA tensor [P, n] with unit inner stride")
    wp, ws = _weights(w)
    ep, es = _rows(err, "err")
    _check(lib().a2sgd_step_bf16(ctx.handle, wp, ws, grad.data_ptr(), grad.stride(0), ep, es, float(lr),
                                 _stream(stream)), "a2sgd_step_bf16")


def a2sgd_materialize_err(ctx: Context, err: torch.Tensor, stream=None) -> None:
    """Deferred-residual contexts: turn the buffer (holding v) back into the true residual, in place."""
    ep, es = _rows(err, "err")
    _check(lib().a2sgd_materialize_err(ctx.handle, ep, es, _stream(stream)), "a2sgd_materialize_err")


def a2sgd_step_f16(ctx: Context, w: torch.Tensor, grad: torch.Tensor, err: Optional[torch.Tensor], lr: float,
                   stream=None) -> None:
    """a2sgd_step with half-precision gradients: grad is a torch.float16 CUDA tensor [P, >= n]."""
    if grad.dtype != torch.float16 or not grad.is_cuda or grad.dim() != 2 or (grad.shape[1] > 1 and grad.stride(1) != 1):
        raise ValueError("grad: need a float16 CUDA tensor [P, n] with unit inner stride")
    wp, ws = _weights(w)
    ep, es = _rows(err, "err")
    _check(lib().a2sgd_step_f16(ctx.handle, wp, ws, grad.data_ptr(), grad.stride(0), ep, es, float(lr),
                                _stream(stream)), "a2sgd_step_f16")


def a2sgd_dense_sync(ctx: Context, w: torch.Tensor, grad: torch.Tensor, lr: float, stream=None) -> None:
    """Algorithm 1 lines 9-10: w <- w - lr * mean over workers of grad."""
    wp, ws = _weights(w)
    gp, gs = _rows(grad, "grad")
    _check(lib().a2sgd_dense_sync(ctx.handle, wp, ws, gp, gs, float(lr), _stream(stream)), "a2sgd_dense_sync")


class Segments:
    """Owns an ``a2sgd_segments`` plan and keeps the tensors it points at alive."""

    def __init__(self, ctx: Context, grad, err, w, w_replicated: bool):
        self.ctx = ctx
        self._keep = (grad, err, w)
        P, S = ctx.P, len(grad[0])
        numel = (ctypes.c_uint64 * S)(*[t.numel() for t in grad[0]])

        def table(rows):
            flat = [t for row in rows for t in row]
            for t in flat:
                if t.dtype != torch.float32 or not t.is_cuda or not t.is_contiguous():
                    raise ValueError("segments: need contiguous float32 CUDA tensors")
            return (_vp * len(flat))(*[t.data_ptr() for t in flat])

        if len(grad) != P or any(len(r) != S for r in grad):
            raise ValueError("grad: need P lists of S tensors")
        g_tab = table(grad)
        e_tab = table(err) if err is not None else None
        w_tab = table(w if w_replicated else [w])
        self._h = _vp()
        _check(lib().a2sgd_segments_create(ctx.handle, S, numel, g_tab, e_tab, w_tab, 1 if w_replicated else 0,
                                           ctypes.byref(self._h)), "a2sgd_segments_create")

    @property
    def handle(self):
        if not self._h:
            raise RuntimeError("segment plan destroyed")
        return self._h

    def destroy(self) -> None:
        if self._h:
            lib().a2sgd_segments_destroy(self._h)
            self._h = _vp()

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


def a2sgd_segments_create(ctx: Context, grad, err, w, w_replicated: bool = False) -> Segments:
    """grad / err: P lists of S tensors (err None in ALG1 mode when eps is not wanted);
    w: a list of S tensors (shared) or P lists of S tensors (replicated)."""
    return Segments(ctx, grad, err, w, w_replicated)


def a2sgd_segments_destroy(plan: Segments) -> None:
    plan.destroy()


def a2sgd_step_segments(ctx: Context, plan: Segments, lr: float, stream=None) -> None:
    _check(lib().a2sgd_step_segments(ctx.handle, plan.handle, float(lr), _stream(stream)), "a2sgd_step_segments")


def a2sgd_encode_segments(ctx: Context, plan: Segments, local_means: torch.Tensor,
                          pos_counts: Optional[torch.Tensor] = None, stream=None) -> None:
    _check(lib().a2sgd_encode_segments(ctx.handle, plan.handle, local_means.data_ptr(),
                                       pos_counts.data_ptr() if pos_counts is not None else None, _stream(stream)),
           "a2sgd_encode_segments")


def a2sgd_decode_update_segments(ctx: Context, plan: Segments, local_means: Optional[torch.Tensor],
                                 global_means: torch.Tensor, lr: float,
                                 lr_per_segment: Optional[torch.Tensor] = None, stream=None) -> None:
    _check(lib().a2sgd_decode_update_segments(ctx.handle, plan.handle,
                                              local_means.data_ptr() if local_means is not None else None,
                                              global_means.data_ptr(), float(lr),
                                              lr_per_segment.data_ptr() if lr_per_segment is not None else None,
                                              _stream(stream)), "a2sgd_decode_update_segments")


def a2sgd_step_segments_per_tensor(ctx: Context, plan: Segments, lr: float,
                                   lr_per_segment: Optional[torch.Tensor] = None, stream=None) -> None:
    """Every tensor compressed on its own (its own local and global means)."""
    _check(lib().a2sgd_step_segments_per_tensor(ctx.handle, plan.handle, float(lr),
                                                lr_per_segment.data_ptr() if lr_per_segment is not None else None,
                                                _stream(stream)), "a2sgd_step_segments_per_tensor")


def a2sgd_read_segment_stats(ctx: Context, plan: Segments, S: int, stream=None):
    """Synchronises the stream.  Returns (local_means [S,P,2], global_means [S,2], pos_counts [S,P])."""
    import numpy as np
    lm = np.zeros((S, ctx.P, 2), np.float32)
    gm = np.zeros((S, 2), np.float32)
    pc = np.zeros((S, ctx.P), np.uint64)
    _check(lib().a2sgd_read_segment_stats(ctx.handle, plan.handle, lm.ctypes.data, gm.ctypes.data, pc.ctypes.data,
                                          _stream(stream)), "a2sgd_read_segment_stats")
    return lm, gm, pc


def a2sgd_step_segments_lr(ctx: Context, plan: Segments, lr_per_segment: torch.Tensor, stream=None) -> None:
    """lr_per_segment: float32 CUDA tensor of S learning rates (layer-wise policies such as LARS)."""
    if lr_per_segment.dtype != torch.float32 or not lr_per_segment.is_cuda or not lr_per_segment.is_contiguous():
        raise ValueError("lr_per_segment: need a contiguous float32 CUDA tensor")
    _check(lib().a2sgd_step_segments_lr(ctx.handle, plan.handle, lr_per_segment.data_ptr(), _stream(stream)),
           "a2sgd_step_segments_lr")


def a2sgd_step_host(ctx: Context, w: torch.Tensor, grad_host: torch.Tensor, grad_staging: torch.Tensor,
                    err: Optional[torch.Tensor], lr: float, means_host: torch.Tensor, stream=None) -> None:
    """grad_host: float32 CPU [P, >= n] (pinned for asynchronous copies); means_host: float32 CPU [2P + 2]."""
    if grad_host.is_cuda or grad_host.dtype != torch.float32 or grad_host.dim() != 2 or grad_host.stride(1) != 1:
        raise ValueError("grad_host: need a float32 CPU tensor [P, n] with unit inner stride")
    if means_host.is_cuda or means_host.dtype != torch.float32 or means_host.numel() < 2 * ctx.P + 2:
        raise ValueError("means_host: need a float32 CPU tensor of 2P + 2 elements")
    wp, ws = _weights(w)
    sp, ss = _rows(grad_staging, "grad_staging")
    ep, es = _rows(err, "err")
    _check(lib().a2sgd_step_host(ctx.handle, wp, ws, grad_host.data_ptr(), grad_host.stride(0), sp, ss, ep, es,
                                 float(lr), means_host.data_ptr(), _stream(stream)), "a2sgd_step_host")


def a2sgd_read_stats(ctx: Context, stream=None):
    """Synchronises the stream.  Returns (local_means [P,2], global_means [2], pos_counts [P], device_status)."""
    import numpy as np
    lm = np.zeros((ctx.P, 2), np.float32)
    gm = np.zeros(2, np.float32)
    pc = np.zeros(ctx.P, np.uint64)
    st = ctypes.c_int(0)
    _check(lib().a2sgd_read_stats(ctx.handle, lm.ctypes.data, gm.ctypes.data, pc.ctypes.data, ctypes.byref(st),
                                  _stream(stream)), "a2sgd_read_stats")
    return lm, gm, pc, st.value


def a2sgd_launch_info(ctx: Context, shared_w: bool = True) -> dict:
    out = (ctypes.c_uint32 * 5)()
    _check(lib().a2sgd_launch_info(ctx.handle, 0 if shared_w else ctx.n, out), "a2sgd_launch_info")
    return {"encode_ctas": out[0], "decode_ctas": out[1], "threads": out[2], "single_launch": bool(out[3]),
            "sms": out[4]}


# ---------------------------------------------------------------------------------------------
# Training operators (AdamW over a list of tensors, layer norm, gated feed-forward block): see the
# section of that name in include/a2sgd.h.  Argument checks and marshalling only, as above.

F32, BF16, F16 = 0, 1, 2
ADAMW_BLOCK = 256
_DTYPE_CODES = {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}


def _dtype_code(t: torch.Tensor, name: str) -> int:
    code = _DTYPE_CODES.get(t.dtype)
    if code is None:
        raise ValueError(f"{name}: need float32, bfloat16 or float16, got {t.dtype}")
    return code


# The calls below are short enough for the host's share to count (a layer norm of few rows takes less time on the
# device than its launch): one pass over each tensor's properties, devices as indices.

def _matrix(t: torch.Tensor, name: str, shape, dtype: torch.dtype, index: int) -> Tuple[int, int]:
    """CUDA [rows, columns] with unit inner stride -> (address, row stride in elements)."""
    if t.dtype is not dtype or t.get_device() != index or t.shape != shape:
        raise ValueError(f"{name}: need a {dtype} tensor {list(shape)} on cuda:{index}, got {t.dtype} {list(t.shape)} on {t.device}")
    stride, inner = t.stride()
    if inner != 1 and shape[1] > 1:
        raise ValueError(f"{name}: need unit inner stride")
    return t.data_ptr(), stride


def _vector(t: Optional[torch.Tensor], name: str, numel: int, dtype, index: int) -> Optional[int]:
    """A contiguous CUDA tensor of ``numel`` elements (or None) -> address."""
    if t is None:
        return None
    if t.dtype is not dtype or t.get_device() != index or t.numel() != numel or not t.is_contiguous():
        raise ValueError(f"{name}: need a contiguous tensor of {numel} elements of {dtype} on cuda:{index}, got {t.dtype} "
                         f"{list(t.shape)} on {t.device}")
    return t.data_ptr()


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)   # torch.cuda.current_stream without its wrapper: 0.1 us


def _stream_on(index: int, stream) -> int:
    if stream is None:
        return _raw_stream(index) if _raw_stream is not None else torch.cuda.current_stream(index).cuda_stream
    return _stream(stream)


def _cuda_index(t: torch.Tensor, name: str) -> int:
    if not t.is_cuda:
        raise ValueError(f"{name}: need a CUDA tensor")
    return t.get_device()


def a2sgd_adamw_state_elements(params) -> int:
    """Elements of the m and the v buffer for tensors (or element counts): each tensor starts at a multiple of 256."""
    numel = [int(p.numel()) if torch.is_tensor(p) else int(p) for p in params]
    return int(lib().a2sgd_adamw_state_elements(len(numel), (ctypes.c_uint64 * len(numel))(*numel)))


class AdamW:
    """Owns an ``a2sgd_adamw`` plan and keeps the tensors it points at alive."""

    def __init__(self, params, grads, m, v, m_scale=None, v_scale=None, w16=None):
        params, grads = list(params), list(grads)
        S = len(params)
        if S == 0 or len(grads) != S or (w16 is not None and len(w16) != S):
            raise ValueError("params, grads and w16: need lists of the same length, at least 1")
        self.device = _cuda_index(params[0], "params")

        def table(tensors, name, dtype):
            for t, p in zip(tensors, params):
                if t.dtype != dtype or t.get_device() != self.device or not t.is_contiguous() or t.numel() != p.numel():
                    raise ValueError(f"{name}: need contiguous {dtype} tensors on cuda:{self.device}, as long as the parameters")
            return (_vp * S)(*[t.data_ptr() for t in tensors])

        w_tab = table(params, "params", torch.float32)
        g_code = _dtype_code(grads[0], "grads")
        g_tab = table(grads, "grads", grads[0].dtype)
        w16_tab, w16_code = None, F32
        if w16 is not None:
            w16 = list(w16)
            w16_code = _dtype_code(w16[0], "w16")
            w16_tab = table(w16, "w16", w16[0].dtype)
        self.state_elements = n = a2sgd_adamw_state_elements(params)
        self.state_bits = 32 if m.dtype == torch.float32 else 8
        m_type, v_type = (torch.float32, torch.float32) if self.state_bits == 32 else (torch.int8, torch.uint8)
        scales = None if self.state_bits == 32 else n // ADAMW_BLOCK
        if (scales is None) != (m_scale is None) or (scales is None) != (v_scale is None):
            raise ValueError("m_scale, v_scale: needed with 8-bit states, and only there")
        m_ptr = _vector(m, "m", n, m_type, self.device)
        v_ptr = _vector(v, "v", n, v_type, self.device)
        ms_ptr = _vector(m_scale, "m_scale", scales, torch.float32, self.device)
        vs_ptr = _vector(v_scale, "v_scale", scales, torch.float32, self.device)
        self._keep = (params, grads, m, v, m_scale, v_scale, w16)
        numel = (ctypes.c_uint64 * S)(*[p.numel() for p in params])
        self._h = _vp()
        _check(lib().a2sgd_adamw_create(ctypes.byref(self._h), S, numel, w_tab, g_tab, g_code, w16_tab, w16_code,
                                        self.state_bits, m_ptr, v_ptr, ms_ptr, vs_ptr, self.device),
               "a2sgd_adamw_create")

    @property
    def handle(self):
        if not self._h:
            raise RuntimeError("AdamW plan destroyed")
        return self._h

    def destroy(self) -> None:
        if self._h:
            lib().a2sgd_adamw_destroy(self._h)
            self._h = _vp()

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


def a2sgd_adamw_create(params, grads, m: torch.Tensor, v: torch.Tensor, m_scale: Optional[torch.Tensor] = None,
                       v_scale: Optional[torch.Tensor] = None, w16=None) -> AdamW:
    """params: float32 CUDA tensors; grads: as many of one type; w16: 16-bit tensors that receive copies, or None.
    m, v: flat state of a2sgd_adamw_state_elements(params) elements, float32, or int8 and uint8 with one float32
    scale for each 256 (m_scale, v_scale); zero them before the first step."""
    return AdamW(params, grads, m, v, m_scale, v_scale, w16)


def a2sgd_adamw_destroy(plan: AdamW) -> None:
    plan.destroy()


def a2sgd_adamw_step(plan: AdamW, lr: float, step: int, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8,
                     weight_decay: float = 0.0, grad_scale: Optional[torch.Tensor] = None, stream=None) -> None:
    """grad_scale: float32 CUDA tensor of one element, a factor on every gradient; not finite: nothing changes."""
    gs = _vector(grad_scale, "grad_scale", 1, torch.float32, plan.device)
    if step < 1:
        raise ValueError("step: counted from 1")
    _check(lib().a2sgd_adamw_step(plan.handle, lr, beta1, beta2, eps, weight_decay, step, gs,
                                  _stream_on(plan.device, stream)), "a2sgd_adamw_step")


def a2sgd_adamw_grad_norm(plan: AdamW, max_norm: float, norm_and_scale: torch.Tensor, stream=None) -> None:
    """norm_and_scale: float32 CUDA [2], out: the norm of all gradients, and min(1, max_norm / norm)."""
    out = _vector(norm_and_scale, "norm_and_scale", 2, torch.float32, plan.device)
    _check(lib().a2sgd_adamw_grad_norm(plan.handle, max_norm, out, _stream_on(plan.device, stream)),
           "a2sgd_adamw_grad_norm")


def a2sgd_adamw_read_state(plan: AdamW, m_out: Optional[torch.Tensor], v_out: Optional[torch.Tensor], stream=None) -> None:
    """m_out, v_out: float32 CUDA tensors of plan.state_elements (either may be None)."""
    _check(lib().a2sgd_adamw_read_state(plan.handle, _vector(m_out, "m_out", plan.state_elements, torch.float32, plan.device),
                                        _vector(v_out, "v_out", plan.state_elements, torch.float32, plan.device),
                                        _stream_on(plan.device, stream)), "a2sgd_adamw_read_state")


def a2sgd_adamw_write_state(plan: AdamW, m_in: torch.Tensor, v_in: torch.Tensor, stream=None) -> None:
    _check(lib().a2sgd_adamw_write_state(plan.handle, _vector(m_in, "m_in", plan.state_elements, torch.float32, plan.device),
                                         _vector(v_in, "v_in", plan.state_elements, torch.float32, plan.device),
                                         _stream_on(plan.device, stream)), "a2sgd_adamw_write_state")


def _param_dtype(x: torch.Tensor, *vectors) -> torch.dtype:
    for v in vectors:
        if v is not None:
            return v.dtype
    return x.dtype


def a2sgd_layer_norm_forward(x: torch.Tensor, weight: Optional[torch.Tensor], bias: Optional[torch.Tensor],
                             y: torch.Tensor, mean: Optional[torch.Tensor], rstd: Optional[torch.Tensor],
                             eps: float = 1e-5, stream=None) -> None:
    """x, y: CUDA [rows, d], unit inner stride (y may be x); weight, bias: [d] of float32 or x's type, or None;
    mean, rstd: float32 [rows], out, or None."""
    dev, code = _cuda_index(x, "x"), _dtype_code(x, "x")
    if x.dim() != 2:
        raise ValueError("x: need [rows, d]")
    shape = rows, d = x.shape
    pt = _param_dtype(x, weight, bias)
    xp, xs = _matrix(x, "x", shape, x.dtype, dev)
    yp, ys = _matrix(y, "y", shape, x.dtype, dev)
    _check(lib().a2sgd_layer_norm_forward(
        xp, xs, code, _vector(weight, "weight", d, pt, dev), _vector(bias, "bias", d, pt, dev),
        _DTYPE_CODES.get(pt, -1), yp, ys, _vector(mean, "mean", rows, torch.float32, dev),
        _vector(rstd, "rstd", rows, torch.float32, dev), rows, d, eps, dev, _stream_on(dev, stream)),
        "a2sgd_layer_norm_forward")


def a2sgd_layer_norm_workspace(rows: int, d: int, device: Optional[int] = None) -> int:
    """Bytes of workspace of a2sgd_layer_norm_backward."""
    device = torch.cuda.current_device() if device is None else int(device)
    return int(lib().a2sgd_layer_norm_workspace(int(rows), int(d), device))


def a2sgd_layer_norm_backward(dy: torch.Tensor, x: torch.Tensor, weight: Optional[torch.Tensor], mean: torch.Tensor,
                              rstd: torch.Tensor, dx: Optional[torch.Tensor], dweight: Optional[torch.Tensor],
                              dbias: Optional[torch.Tensor], workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    """dx (may be dy or x), dweight, dbias: out, each may be None; workspace: uint8 CUDA tensor of
    a2sgd_layer_norm_workspace bytes, needed for dweight or dbias."""
    dev, code = _cuda_index(x, "x"), _dtype_code(x, "x")
    if x.dim() != 2:
        raise ValueError("x: need [rows, d]")
    shape = rows, d = x.shape
    pt = _param_dtype(x, weight, dweight, dbias)
    xp, xs = _matrix(x, "x", shape, x.dtype, dev)
    gp, gs = _matrix(dy, "dy", shape, x.dtype, dev)
    op, os_ = (None, 0) if dx is None else _matrix(dx, "dx", shape, x.dtype, dev)
    wb = 0 if workspace is None else workspace.numel()
    _check(lib().a2sgd_layer_norm_backward(
        gp, gs, xp, xs, code, _vector(weight, "weight", d, pt, dev), _DTYPE_CODES.get(pt, -1),
        _vector(mean, "mean", rows, torch.float32, dev), _vector(rstd, "rstd", rows, torch.float32, dev), op, os_,
        _vector(dweight, "dweight", d, pt, dev), _vector(dbias, "dbias", d, pt, dev), rows, d,
        _vector(workspace, "workspace", wb, torch.uint8, dev), wb, dev, _stream_on(dev, stream)),
        "a2sgd_layer_norm_backward")


FFN_BACKWARD, FFN_ALIGNED = 1, 2
_ACTIVATIONS = {"silu": 0, "gelu_tanh": 1}


def a2sgd_gated_ffn_workspace(tokens: int, d: int, f: int, backward: bool = False, aligned: bool = False) -> int:
    """Bytes of workspace of a2sgd_gated_ffn_forward (or _backward).  aligned: every matrix that is read, and hidden,
    starts at a multiple of 16 bytes with a row stride that is a multiple of 8 elements."""
    flags = (FFN_BACKWARD if backward else 0) | (FFN_ALIGNED if aligned else 0)
    return int(lib().a2sgd_gated_ffn_workspace(int(tokens), int(d), int(f), flags))


def _ffn_sizes(x: torch.Tensor, w_gate: torch.Tensor, activation: str):
    dev = _cuda_index(x, "x")
    if x.dtype is not torch.bfloat16 and x.dtype is not torch.float16:
        raise ValueError(f"x: need bfloat16 or float16, got {x.dtype}")
    if x.dim() != 2 or w_gate.dim() != 2:
        raise ValueError("x, w_gate: need matrices")
    if activation not in _ACTIVATIONS:
        raise ValueError(f"activation: need one of {sorted(_ACTIVATIONS)}, got {activation!r}")
    return dev, x.dtype, x.shape[0], x.shape[1], w_gate.shape[0]


def _optional_matrix(t, name, shape, dtype, dev):
    return (None, 0) if t is None else _matrix(t, name, shape, dtype, dev)


def a2sgd_gated_ffn_forward(x: torch.Tensor, w_gate: torch.Tensor, w_up: torch.Tensor, w_down: torch.Tensor,
                            y: torch.Tensor, hidden: torch.Tensor, gate: Optional[torch.Tensor] = None,
                            up: Optional[torch.Tensor] = None, activation: str = "silu",
                            workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    """x, y: [tokens, d]; w_gate, w_up: [f, d]; w_down: [d, f]; hidden, gate, up: [tokens, f], out (gate and up, for the
    backward pass, may both be None).  One 16-bit type, unit inner stride.  workspace: uint8 CUDA tensor of
    a2sgd_gated_ffn_workspace bytes."""
    dev, dt, t, d, f = _ffn_sizes(x, w_gate, activation)
    wb = 0 if workspace is None else workspace.numel()
    _check(lib().a2sgd_gated_ffn_forward(
        *_matrix(x, "x", (t, d), dt, dev), *_matrix(w_gate, "w_gate", (f, d), dt, dev),
        *_matrix(w_up, "w_up", (f, d), dt, dev), *_matrix(w_down, "w_down", (d, f), dt, dev),
        *_matrix(y, "y", (t, d), dt, dev), *_matrix(hidden, "hidden", (t, f), dt, dev),
        *_optional_matrix(gate, "gate", (t, f), dt, dev), *_optional_matrix(up, "up", (t, f), dt, dev),
        _DTYPE_CODES[dt], _ACTIVATIONS[activation], t, d, f, _vector(workspace, "workspace", wb, torch.uint8, dev), wb,
        dev, _stream_on(dev, stream)), "a2sgd_gated_ffn_forward")


def a2sgd_gated_ffn_backward(dy: torch.Tensor, x: torch.Tensor, w_gate: torch.Tensor, w_up: torch.Tensor,
                             w_down: torch.Tensor, hidden: torch.Tensor, gate: torch.Tensor, up: torch.Tensor,
                             dx: Optional[torch.Tensor], dw_gate: Optional[torch.Tensor], dw_up: Optional[torch.Tensor],
                             dw_down: Optional[torch.Tensor], activation: str = "silu",
                             workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    """dy: [tokens, d]; hidden, gate, up: what the forward pass left; dx [tokens, d], dw_gate, dw_up [f, d], dw_down [d, f]:
    out, each may be None; workspace: uint8 CUDA tensor of a2sgd_gated_ffn_workspace(..., backward=True) bytes."""
    dev, dt, t, d, f = _ffn_sizes(x, w_gate, activation)
    wb = 0 if workspace is None else workspace.numel()
    _check(lib().a2sgd_gated_ffn_backward(
        *_matrix(dy, "dy", (t, d), dt, dev), *_matrix(x, "x", (t, d), dt, dev),
        *_matrix(w_gate, "w_gate", (f, d), dt, dev), *_matrix(w_up, "w_up", (f, d), dt, dev),
        *_matrix(w_down, "w_down", (d, f), dt, dev), *_matrix(hidden, "hidden", (t, f), dt, dev),
        *_matrix(gate, "gate", (t, f), dt, dev), *_matrix(up, "up", (t, f), dt, dev),
        *_optional_matrix(dx, "dx", (t, d), dt, dev), *_optional_matrix(dw_gate, "dw_gate", (f, d), dt, dev),
        *_optional_matrix(dw_up, "dw_up", (f, d), dt, dev), *_optional_matrix(dw_down, "dw_down", (d, f), dt, dev),
        _DTYPE_CODES[dt], _ACTIVATIONS[activation], t, d, f, _vector(workspace, "workspace", wb, torch.uint8, dev), wb,
        dev, _stream_on(dev, stream)), "a2sgd_gated_ffn_backward")


def a2sgd_gated_ffn_status(device: Optional[int] = None, stream=None) -> int:
    """Synchronises the stream; ERR_TIMEOUT if a wait inside one of the block's kernels has run out on the device since this
    was last asked with the same stream, else OK."""
    device = torch.cuda.current_device() if device is None else int(device)
    st = ctypes.c_int(0)
    _check(lib().a2sgd_gated_ffn_status(device, ctypes.byref(st), _stream_on(device, stream)),
           "a2sgd_gated_ffn_status")
    return st.value


# ---- the attention half of a block: attention, rotary positions, the residual connection with its norms

ATTENTION_BACKWARD, ATTENTION_ALIGNED, ATTENTION_PACKED_Q, ATTENTION_PACKED_K = 1, 2, 4, 8
ROTARY_INTERLEAVED, ROTARY_LADDER_PER_AXIS, ROTARY_INVERSE = 1, 2, 4
RESIDUAL_RMS, RESIDUAL_POST_NORM = 1, 2
NO_WINDOW = 1 << 31


class _AttentionShape(ctypes.Structure):
    _fields_ = [("sequences", ctypes.c_uint32), ("q_heads", ctypes.c_uint32), ("kv_heads", ctypes.c_uint32),
                ("head_dim", ctypes.c_uint32), ("q_rows", ctypes.c_uint64), ("k_rows", ctypes.c_uint64), ("q_ranges", _vp),
                ("k_ranges", _vp), ("window", ctypes.c_uint64), ("sinks", ctypes.c_uint32), ("dtype", ctypes.c_int32),
                ("scale", ctypes.c_double)]


class _ResidualShape(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_uint64), ("gate_rows", ctypes.c_uint64), ("d", ctypes.c_uint32), ("flags", ctypes.c_uint32),
                ("dtype", ctypes.c_int32), ("residual_dtype", ctypes.c_int32), ("param_dtype", ctypes.c_int32),
                ("reserved", ctypes.c_int32), ("alpha", ctypes.c_double), ("eps", ctypes.c_double)] \
        + [(name, _vp) for name in ("post_weight", "post_bias", "gate", "pre_weight", "pre_bias", "post_mean", "post_rstd",
                                    "pre_mean", "pre_rstd")]


# a2sgd_heads and a2sgd_rows as bytes, which ctypes passes by address: a quarter of what an array of its own costs
_pack_heads = struct.Struct("4q").pack
_pack_rows = struct.Struct("2q").pack


def _heads(t: torch.Tensor, name: str, shape, dtype: torch.dtype, index: int) -> bytes:
    """CUDA [sequences, rows, heads, head_dim], or [rows, heads, head_dim] of packed sequences, unit inner stride ->
    address, sequence stride, row stride, head stride."""
    if t.dtype is not dtype or t.get_device() != index or t.shape != shape:
        raise ValueError(f"{name}: need a {dtype} tensor {list(shape)} on cuda:{index}, got {t.dtype} {list(t.shape)} on {t.device}")
    stride = t.stride()
    if stride[-1] != 1 and shape[-1] > 1:
        raise ValueError(f"{name}: need unit inner stride")
    if len(shape) == 3:
        return _pack_heads(t.data_ptr(), 0, stride[0], stride[1])
    return _pack_heads(t.data_ptr(), stride[0], stride[1], stride[2])


def _ranges(t: Optional[torch.Tensor], name: str, sequences: int, index: int) -> Optional[int]:
    if t is None:
        return None
    if t.dtype is not torch.int32 or t.get_device() != index or t.shape != (sequences, 2) or not t.is_contiguous():
        raise ValueError(f"{name}: need a contiguous int32 tensor [{sequences}, 2] on cuda:{index}, got {t.dtype} {list(t.shape)} on {t.device}")
    return t.data_ptr()


def _attention_shape(q, k, window, sinks, scale, q_ranges, k_ranges):
    dev = _cuda_index(q, "q")
    if q.dtype is not torch.bfloat16 and q.dtype is not torch.float16:
        raise ValueError(f"q: need bfloat16 or float16, got {q.dtype}")
    if q.dim() not in (3, 4) or k.dim() not in (3, 4):
        raise ValueError("q, k: need [sequences, rows, heads, head_dim], or [rows, heads, head_dim] of packed sequences")
    sequences = None
    for t, ranges, name in ((q, q_ranges, "q"), (k, k_ranges, "k")):
        if t.dim() == 3 and ranges is None:
            raise ValueError(f"{name}: packed sequences need {name}_ranges")
        n = t.shape[0] if t.dim() == 4 else ranges.shape[0]
        if sequences is not None and n != sequences:
            raise ValueError(f"q, k: {sequences} and {n} sequences")
        sequences = n
    if q.shape[-1] != k.shape[-1]:
        raise ValueError("q, k: head_dim differs")
    window = NO_WINDOW if window is None else int(window)
    if window < 1 or sinks < 0:
        raise ValueError("window: at least 1 (None: all keys up to the query's own place); sinks: at least 0")
    d = q.shape[-1]
    shape = _AttentionShape(sequences, q.shape[-2], k.shape[-2], d, q.shape[-3], k.shape[-3], _ranges(q_ranges, "q_ranges", sequences, dev),
                            _ranges(k_ranges, "k_ranges", sequences, dev), window, min(int(sinks), NO_WINDOW), _DTYPE_CODES[q.dtype],
                            d ** -0.5 if scale is None else scale)
    return dev, shape


def _lse(t, q, dev):
    if t is None:
        return None
    want = (q.shape[1], q.shape[0]) if q.dim() == 3 else (q.shape[0], q.shape[2], q.shape[1])
    if t.shape != want:
        raise ValueError(f"lse: need {list(want)}, got {list(t.shape)}")
    return _vector(t, "lse", t.numel(), torch.float32, dev)


def a2sgd_window_attention_workspace(q: torch.Tensor, k: torch.Tensor, window: Optional[int], sinks: int, sequences: int,
                                     backward: bool = False, aligned: bool = False) -> int:
    """Bytes of workspace of a2sgd_window_attention_forward (or _backward).  aligned: every tensor that is read starts at a multiple
    of 16 bytes and has strides that are multiples of 8 elements."""
    shape = _AttentionShape(int(sequences), q.shape[-2], k.shape[-2], q.shape[-1], q.shape[-3], k.shape[-3], None, None,
                            NO_WINDOW if window is None else int(window), min(int(sinks), NO_WINDOW), _DTYPE_CODES.get(q.dtype, -1), 1.0)
    flags = (ATTENTION_BACKWARD if backward else 0) | (ATTENTION_ALIGNED if aligned else 0) \
        | (ATTENTION_PACKED_Q if q.dim() == 3 else 0) | (ATTENTION_PACKED_K if k.dim() == 3 else 0)
    return int(lib().a2sgd_window_attention_workspace(ctypes.addressof(shape), flags))


def a2sgd_window_attention_forward(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, o: torch.Tensor,
                                   lse: Optional[torch.Tensor] = None, window: Optional[int] = None, sinks: int = 0,
                                   scale: Optional[float] = None, q_ranges: Optional[torch.Tensor] = None,
                                   k_ranges: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                                   stream=None) -> None:
    """q, o: [sequences, q_rows, q_heads, head_dim]; k, v: [sequences, k_rows, kv_heads, head_dim]; without the first dimension
    for packed sequences.  One 16-bit type, unit inner stride.  lse: float32 [sequences, q_heads, q_rows] (packed: [q_heads, q_rows]),
    out, or None.  window: None for every key up to the query's own place; scale: None for head_dim ** -0.5.  q_ranges, k_ranges: int32
    [sequences, 2], first row and number of rows, or None for all.  workspace: uint8 CUDA tensor of
    a2sgd_window_attention_workspace bytes."""
    dev, shape = _attention_shape(q, k, window, sinks, scale, q_ranges, k_ranges)
    dt, wb, qs, ks = q.dtype, 0 if workspace is None else workspace.numel(), q.shape, k.shape
    _check(lib().a2sgd_window_attention_forward(
        ctypes.addressof(shape), _heads(q, "q", qs, dt, dev), _heads(k, "k", ks, dt, dev), _heads(v, "v", ks, dt, dev),
        _heads(o, "o", qs, dt, dev), _lse(lse, q, dev), _vector(workspace, "workspace", wb, torch.uint8, dev), wb, dev,
        _stream_on(dev, stream)), "a2sgd_window_attention_forward")


def a2sgd_window_attention_backward(dout: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, o: torch.Tensor,
                                    lse: torch.Tensor, dq: Optional[torch.Tensor], dk: Optional[torch.Tensor],
                                    dv: Optional[torch.Tensor], window: Optional[int] = None, sinks: int = 0,
                                    scale: Optional[float] = None, q_ranges: Optional[torch.Tensor] = None,
                                    k_ranges: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                                    stream=None) -> None:
    """dout: as o; o, lse: what the forward pass left; dq, dk, dv: out, as q, k, v, each may be None; the rest as in the forward pass,
    workspace of a2sgd_window_attention_workspace(..., backward=True) bytes."""
    dev, shape = _attention_shape(q, k, window, sinks, scale, q_ranges, k_ranges)
    dt, wb = q.dtype, 0 if workspace is None else workspace.numel()
    maybe = lambda t, name, like: None if t is None else _heads(t, name, like.shape, dt, dev)  # noqa: E731
    _check(lib().a2sgd_window_attention_backward(
        ctypes.addressof(shape), _heads(dout, "dout", q.shape, dt, dev), _heads(q, "q", q.shape, dt, dev), _heads(k, "k", k.shape, dt, dev),
        _heads(v, "v", k.shape, dt, dev), _heads(o, "o", q.shape, dt, dev), _lse(lse, q, dev), maybe(dq, "dq", q), maybe(dk, "dk", k),
        maybe(dv, "dv", k), _vector(workspace, "workspace", wb, torch.uint8, dev), wb, dev, _stream_on(dev, stream)),
        "a2sgd_window_attention_backward")


def a2sgd_window_attention_status(device: Optional[int] = None, stream=None) -> int:
    """Synchronises the stream; ERR_TIMEOUT if a wait inside one of the attention's kernels has run out on the device since this
    was last asked with the same stream, else OK."""
    device = torch.cuda.current_device() if device is None else int(device)
    st = ctypes.c_int(0)
    _check(lib().a2sgd_window_attention_status(device, ctypes.byref(st), _stream_on(device, stream)),
           "a2sgd_window_attention_status")
    return st.value


def a2sgd_rotary(q: torch.Tensor, k: Optional[torch.Tensor], q_out: torch.Tensor, k_out: Optional[torch.Tensor],
                 positions: torch.Tensor, sections, base: float = 10000.0, interleaved: bool = False,
                 ladder_per_axis: bool = False, inverse: bool = False, stream=None) -> None:
    """q, q_out: [tokens, q_heads, head_dim], unit inner stride; k, k_out: [tokens, k_heads, head_dim], or None; an output may be its
    input.  positions: int32 [axes, tokens], contiguous; sections: pairs of each axis.  inverse: the opposite angles, which is the
    backward pass."""
    dev, code = _cuda_index(q, "q"), _dtype_code(q, "q")
    if q.dim() != 3 or (k is not None and k.dim() != 3):
        raise ValueError("q, k: need [tokens, heads, head_dim]")
    tokens, heads, d = q.shape
    if (k is None) != (k_out is None) or (k is not None and (k.shape[0] != tokens or k.shape[2] != d)):
        raise ValueError("k, k_out: need as many tokens and elements as q, or neither")
    axes = len(sections)
    if positions.shape != (axes, tokens):
        raise ValueError(f"positions: need {[axes, tokens]}, got {list(positions.shape)}")
    pos = _vector(positions, "positions", axes * tokens, torch.int32, dev)
    if axes and min(sections) < 1:
        raise ValueError("sections: need at least one pair each")
    shape, dt = q.shape, q.dtype
    k_shape, k_in, k_turned = None, None, None
    if k is not None:
        k_shape = k.shape
        k_in, k_turned = _heads(k, "k", k_shape, dt, dev), _heads(k_out, "k_out", k_shape, dt, dev)
    flags = (ROTARY_INTERLEAVED if interleaved else 0) | (ROTARY_LADDER_PER_AXIS if ladder_per_axis else 0) | (ROTARY_INVERSE if inverse else 0)
    _check(lib().a2sgd_rotary(_heads(q, "q", shape, dt, dev), k_in, _heads(q_out, "q_out", shape, dt, dev), k_turned, pos, axes,
                              struct.pack(f"{axes}I", *sections), base, flags, tokens, heads, k_shape[1] if k_shape else 0, d, code, dev,
                              _stream_on(dev, stream)), "a2sgd_rotary")


_NORM_KINDS = {"layer": 0, "rms": RESIDUAL_RMS}


def _residual_shape(y, residual, kind, post, post_weight, post_bias, gate, gate_rows, alpha, pre_weight, pre_bias, stats, eps, *params):
    dev, code = _cuda_index(y, "y"), _dtype_code(y, "y")
    if y.dim() != 2:
        raise ValueError("y: need [rows, d]")
    if kind not in _NORM_KINDS:
        raise ValueError(f"kind: need one of {sorted(_NORM_KINDS)}, got {kind!r}")
    rows, d = y.shape
    pt = _param_dtype(y, post_weight, post_bias, gate, pre_weight, pre_bias, *params)
    groups = 0
    if gate is not None:
        if gate_rows < 1:
            raise ValueError("gate_rows: at least 1 with a gate")
        groups = -(-rows // gate_rows)
    rest = [None if t is None else _vector(t, name, n, pt, dev) for t, name, n in
            ((post_weight, "post_weight", d), (post_bias, "post_bias", d), (gate, "gate", groups * d), (pre_weight, "pre_weight", d),
             (pre_bias, "pre_bias", d))]
    rest += [None if t is None else _vector(t, name, rows, torch.float32, dev)
             for t, name in zip(stats, ("post_mean", "post_rstd", "pre_mean", "pre_rstd"))]
    shape = _ResidualShape(rows, gate_rows if gate is not None else 0, d, _NORM_KINDS[kind] | (RESIDUAL_POST_NORM if post else 0), code,
                           _dtype_code(residual, "x or z"), _DTYPE_CODES.get(pt, -1), 0, alpha, eps, *rest)
    return dev, shape, pt, groups


def _row_matrix(t: Optional[torch.Tensor], name: str, shape, dtype: torch.dtype, index: int) -> Optional[bytes]:
    return None if t is None else _pack_rows(*_matrix(t, name, shape, dtype, index))


def a2sgd_residual_norm_forward(x: torch.Tensor, y: torch.Tensor, z: torch.Tensor, u: torch.Tensor, kind: str = "rms",
                                post: bool = True, post_weight: Optional[torch.Tensor] = None,
                                post_bias: Optional[torch.Tensor] = None, gate: Optional[torch.Tensor] = None, gate_rows: int = 0,
                                alpha: float = 1.0, pre_weight: Optional[torch.Tensor] = None,
                                pre_bias: Optional[torch.Tensor] = None, post_mean: Optional[torch.Tensor] = None,
                                post_rstd: Optional[torch.Tensor] = None, pre_mean: Optional[torch.Tensor] = None,
                                pre_rstd: Optional[torch.Tensor] = None, eps: float = 1e-5, stream=None) -> None:
    """z = x + alpha * gate * norm(y), u = norm(z).  y, u: [rows, d]; x, z: the same in float32 or y's type, unit inner stride; z
    may be x, u may be y.  kind: "rms" or "layer"; post False: y is not normed.  weights, biases: [d]; gate: [ceil(rows / gate_rows), d];
    of float32 or y's type, each may be None.  post_mean ... pre_rstd: float32 [rows], out, or None."""
    dev, shape, _, _ = _residual_shape(y, x, kind, post, post_weight, post_bias, gate, gate_rows, alpha, pre_weight, pre_bias,
                                       (post_mean, post_rstd, pre_mean, pre_rstd), eps)
    rows_d, yt, xt = y.shape, y.dtype, x.dtype
    _check(lib().a2sgd_residual_norm_forward(
        ctypes.addressof(shape), _row_matrix(x, "x", rows_d, xt, dev), _row_matrix(y, "y", rows_d, yt, dev), _row_matrix(z, "z", rows_d, xt, dev),
        _row_matrix(u, "u", rows_d, yt, dev), dev, _stream_on(dev, stream)), "a2sgd_residual_norm_forward")


def a2sgd_residual_norm_workspace(rows: int, d: int, gate_rows: int = 0, device: Optional[int] = None) -> int:
    """Bytes of workspace of a2sgd_residual_norm_backward (gate_rows: 0 without a gate)."""
    device = torch.cuda.current_device() if device is None else int(device)
    return int(lib().a2sgd_residual_norm_workspace(int(rows), int(d), int(gate_rows), device))


def a2sgd_residual_norm_backward(dz: Optional[torch.Tensor], du: torch.Tensor, y: torch.Tensor, z: torch.Tensor,
                                 dx: Optional[torch.Tensor], dy: Optional[torch.Tensor], kind: str = "rms", post: bool = True,
                                 post_weight: Optional[torch.Tensor] = None, post_bias: Optional[torch.Tensor] = None,
                                 gate: Optional[torch.Tensor] = None, gate_rows: int = 0, alpha: float = 1.0,
                                 pre_weight: Optional[torch.Tensor] = None, post_mean: Optional[torch.Tensor] = None,
                                 post_rstd: Optional[torch.Tensor] = None, pre_mean: Optional[torch.Tensor] = None,
                                 pre_rstd: Optional[torch.Tensor] = None, dpost_weight: Optional[torch.Tensor] = None,
                                 dpost_bias: Optional[torch.Tensor] = None, dgate: Optional[torch.Tensor] = None,
                                 dpre_weight: Optional[torch.Tensor] = None, dpre_bias: Optional[torch.Tensor] = None,
                                 workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    """dz: what reaches z beside u (None: nothing); du, y, z and the statistics as the forward pass left them; dx (may be dz), dy (may be
    du or y) and the sums over the rows: out, each may be None.  workspace: uint8 CUDA tensor of a2sgd_residual_norm_workspace bytes,
    needed for any of the sums."""
    dev, shape, pt, groups = _residual_shape(y, z, kind, post, post_weight, post_bias, gate, gate_rows, alpha, pre_weight, None,
                                             (post_mean, post_rstd, pre_mean, pre_rstd), 0.0, dpost_weight, dpost_bias, dgate,
                                             dpre_weight, dpre_bias)
    d = y.shape[1]
    tensors = [_row_matrix(t, name, y.shape, dtype, dev) for t, name, dtype in
               ((dz, "dz", z.dtype), (du, "du", y.dtype), (y, "y", y.dtype), (z, "z", z.dtype), (dx, "dx", z.dtype), (dy, "dy", y.dtype))]
    sums = (_vp * 5)(_vector(dpost_weight, "dpost_weight", d, pt, dev), _vector(dpost_bias, "dpost_bias", d, pt, dev),
                     _vector(dgate, "dgate", groups * d, pt, dev), _vector(dpre_weight, "dpre_weight", d, pt, dev),
                     _vector(dpre_bias, "dpre_bias", d, pt, dev))
    wb = 0 if workspace is None else workspace.numel()
    _check(lib().a2sgd_residual_norm_backward(ctypes.addressof(shape), *tensors, ctypes.addressof(sums),
                                              _vector(workspace, "workspace", wb, torch.uint8, dev), wb, dev, _stream_on(dev, stream)),
           "a2sgd_residual_norm_backward")
