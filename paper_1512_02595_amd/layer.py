"""Binding of the output layer's calls (include/ctc_layer.h): argument marshalling only.

The functions mirror the header: the same arguments in the same order, device buffers as integer addresses (for
instance torch.Tensor.data_ptr(); None or 0 where the header allows NULL).  Each raises `ctc.CTCError` with the
status; its twin `..._status` returns it.  They go through the native module `_layer_binding`; there is no
fallback.
"""
from __future__ import annotations

import ctypes
import operator

from . import ctc

MAX_STATE_WIDTH = 16384

EXPORTS = ("ctc_row_pitch", "ctc_pack_frames", "ctc_quantize_rows", "ctc_dequantize_rows", "ctc_rms_norm_i8",
           "ctc_rms_norm_workspace_size", "ctc_rms_norm_backward", "ctc_linear_i8", "ctc_weight_gradient_workspace_size",
           "ctc_weight_gradient_i8", "ctc_layer_last_hip_error")
_CALLS = ("pack_frames", "quantize_rows", "dequantize_rows", "rms_norm_i8", "rms_norm_backward", "linear_i8",
          "weight_gradient_i8")

_lib = None
_native = None                # the module `_layer_binding`, once load() has given it the library's addresses


def load() -> ctypes.CDLL:
    """The HIP library with these calls declared (once).  Raises if it has not been built."""
    global _lib, _native
    if _lib is not None:
        return _lib
    lib = ctc.load()
    from . import _layer_binding                                 # (built by the same command)
    ci, st, sizes = ctypes.c_int, ctypes.c_int, ctypes.POINTER(ctypes.c_size_t)
    lib.ctc_row_pitch.restype = ci
    lib.ctc_row_pitch.argtypes = [ci]
    lib.ctc_layer_last_hip_error.restype = ci
    lib.ctc_layer_last_hip_error.argtypes = []
    lib.ctc_rms_norm_workspace_size.restype = st
    lib.ctc_rms_norm_workspace_size.argtypes = [ci, ci, sizes]
    lib.ctc_weight_gradient_workspace_size.restype = st
    lib.ctc_weight_gradient_workspace_size.argtypes = [ci, ci, ci, sizes]
    _layer_binding.bind(*(ctypes.cast(getattr(lib, "ctc_" + name), ctypes.c_void_p).value for name in _CALLS))
    _native = _layer_binding
    _lib = lib
    return lib


def last_hip_error() -> int:
    return int(load().ctc_layer_last_hip_error())


def _size(v) -> int:
    """A whole number that a C int holds, as the native module takes one (ctypes would drop what does not fit)."""
    v = operator.index(v)
    if not -2 ** 31 <= v < 2 ** 31:
        raise OverflowError("a size is out of a 32-bit integer's range")
    return v


def row_pitch(H) -> int:
    """Bytes from one row in 8 bits to the next; 0 for a width that is refused."""
    return int(load().ctc_row_pitch(_size(H)))


def _check(status: int, where: str) -> None:
    if status:
        extra = f" (hipError {last_hip_error()})" if status == ctc.STATUS_HIP_ERROR else ""
        raise ctc.CTCError(status, where + extra)


def _module():
    if _native is None:
        load()
    return _native


def rms_norm_workspace_size_status(rows, H):
    """(status, bytes), without raising."""
    out = ctypes.c_size_t(0)
    return int(load().ctc_rms_norm_workspace_size(_size(rows), _size(H), ctypes.byref(out))), int(out.value)


def rms_norm_workspace_size(rows, H) -> int:
    st, n = rms_norm_workspace_size_status(rows, H)
    _check(st, "ctc_rms_norm_workspace_size")
    return n


def weight_gradient_workspace_size_status(rows, H, A):
    """(status, bytes), without raising."""
    out = ctypes.c_size_t(0)
    st = load().ctc_weight_gradient_workspace_size(_size(rows), _size(H), _size(A), ctypes.byref(out))
    return int(st), int(out.value)


def weight_gradient_workspace_size(rows, H, A) -> int:
    st, n = weight_gradient_workspace_size_status(rows, H, A)
    _check(st, "ctc_weight_gradient_workspace_size")
    return n


def pack_frames_status(input_lengths_ptr, T, B, frames_ptr, stream=0) -> int:
    return _module().pack_frames(input_lengths_ptr, T, B, frames_ptr, stream)


def pack_frames(input_lengths_ptr, T, B, frames_ptr, stream=0) -> None:
    """The list of a minibatch's frames, int32 [1 + T * B], from its input lengths on the GPU: their number, then their rows in ascending order."""
    st = (_native or _module()).pack_frames(input_lengths_ptr, T, B, frames_ptr, stream)
    if st:
        _check(st, "ctc_pack_frames")


def quantize_rows_status(x_ptr, frames_ptr, rows, H, dtype, q_ptr, scales_ptr, stream=0) -> int:
    return _module().quantize_rows(x_ptr, frames_ptr, rows, H, dtype, q_ptr, scales_ptr, stream)


def quantize_rows(x_ptr, frames_ptr, rows, H, dtype, q_ptr, scales_ptr, stream=0) -> None:
    """Rows to 8 bits: int8 [rows, row_pitch(H)] and a scale each."""
    st = (_native or _module()).quantize_rows(x_ptr, frames_ptr, rows, H, dtype, q_ptr, scales_ptr, stream)
    if st:
        _check(st, "ctc_quantize_rows")


def dequantize_rows_status(q_ptr, scales_ptr, frames_ptr, rows, H, dtype, out_ptr, stream=0) -> int:
    return _module().dequantize_rows(q_ptr, scales_ptr, frames_ptr, rows, H, dtype, out_ptr, stream)


def dequantize_rows(q_ptr, scales_ptr, frames_ptr, rows, H, dtype, out_ptr, stream=0) -> None:
    """Rows from 8 bits."""
    st = (_native or _module()).dequantize_rows(q_ptr, scales_ptr, frames_ptr, rows, H, dtype, out_ptr, stream)
    if st:
        _check(st, "ctc_dequantize_rows")


def rms_norm_i8_status(x_ptr, residual_ptr, weight_ptr, eps, frames_ptr, rows, H, dtype, sum_ptr, q_ptr, scales_ptr,
                       stream=0) -> int:
    return _module().rms_norm_i8(x_ptr, residual_ptr, weight_ptr, eps, frames_ptr, rows, H, dtype, sum_ptr, q_ptr, scales_ptr,
                                 stream)


def rms_norm_i8(x_ptr, residual_ptr, weight_ptr, eps, frames_ptr, rows, H, dtype, sum_ptr, q_ptr, scales_ptr, stream=0) -> None:
    """Residual added, root-mean-square norm, rows to 8 bits."""
    st = (_native or _module()).rms_norm_i8(x_ptr, residual_ptr, weight_ptr, eps, frames_ptr, rows, H, dtype, sum_ptr, q_ptr,
                                            scales_ptr, stream)
    if st:
        _check(st, "ctc_rms_norm_i8")


def rms_norm_backward_status(dy_ptr, sum_ptr, weight_ptr, eps, dresidual_ptr, frames_ptr, rows, H, dtype, dsum_ptr,
                             dweight_ptr, workspace_ptr, workspace_bytes, stream=0) -> int:
    return _module().rms_norm_backward(dy_ptr, sum_ptr, weight_ptr, eps, dresidual_ptr, frames_ptr, rows, H, dtype, dsum_ptr,
                                       dweight_ptr, workspace_ptr, workspace_bytes, stream)


def rms_norm_backward(dy_ptr, sum_ptr, weight_ptr, eps, dresidual_ptr, frames_ptr, rows, H, dtype, dsum_ptr, dweight_ptr,
                      workspace_ptr, workspace_bytes, stream=0) -> None:
    """Gradient of the norm."""
    st = (_native or _module()).rms_norm_backward(dy_ptr, sum_ptr, weight_ptr, eps, dresidual_ptr, frames_ptr, rows, H, dtype,
                                                  dsum_ptr, dweight_ptr, workspace_ptr, workspace_bytes, stream)
    if st:
        _check(st, "ctc_rms_norm_backward")


def linear_i8_status(q_ptr, scales_ptr, weight_q_ptr, weight_scales_ptr, bias_ptr, frames_ptr, rows, H, A, dtype, logits_ptr,
                     stream=0) -> int:
    return _module().linear_i8(q_ptr, scales_ptr, weight_q_ptr, weight_scales_ptr, bias_ptr, frames_ptr, rows, H, A, dtype,
                               logits_ptr, stream)


def linear_i8(q_ptr, scales_ptr, weight_q_ptr, weight_scales_ptr, bias_ptr, frames_ptr, rows, H, A, dtype, logits_ptr,
              stream=0) -> None:
    """Activations from rows and weights in 8 bits."""
    st = (_native or _module()).linear_i8(q_ptr, scales_ptr, weight_q_ptr, weight_scales_ptr, bias_ptr, frames_ptr, rows, H, A,
                                          dtype, logits_ptr, stream)
    if st:
        _check(st, "ctc_linear_i8")


def weight_gradient_i8_status(grads_ptr, q_ptr, scales_ptr, frames_ptr, rows, H, A, dtype, dweight_ptr, dbias_ptr,
                              workspace_ptr, workspace_bytes, stream=0) -> int:
    return _module().weight_gradient_i8(grads_ptr, q_ptr, scales_ptr, frames_ptr, rows, H, A, dtype, dweight_ptr, dbias_ptr,
                                        workspace_ptr, workspace_bytes, stream)


def weight_gradient_i8(grads_ptr, q_ptr, scales_ptr, frames_ptr, rows, H, A, dtype, dweight_ptr, dbias_ptr, workspace_ptr,
                       workspace_bytes, stream=0) -> None:
    """The weights' and the bias's gradient from the activations' gradient and the rows in 8 bits."""
    st = (_native or _module()).weight_gradient_i8(grads_ptr, q_ptr, scales_ptr, frames_ptr, rows, H, A, dtype, dweight_ptr,
                                                   dbias_ptr, workspace_ptr, workspace_bytes, stream)
    if st:
        _check(st, "ctc_weight_gradient_i8")
