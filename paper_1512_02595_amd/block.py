"""Binding of the recurrent block's calls (include/ctc_block.h): argument marshalling only.

The functions mirror the header: the same arguments in the same order, device buffers as integer addresses (for
instance torch.Tensor.data_ptr(); None or 0 where the header allows NULL).  Each raises `ctc.CTCError` with the
status; its twin `..._status` returns it.  They go through the native module `_block_binding`; there is no
fallback.
"""
from __future__ import annotations

import ctypes

from . import ctc, layer

EXPORTS = ("ctc_recurrence_workspace_size", "ctc_recurrence", "ctc_recurrence_backward", "ctc_block_norm",
           "ctc_block_norm_workspace_size", "ctc_block_norm_backward", "ctc_clear_frames", "ctc_weights_i4_sizes",
           "ctc_quantize_weights_i4", "ctc_dequantize_weights_i4", "ctc_linear_i4")
_CALLS = ("recurrence", "recurrence_backward", "block_norm", "block_norm_backward", "clear_frames", "quantize_weights_i4",
          "dequantize_weights_i4", "linear_i4")

_lib = None
_native = None                # the module `_block_binding`, once load() has given it the library's addresses


def load() -> ctypes.CDLL:
    """The HIP library with these calls declared (once).  Raises if it has not been built."""
    global _lib, _native
    if _lib is not None:
        return _lib
    lib = layer.load()
    from . import _block_binding                                 # (built by the same command)
    ci, st, sizes = ctypes.c_int, ctypes.c_int, ctypes.POINTER(ctypes.c_size_t)
    lib.ctc_recurrence_workspace_size.restype = st
    lib.ctc_recurrence_workspace_size.argtypes = [ci, ci, ci, sizes]
    lib.ctc_block_norm_workspace_size.restype = st
    lib.ctc_block_norm_workspace_size.argtypes = [ci, ci, sizes]
    lib.ctc_weights_i4_sizes.restype = st
    lib.ctc_weights_i4_sizes.argtypes = [ci, ci, ci, sizes, sizes]
    _block_binding.bind(*(ctypes.cast(getattr(lib, "ctc_" + name), ctypes.c_void_p).value for name in _CALLS))
    _native = _block_binding
    _lib = lib
    return lib


def _module():
    if _native is None:
        load()
    return _native


def recurrence_workspace_size_status(T, B, H):
    """(status, bytes), without raising."""
    out = ctypes.c_size_t(0)
    st = load().ctc_recurrence_workspace_size(layer._size(T), layer._size(B), layer._size(H), ctypes.byref(out))
    return int(st), int(out.value)


def recurrence_workspace_size(T, B, H) -> int:
    st, n = recurrence_workspace_size_status(T, B, H)
    layer._check(st, "ctc_recurrence_workspace_size")
    return n


def block_norm_workspace_size_status(rows, H):
    """(status, bytes), without raising."""
    out = ctypes.c_size_t(0)
    return int(load().ctc_block_norm_workspace_size(layer._size(rows), layer._size(H), ctypes.byref(out))), int(out.value)


def block_norm_workspace_size(rows, H) -> int:
    st, n = block_norm_workspace_size_status(rows, H)
    layer._check(st, "ctc_block_norm_workspace_size")
    return n


def weights_i4_sizes_status(A, H, group):
    """(status, (bytes of the weights, bytes of their scales)), without raising."""
    w, s = ctypes.c_size_t(0), ctypes.c_size_t(0)
    st = load().ctc_weights_i4_sizes(layer._size(A), layer._size(H), layer._size(group), ctypes.byref(w), ctypes.byref(s))
    return int(st), (int(w.value), int(s.value))


def weights_i4_sizes(A, H, group):
    """(bytes of the weights, bytes of their scales)."""
    st, both = weights_i4_sizes_status(A, H, group)
    layer._check(st, "ctc_weights_i4_sizes")
    return both


def recurrence_status(inputs_ptr, input_pitch, input_lengths_ptr, initial_ptr, T, B, H, forward_channels, dtype, states_ptr,
                      final_ptr, workspace_ptr, workspace_bytes, stream=0) -> int:
    return _module().recurrence(inputs_ptr, input_pitch, input_lengths_ptr, initial_ptr, T, B, H, forward_channels, dtype,
                                states_ptr, final_ptr, workspace_ptr, workspace_bytes, stream)


def recurrence(inputs_ptr, input_pitch, input_lengths_ptr, initial_ptr, T, B, H, forward_channels, dtype, states_ptr,
               final_ptr, workspace_ptr, workspace_bytes, stream=0) -> None:
    """States of all frames from gates and candidates."""
    st = (_native or _module()).recurrence(inputs_ptr, input_pitch, input_lengths_ptr, initial_ptr, T, B, H,
                                           forward_channels, dtype, states_ptr, final_ptr, workspace_ptr, workspace_bytes,
                                           stream)
    if st:
        layer._check(st, "ctc_recurrence")


def recurrence_backward_status(dstates_ptr, dfinal_ptr, inputs_ptr, input_pitch, states_ptr, input_lengths_ptr, initial_ptr,
                               T, B, H, forward_channels, dtype, dinputs_ptr, dinitial_ptr, workspace_ptr, workspace_bytes,
                               stream=0) -> int:
    return _module().recurrence_backward(dstates_ptr, dfinal_ptr, inputs_ptr, input_pitch, states_ptr, input_lengths_ptr,
                                         initial_ptr, T, B, H, forward_channels, dtype, dinputs_ptr, dinitial_ptr,
                                         workspace_ptr, workspace_bytes, stream)


def recurrence_backward(dstates_ptr, dfinal_ptr, inputs_ptr, input_pitch, states_ptr, input_lengths_ptr, initial_ptr, T, B,
                        H, forward_channels, dtype, dinputs_ptr, dinitial_ptr, workspace_ptr, workspace_bytes, stream=0) -> None:
    """Gradient of the recurrence's gates, candidates and initial states."""
    st = (_native or _module()).recurrence_backward(dstates_ptr, dfinal_ptr, inputs_ptr, input_pitch, states_ptr,
                                                    input_lengths_ptr, initial_ptr, T, B, H, forward_channels, dtype,
                                                    dinputs_ptr, dinitial_ptr, workspace_ptr, workspace_bytes, stream)
    if st:
        layer._check(st, "ctc_recurrence_backward")


def block_norm_status(x_ptr, gate_ptr, gate_pitch, residual_ptr, weight_after_ptr, scale_ptr, weight_before_ptr, eps,
                      frames_ptr, rows, H, dtype, sum_ptr, normed_ptr, stream=0) -> int:
    return _module().block_norm(x_ptr, gate_ptr, gate_pitch, residual_ptr, weight_after_ptr, scale_ptr, weight_before_ptr,
                                eps, frames_ptr, rows, H, dtype, sum_ptr, normed_ptr, stream)


def block_norm(x_ptr, gate_ptr, gate_pitch, residual_ptr, weight_after_ptr, scale_ptr, weight_before_ptr, eps, frames_ptr,
               rows, H, dtype, sum_ptr, normed_ptr, stream=0) -> None:
    """Norm after a block, gate, residual scale, residual, norm before the next."""
    st = (_native or _module()).block_norm(x_ptr, gate_ptr, gate_pitch, residual_ptr, weight_after_ptr, scale_ptr,
                                           weight_before_ptr, eps, frames_ptr, rows, H, dtype, sum_ptr, normed_ptr, stream)
    if st:
        layer._check(st, "ctc_block_norm")


def block_norm_backward_status(dnormed_ptr, dsum_ptr, x_ptr, gate_ptr, gate_pitch, sum_ptr, weight_after_ptr, scale_ptr,
                               weight_before_ptr, eps, frames_ptr, rows, H, dtype, dx_ptr, dgate_ptr, dresidual_ptr,
                               dweight_after_ptr, dscale_ptr, dweight_before_ptr, workspace_ptr, workspace_bytes, stream=0) -> int:
    return _module().block_norm_backward(dnormed_ptr, dsum_ptr, x_ptr, gate_ptr, gate_pitch, sum_ptr, weight_after_ptr,
                                         scale_ptr, weight_before_ptr, eps, frames_ptr, rows, H, dtype, dx_ptr, dgate_ptr,
                                         dresidual_ptr, dweight_after_ptr, dscale_ptr, dweight_before_ptr, workspace_ptr,
                                         workspace_bytes, stream)


def block_norm_backward(dnormed_ptr, dsum_ptr, x_ptr, gate_ptr, gate_pitch, sum_ptr, weight_after_ptr, scale_ptr,
                        weight_before_ptr, eps, frames_ptr, rows, H, dtype, dx_ptr, dgate_ptr, dresidual_ptr,
                        dweight_after_ptr, dscale_ptr, dweight_before_ptr, workspace_ptr, workspace_bytes, stream=0) -> None:
    """Gradient of the norms around a block."""
    st = (_native or _module()).block_norm_backward(dnormed_ptr, dsum_ptr, x_ptr, gate_ptr, gate_pitch, sum_ptr,
                                                    weight_after_ptr, scale_ptr, weight_before_ptr, eps, frames_ptr, rows, H,
                                                    dtype, dx_ptr, dgate_ptr, dresidual_ptr, dweight_after_ptr, dscale_ptr,
                                                    dweight_before_ptr, workspace_ptr, workspace_bytes, stream)
    if st:
        layer._check(st, "ctc_block_norm_backward")


def clear_frames_status(x_ptr, pitch, input_lengths_ptr, T, B, width, dtype, stream=0) -> int:
    return _module().clear_frames(x_ptr, pitch, input_lengths_ptr, T, B, width, dtype, stream)


def clear_frames(x_ptr, pitch, input_lengths_ptr, T, B, width, dtype, stream=0) -> None:
    """Zeros behind the utterances' ends."""
    st = (_native or _module()).clear_frames(x_ptr, pitch, input_lengths_ptr, T, B, width, dtype, stream)
    if st:
        layer._check(st, "ctc_clear_frames")


def quantize_weights_i4_status(weights_ptr, A, H, group, dtype, weight_q_ptr, weight_scales_ptr, stream=0) -> int:
    return _module().quantize_weights_i4(weights_ptr, A, H, group, dtype, weight_q_ptr, weight_scales_ptr, stream)


def quantize_weights_i4(weights_ptr, A, H, group, dtype, weight_q_ptr, weight_scales_ptr, stream=0) -> None:
    """Weights to 4 bits with a scale per group of columns."""
    st = (_native or _module()).quantize_weights_i4(weights_ptr, A, H, group, dtype, weight_q_ptr, weight_scales_ptr, stream)
    if st:
        layer._check(st, "ctc_quantize_weights_i4")


def dequantize_weights_i4_status(weight_q_ptr, weight_scales_ptr, A, H, group, dtype, out_ptr, stream=0) -> int:
    return _module().dequantize_weights_i4(weight_q_ptr, weight_scales_ptr, A, H, group, dtype, out_ptr, stream)


def dequantize_weights_i4(weight_q_ptr, weight_scales_ptr, A, H, group, dtype, out_ptr, stream=0) -> None:
    """Weights from 4 bits."""
    st = (_native or _module()).dequantize_weights_i4(weight_q_ptr, weight_scales_ptr, A, H, group, dtype, out_ptr, stream)
    if st:
        layer._check(st, "ctc_dequantize_weights_i4")


def linear_i4_status(q_ptr, scales_ptr, weight_q_ptr, weight_scales_ptr, group, bias_ptr, frames_ptr, rows, H, A, dtype,
                     logits_ptr, stream=0) -> int:
    return _module().linear_i4(q_ptr, scales_ptr, weight_q_ptr, weight_scales_ptr, group, bias_ptr, frames_ptr, rows, H, A,
                               dtype, logits_ptr, stream)


def linear_i4(q_ptr, scales_ptr, weight_q_ptr, weight_scales_ptr, group, bias_ptr, frames_ptr, rows, H, A, dtype, logits_ptr,
              stream=0) -> None:
    """Activations from rows in 8 bits and weights in 4."""
    st = (_native or _module()).linear_i4(q_ptr, scales_ptr, weight_q_ptr, weight_scales_ptr, group, bias_ptr, frames_ptr,
                                          rows, H, A, dtype, logits_ptr, stream)
    if st:
        layer._check(st, "ctc_linear_i4")
