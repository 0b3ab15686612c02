// Host side of the recurrent block's calls: what ctc_block.h says about arguments is checked here, then one to three
// kernels are enqueued.  Nothing is allocated, waited for or kept.

#include <cmath>

#include "layer_block_internal.h"
#include "layer_checks.h"

namespace layer {
namespace {

bool known(ctc_dtype_t dtype) { return dtype == CTC_DTYPE_F32 || dtype == CTC_DTYPE_BF16; }

// Bytes from a matrix's first element to its last, where rows of `width` lie `pitch` apart.
size_t pitched(int rows, int64_t pitch, int64_t width, size_t elem) { return (static_cast<size_t>(rows - 1) * pitch + width) * elem; }

ctc_status_t minibatch_in_range(int T, int B, int H)
{
    if (T < 1 || B < 1 || H < 1) return CTC_STATUS_INVALID_VALUE;
    if (B > kMaxUtterances || H > kMaxWidth || static_cast<int64_t>(T) * B > kMaxRows) return CTC_STATUS_UNSUPPORTED;
    return CTC_STATUS_SUCCESS;
}

ctc_status_t recurrence_in_range(int pitch, int T, int B, int H, int forward_channels, ctc_dtype_t dtype)
{
    if (!known(dtype) || forward_channels < 0 || forward_channels > H) return CTC_STATUS_INVALID_VALUE;
    const ctc_status_t st = minibatch_in_range(T, B, H);
    if (st != CTC_STATUS_SUCCESS) return st;
    if (pitch < 2 * H) return CTC_STATUS_INVALID_VALUE;
    return pitch > kMaxPitch ? CTC_STATUS_UNSUPPORTED : CTC_STATUS_SUCCESS;
}

ctc_status_t rows_in_range(int rows, int H, const void* gate, int gate_pitch, float eps, ctc_dtype_t dtype)
{
    if (!known(dtype) || rows < 1 || H < 1 || !std::isfinite(eps) || eps <= 0.0f) return CTC_STATUS_INVALID_VALUE;
    if (rows > kMaxRows || H > kMaxWidth) return CTC_STATUS_UNSUPPORTED;
    if (!gate) return CTC_STATUS_SUCCESS;
    if (gate_pitch < H) return CTC_STATUS_INVALID_VALUE;
    return gate_pitch > kMaxPitch ? CTC_STATUS_UNSUPPORTED : CTC_STATUS_SUCCESS;
}

ctc_status_t weights_in_range(int A, int H, int group)
{
    if (A < 1 || H < 1 || !group_in_order(group)) return CTC_STATUS_INVALID_VALUE;
    return H > kMaxWidth || A > kMaxSymbols ? CTC_STATUS_UNSUPPORTED : CTC_STATUS_SUCCESS;
}

size_t block_norm_workspace(int rows, int H) { return round_up(static_cast<size_t>(block_norm_groups(rows, H)) * 2 * H * 4); }

}  // namespace
}  // namespace layer

using namespace layer;

extern "C" {

ctc_status_t ctc_recurrence_workspace_size(int T, int B, int H, size_t* bytes_out)
{
    if (!bytes_out) return CTC_STATUS_INVALID_VALUE;
    const ctc_status_t st = minibatch_in_range(T, B, H);
    if (st == CTC_STATUS_SUCCESS) *bytes_out = round_up(recurrence_bytes(T, B, H));
    return st;
}

ctc_status_t ctc_recurrence(const void* inputs, int input_pitch, const int32_t* input_lengths, const float* initial, int T, int B,
                            int H, int forward_channels, ctc_dtype_t dtype, void* states, float* final_states, void* workspace,
                            size_t workspace_bytes, hipStream_t stream)
{
    const ctc_status_t st = recurrence_in_range(input_pitch, T, B, H, forward_channels, dtype);
    if (st != CTC_STATUS_SUCCESS) return st;
    const size_t e = element(dtype), needed = round_up(recurrence_bytes(T, B, H)), carried = matrix(B, H, 4);
    if (!buffers_in_order({{inputs, pitched(T * B, input_pitch, 2 * H, e), false, true, e},
                           {input_lengths, matrix(B, 1, 4), false, false},
                           {initial, carried, false, false, 4, true},
                           {states, matrix(T * B, H, e), true, true, e},
                           {final_states, carried, true, false, 4, false, true},
                           {needed ? workspace : nullptr, needed, true, needed != 0, 256}}))
        return CTC_STATUS_INVALID_VALUE;
    if (workspace_bytes < needed) return CTC_STATUS_WORKSPACE_TOO_SMALL;
    const RecurrenceArgs p = {inputs, input_pitch, input_lengths, initial, T, B, H, forward_channels, nullptr, nullptr, nullptr, states,
                              final_states, static_cast<double*>(workspace)};
    return launched(launch_recurrence(p, dtype == CTC_DTYPE_BF16, false, stream));
}

ctc_status_t ctc_recurrence_backward(const void* dstates, const float* dfinal, const void* inputs, int input_pitch, const void* states,
                                     const int32_t* input_lengths, const float* initial, int T, int B, int H, int forward_channels,
                                     ctc_dtype_t dtype, void* dinputs, float* dinitial, void* workspace, size_t workspace_bytes,
                                     hipStream_t stream)
{
    const ctc_status_t st = recurrence_in_range(input_pitch, T, B, H, forward_channels, dtype);
    if (st != CTC_STATUS_SUCCESS) return st;
    const size_t e = element(dtype), needed = round_up(recurrence_bytes(T, B, H)), carried = matrix(B, H, 4);
    const size_t projected = pitched(T * B, input_pitch, 2 * H, e), all = matrix(T * B, H, e);
    if (!buffers_in_order({{dstates, all, false, true, e},
                           {dfinal, carried, false, false, 4, true},
                           {inputs, projected, false, true, e},
                           {states, all, false, true, e},
                           {input_lengths, matrix(B, 1, 4), false, false},
                           {initial, carried, false, false},
                           {dinputs, projected, true, true, e},
                           {dinitial, carried, true, false, 4, false, true},
                           {needed ? workspace : nullptr, needed, true, needed != 0, 256}}))
        return CTC_STATUS_INVALID_VALUE;
    if (workspace_bytes < needed) return CTC_STATUS_WORKSPACE_TOO_SMALL;
    const RecurrenceArgs p = {inputs, input_pitch, input_lengths, initial, T, B, H, forward_channels, states, dstates, dfinal, dinputs,
                              dinitial, static_cast<double*>(workspace)};
    return launched(launch_recurrence(p, dtype == CTC_DTYPE_BF16, true, stream));
}

ctc_status_t ctc_block_norm(const void* x, const void* gate, int gate_pitch, const void* residual, const float* weight_after,
                            const float* scale, const float* weight_before, float eps, const int32_t* frames, int rows, int H,
                            ctc_dtype_t dtype, void* sum, void* normed, hipStream_t stream)
{
    const ctc_status_t st = rows_in_range(rows, H, gate, gate_pitch, eps, dtype);
    if (st != CTC_STATUS_SUCCESS) return st;
    if (!sum && !normed) return CTC_STATUS_INVALID_VALUE;
    const size_t e = element(dtype), states = matrix(rows, H, e), weights = matrix(H, 1, 4);
    if (!buffers_in_order({{x, states, false, true, e, true},
                           {gate, pitched(rows, gate_pitch, H, e), false, false, e},
                           {residual, states, false, false, e, true},
                           {weight_after, weights, false, false},
                           {scale, weights, false, false},
                           {weight_before, weights, false, false},
                           {frames, list_bytes(rows), false, false},
                           {sum, states, true, false, e, false, true},
                           {normed, states, true, false, e, false, true}}))
        return CTC_STATUS_INVALID_VALUE;
    const BlockNormArgs p = {x, gate, gate_pitch, residual, weight_after, scale, weight_before, eps, frames, rows, H, sum, normed};
    return launched(launch_block_norm(p, dtype == CTC_DTYPE_BF16, stream));
}

ctc_status_t ctc_block_norm_workspace_size(int rows, int H, size_t* bytes_out)
{
    if (!bytes_out || rows < 1 || H < 1) return CTC_STATUS_INVALID_VALUE;
    if (rows > kMaxRows || H > kMaxWidth) return CTC_STATUS_UNSUPPORTED;
    *bytes_out = block_norm_workspace(rows, H);
    return CTC_STATUS_SUCCESS;
}

ctc_status_t ctc_block_norm_backward(const void* dnormed, const void* dsum, const void* x, const void* gate, int gate_pitch,
                                     const void* sum, const float* weight_after, const float* scale, const float* weight_before,
                                     float eps, const int32_t* frames, int rows, int H, ctc_dtype_t dtype, void* dx, void* dgate,
                                     void* dresidual, float* dweight_after, float* dscale, float* dweight_before, void* workspace,
                                     size_t workspace_bytes, hipStream_t stream)
{
    const ctc_status_t st = rows_in_range(rows, H, gate, gate_pitch, eps, dtype);
    if (st != CTC_STATUS_SUCCESS) return st;
    if ((!dnormed && !dsum) || (dnormed && !sum) || (gate != nullptr) != (dgate != nullptr)) return CTC_STATUS_INVALID_VALUE;
    const bool sums = dweight_after || dscale || dweight_before;
    const size_t e = element(dtype), states = matrix(rows, H, e), weights = matrix(H, 1, 4), needed = block_norm_workspace(rows, H);
    const size_t gates = gate ? pitched(rows, gate_pitch, H, e) : 0;
    if (!buffers_in_order({{dnormed, states, false, false, e, true},
                           {dsum, states, false, false, e, true},
                           {x, states, false, true, e, true},
                           {gate, gates, false, false, e},
                           {sum, states, false, false, e, true},
                           {weight_after, weights, false, false},
                           {scale, weights, false, false},
                           {weight_before, weights, false, false},
                           {frames, list_bytes(rows), false, false},
                           {dx, states, true, true, e, false, true},
                           {dgate, gates, true, false, e},
                           {dresidual, states, true, false, e, false, true},
                           {dweight_after, weights, true, false},
                           {dscale, weights, true, false},
                           {dweight_before, weights, true, false},
                           {sums ? workspace : nullptr, needed, true, sums, 256}}))
        return CTC_STATUS_INVALID_VALUE;
    if (sums && workspace_bytes < needed) return CTC_STATUS_WORKSPACE_TOO_SMALL;
    const BlockNormBackArgs p = {dnormed, dsum, x, gate, gate_pitch, sum, weight_after, scale, weight_before, eps, frames, rows, H, dx, dgate,
                                 dresidual, sums ? static_cast<float*>(workspace) : nullptr};
    return launched(launch_block_norm_backward(p, dtype == CTC_DTYPE_BF16, dweight_after, dscale, dweight_before, stream));
}

ctc_status_t ctc_clear_frames(void* x, int pitch, const int32_t* input_lengths, int T, int B, int width, ctc_dtype_t dtype, hipStream_t stream)
{
    if (!known(dtype) || T < 1 || B < 1 || width < 1 || pitch < width) return CTC_STATUS_INVALID_VALUE;
    if (B > kMaxUtterances || static_cast<int64_t>(T) * B > kMaxRows || pitch > kMaxPitch) return CTC_STATUS_UNSUPPORTED;
    const size_t e = element(dtype);
    if (!buffers_in_order({{x, pitched(T * B, pitch, width, e), true, true, e}, {input_lengths, matrix(B, 1, 4), false}})) return CTC_STATUS_INVALID_VALUE;
    return launched(launch_clear_frames(x, pitch, input_lengths, T, B, width, dtype == CTC_DTYPE_BF16, stream));
}

ctc_status_t ctc_weights_i4_sizes(int A, int H, int group, size_t* weight_bytes_out, size_t* scale_bytes_out)
{
    if (!weight_bytes_out || !scale_bytes_out) return CTC_STATUS_INVALID_VALUE;
    const ctc_status_t st = weights_in_range(A, H, group);
    if (st != CTC_STATUS_SUCCESS) return st;
    *weight_bytes_out = weights_i4_bytes(A, H);
    *scale_bytes_out = scales_i4_bytes(A, H, group);
    return st;
}

ctc_status_t ctc_quantize_weights_i4(const void* weights, int A, int H, int group, ctc_dtype_t dtype, uint8_t* weight_q,
                                     float* weight_scales, hipStream_t stream)
{
    const ctc_status_t st = known(dtype) ? weights_in_range(A, H, group) : CTC_STATUS_INVALID_VALUE;
    if (st != CTC_STATUS_SUCCESS) return st;
    const size_t e = element(dtype);
    if (!buffers_in_order({{weights, matrix(A, H, e), false, true, e},
                           {weight_q, weights_i4_bytes(A, H), true, true, 16},
                           {weight_scales, scales_i4_bytes(A, H, group), true, true, 16}}))
        return CTC_STATUS_INVALID_VALUE;
    return launched(launch_quantize_i4(weights, A, H, group, dtype == CTC_DTYPE_BF16, weight_q, weight_scales, stream));
}

ctc_status_t ctc_dequantize_weights_i4(const uint8_t* weight_q, const float* weight_scales, int A, int H, int group, ctc_dtype_t dtype,
                                       void* out, hipStream_t stream)
{
    const ctc_status_t st = known(dtype) ? weights_in_range(A, H, group) : CTC_STATUS_INVALID_VALUE;
    if (st != CTC_STATUS_SUCCESS) return st;
    const size_t e = element(dtype);
    if (!buffers_in_order({{weight_q, weights_i4_bytes(A, H), false, true, 16},
                           {weight_scales, scales_i4_bytes(A, H, group), false, true, 16},
                           {out, matrix(A, H, e), true, true, e}}))
        return CTC_STATUS_INVALID_VALUE;
    return launched(launch_dequantize_i4(weight_q, weight_scales, A, H, group, dtype == CTC_DTYPE_BF16, out, stream));
}

ctc_status_t ctc_linear_i4(const int8_t* q, const float* scales, const uint8_t* weight_q, const float* weight_scales, int group,
                           const float* bias, const int32_t* frames, int rows, int H, int A, ctc_dtype_t dtype, void* logits,
                           hipStream_t stream)
{
    if (rows < 1 || !known(dtype)) return CTC_STATUS_INVALID_VALUE;
    const ctc_status_t st = weights_in_range(A, H, group);
    if (st != CTC_STATUS_SUCCESS) return st;
    if (rows > kMaxRows) return CTC_STATUS_UNSUPPORTED;
    const size_t e = element(dtype);
    if (!buffers_in_order({{q, matrix(rows, pitch_of(H), 1), false, true, 16},
                           {scales, matrix(rows, 1, 4), false},
                           {weight_q, weights_i4_bytes(A, H), false, true, 16},
                           {weight_scales, scales_i4_bytes(A, H, group), false, true, 16},
                           {bias, matrix(A, 1, 4), false, false},
                           {frames, list_bytes(rows), false, false},
                           {logits, matrix(rows, A, e), true, true, e}}))
        return CTC_STATUS_INVALID_VALUE;
    const LinearI4Args p = {q, scales, weight_q, weight_scales, group, groups_of(H, group), bias, frames, rows, A, pitch_of(H), logits};
    return launched(launch_linear_i4(p, dtype == CTC_DTYPE_BF16, stream));
}

}  // extern "C"
