// Host side of the output layer's calls: what ctc_layer.h says about arguments is checked here, then one or two
// kernels are enqueued.  Nothing is allocated, waited for or kept.

#include <cmath>

#include "layer_checks.h"
#include "layer_internal.h"

namespace layer {
namespace {

thread_local int g_last_hip_error = 0;

ctc_status_t sizes_in_range(int rows, int H, int A, ctc_dtype_t dtype)
{
    if (rows < 1 || H < 1 || A < 1) return CTC_STATUS_INVALID_VALUE;
    if (dtype != CTC_DTYPE_F32 && dtype != CTC_DTYPE_BF16) return CTC_STATUS_INVALID_VALUE;
    if (rows > kMaxRows || H > kMaxWidth || A > kMaxSymbols) return CTC_STATUS_UNSUPPORTED;
    return CTC_STATUS_SUCCESS;
}

size_t norm_workspace(int rows, int H) { return round_up(static_cast<size_t>(norm_partials(rows, H)) * H * 4); }

}  // namespace

ctc_status_t launched(int err)
{
    if (err == 0) return CTC_STATUS_SUCCESS;
    g_last_hip_error = err;
    return CTC_STATUS_HIP_ERROR;
}

}  // namespace layer

using namespace layer;

extern "C" {

int ctc_row_pitch(int H) { return H < 1 || H > kMaxWidth ? 0 : pitch_of(H); }

int ctc_layer_last_hip_error(void) { return g_last_hip_error; }

ctc_status_t ctc_pack_frames(const int32_t* input_lengths, int T, int B, int32_t* frames, hipStream_t stream)
{
    if (T < 1 || B < 1) return CTC_STATUS_INVALID_VALUE;
    if (B > 65535 || static_cast<int64_t>(T) * B > kMaxRows) return CTC_STATUS_UNSUPPORTED;
    if (!buffers_in_order({{input_lengths, matrix(B, 1, 4), false}, {frames, list_bytes(T * B), true}}))
        return CTC_STATUS_INVALID_VALUE;
    return launched(launch_pack_frames(input_lengths, T, B, frames, stream));
}

ctc_status_t ctc_quantize_rows(const void* x, const int32_t* frames, int rows, int H, ctc_dtype_t dtype, int8_t* q,
                               float* scales, hipStream_t stream)
{
    const ctc_status_t st = sizes_in_range(rows, H, 1, dtype);
    if (st != CTC_STATUS_SUCCESS) return st;
    const size_t e = element(dtype);
    if (!buffers_in_order({{x, matrix(rows, H, e), false, true, e},
                           {frames, list_bytes(rows), false, false},
                           {q, matrix(rows, pitch_of(H), 1), true, true, 16},
                           {scales, matrix(rows, 1, 4), true}}))
        return CTC_STATUS_INVALID_VALUE;
    return launched(launch_quantize(x, frames, rows, H, dtype == CTC_DTYPE_BF16, q, scales, stream));
}

ctc_status_t ctc_dequantize_rows(const int8_t* q, const float* scales, const int32_t* frames, int rows, int H,
                                 ctc_dtype_t dtype, void* out, hipStream_t stream)
{
    const ctc_status_t st = sizes_in_range(rows, H, 1, dtype);
    if (st != CTC_STATUS_SUCCESS) return st;
    const size_t e = element(dtype);
    if (!buffers_in_order({{q, matrix(rows, pitch_of(H), 1), false, true, 16},
                           {scales, matrix(rows, 1, 4), false},
                           {frames, list_bytes(rows), false, false},
                           {out, matrix(rows, H, e), true, true, e}}))
        return CTC_STATUS_INVALID_VALUE;
    return launched(launch_dequantize(q, scales, frames, rows, H, dtype == CTC_DTYPE_BF16, out, stream));
}

ctc_status_t ctc_rms_norm_i8(const void* x, const void* residual, const float* weight, float eps, const int32_t* frames,
                             int rows, int H, ctc_dtype_t dtype, void* sum, int8_t* q, float* scales, hipStream_t stream)
{
    const ctc_status_t st = sizes_in_range(rows, H, 1, dtype);
    if (st != CTC_STATUS_SUCCESS) return st;
    if (!std::isfinite(eps) || eps <= 0.0f) return CTC_STATUS_INVALID_VALUE;
    const size_t e = element(dtype), states = matrix(rows, H, e);
    if (!buffers_in_order({{x, states, false, true, e, true},
                           {residual, states, false, false, e, true},
                           {weight, matrix(H, 1, 4), false, false},
                           {frames, list_bytes(rows), false, false},
                           {sum, states, true, false, e, false, true},
                           {q, matrix(rows, pitch_of(H), 1), true, true, 16},
                           {scales, matrix(rows, 1, 4), true}}))
        return CTC_STATUS_INVALID_VALUE;
    return launched(launch_norm(x, residual, weight, eps, frames, rows, H, dtype == CTC_DTYPE_BF16, sum, q, scales, stream));
}

ctc_status_t ctc_rms_norm_workspace_size(int rows, int H, size_t* bytes_out)
{
    if (!bytes_out) return CTC_STATUS_INVALID_VALUE;
    const ctc_status_t st = sizes_in_range(rows, H, 1, CTC_DTYPE_F32);
    if (st == CTC_STATUS_SUCCESS) *bytes_out = norm_workspace(rows, H);
    return st;
}

ctc_status_t ctc_rms_norm_backward(const void* dy, const void* sum, const float* weight, float eps, const void* dresidual,
                                   const int32_t* frames, int rows, int H, ctc_dtype_t dtype, void* dsum, float* dweight,
                                   void* workspace, size_t workspace_bytes, hipStream_t stream)
{
    const ctc_status_t st = sizes_in_range(rows, H, 1, dtype);
    if (st != CTC_STATUS_SUCCESS) return st;
    if (!std::isfinite(eps) || eps <= 0.0f) return CTC_STATUS_INVALID_VALUE;
    const size_t e = element(dtype), states = matrix(rows, H, e), needed = norm_workspace(rows, H);
    if (!buffers_in_order({{dy, states, false, true, e, true},
                           {sum, states, false, true, e, true},
                           {dresidual, states, false, false, e, true},
                           {weight, matrix(H, 1, 4), false, false},
                           {frames, list_bytes(rows), false, false},
                           {dsum, states, true, true, e, false, true},
                           {dweight, matrix(H, 1, 4), true, false},
                           {dweight ? workspace : nullptr, needed, true, dweight != nullptr, 256}}))
        return CTC_STATUS_INVALID_VALUE;
    if (dweight && workspace_bytes < needed) return CTC_STATUS_WORKSPACE_TOO_SMALL;
    return launched(launch_norm_backward(dy, sum, weight, eps, dresidual, frames, rows, H, dtype == CTC_DTYPE_BF16, dsum,
                                         dweight, static_cast<float*>(workspace), stream));
}

ctc_status_t ctc_linear_i8(const int8_t* q, const float* scales, const int8_t* weight_q, const float* weight_scales,
                           const float* bias, const int32_t* frames, int rows, int H, int A, ctc_dtype_t dtype, void* logits,
                           hipStream_t stream)
{
    const ctc_status_t st = sizes_in_range(rows, H, A, dtype);
    if (st != CTC_STATUS_SUCCESS) return st;
    const size_t e = element(dtype);
    if (!buffers_in_order({{q, matrix(rows, pitch_of(H), 1), false, true, 16},
                           {scales, matrix(rows, 1, 4), false},
                           {weight_q, matrix(A, pitch_of(H), 1), false, true, 16},
                           {weight_scales, matrix(A, 1, 4), false},
                           {bias, matrix(A, 1, 4), false, false},
                           {frames, list_bytes(rows), false, false},
                           {logits, matrix(rows, A, e), true, true, e}}))
        return CTC_STATUS_INVALID_VALUE;
    return launched(launch_linear(q, scales, weight_q, weight_scales, bias, frames, rows, H, A, dtype == CTC_DTYPE_BF16,
                                  logits, stream));
}

ctc_status_t ctc_weight_gradient_workspace_size(int rows, int H, int A, size_t* bytes_out)
{
    if (!bytes_out) return CTC_STATUS_INVALID_VALUE;
    const ctc_status_t st = sizes_in_range(rows, H, A, CTC_DTYPE_F32);
    if (st == CTC_STATUS_SUCCESS) *bytes_out = round_up(gradient_bytes(rows, H, A));
    return st;
}

ctc_status_t ctc_weight_gradient_i8(const void* grads, const int8_t* q, const float* scales, const int32_t* frames, int rows,
                                    int H, int A, ctc_dtype_t dtype, float* dweight, float* dbias, void* workspace,
                                    size_t workspace_bytes, hipStream_t stream)
{
    const ctc_status_t st = sizes_in_range(rows, H, A, dtype);
    if (st != CTC_STATUS_SUCCESS) return st;
    const GradientPlan plan = gradient_plan(rows, H, A);
    const size_t e = element(dtype), needed = round_up(plan.bytes);
    if (!buffers_in_order({{grads, matrix(rows, A, e), false, true, e},
                           {q, matrix(rows, pitch_of(H), 1), false, true, 16},
                           {scales, matrix(rows, 1, 4), false},
                           {frames, list_bytes(rows), false, false},
                           {dweight, matrix(A, H, 4), true},
                           {dbias, matrix(A, 1, 4), true, false},
                           {workspace, needed, true, true, 256}}))
        return CTC_STATUS_INVALID_VALUE;
    if (workspace_bytes < needed) return CTC_STATUS_WORKSPACE_TOO_SMALL;
    return launched(launch_weight_gradient(grads, q, scales, frames, rows, H, A, dtype == CTC_DTYPE_BF16, plan, dweight, dbias,
                                           static_cast<float*>(workspace), stream));
}

}  // extern "C"
