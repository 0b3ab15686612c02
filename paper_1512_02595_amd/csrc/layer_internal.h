// What the host side of the output layer's calls (layer_api.cpp) and their kernels (layer_kernels.hip) share.
#ifndef LAYER_INTERNAL_H
#define LAYER_INTERNAL_H

#include <cstddef>
#include <cstdint>

#include "ctc_layer.h"

namespace layer {

constexpr int kPitch = 128;                     // rows in 8 bits lie a multiple of this apart
constexpr int kMaxWidth = CTC_MAX_STATE_WIDTH;
constexpr int kMaxRows = 1 << 30;
constexpr int kMaxSymbols = 1 << 20;

inline int pitch_of(int H) { return (H + kPitch - 1) / kPitch * kPitch; }

// The norm's backward pass: so many workgroups leave a partial sum of dweight each.
inline int norm_partials(int rows)
{
    constexpr int kRowsOfGroup = 8;
    const int groups = (rows + kRowsOfGroup - 1) / kRowsOfGroup;
    return groups < 1024 ? groups : 1024;
}

// The weights' gradient: the listed rows are dealt out to so many slabs, each summed by workgroups of its own.
inline int gradient_slabs(int rows, int H, int A)
{
    const long tiles = ((H + 63L) / 64) * ((A + 63L) / 64);
    long slabs = (2048 + tiles - 1) / tiles;
    const long most = (rows + 255L) / 256;
    if (slabs > most) slabs = most;
    return static_cast<int>(slabs < 1 ? 1 : slabs > 256 ? 256 : slabs);
}

// Every launch returns a hipError_t.
int launch_pack_frames(const int32_t* lengths, int T, int B, int32_t* frames, void* stream);
int launch_quantize(const void* x, const int32_t* frames, int rows, int H, bool bf16, int8_t* q, float* scales, void* stream);
int launch_dequantize(const int8_t* q, const float* scales, const int32_t* frames, int rows, int H, bool bf16, void* out,
                      void* stream);
int launch_norm(const void* x, const void* residual, const float* weight, float eps, const int32_t* frames, int rows, int H,
                bool bf16, void* sum, int8_t* q, float* scales, void* stream);
int launch_norm_backward(const void* dy, const void* sum, const float* weight, float eps, const void* dresidual,
                         const int32_t* frames, int rows, int H, bool bf16, void* dsum, float* dweight, float* partials,
                         void* stream);
int launch_linear(const int8_t* q, const float* scales, const int8_t* weight_q, const float* weight_scales, const float* bias,
                  const int32_t* frames, int rows, int H, int A, bool bf16, void* logits, void* stream);
int launch_weight_gradient(const void* grads, const int8_t* q, const float* scales, const int32_t* frames, int rows, int H,
                           int A, bool bf16, float* dweight, float* dbias, float* partials, void* stream);

}  // namespace layer

#endif  // LAYER_INTERNAL_H
