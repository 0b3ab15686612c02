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

// The norm's backward pass: so many workgroups leave a partial sum of dweight each; they take one turn of rows (four rows at once up to
// 1024 wide) or two.  (300 rows of 1024 bf16: one turn of four 6.6 us, two 7.4; 300 of 2048: two rows 8.0, four 9.1; 27200 of 1024 fp32: 1024
// workgroups 57.2, 2048 59.6.)
inline int norm_partials(int rows, int H)
{
    const int per_group = H <= 1024 ? 4 : 2;
    const int groups = (rows + per_group - 1) / per_group;
    return groups < 1024 ? groups : 1024;
}

// The weights' gradient: symbols and columns in tiles, the listed rows dealt out to so many slabs, each summed by workgroups
// of its own.
constexpr int kColumnSlabs = 64;                // workgroups that look at one symbol's gradients first
struct GradientPlan {
    int symbols, columns;                       // of a tile: 32 or 64 by 256, 128 by 512
    int slabs;
    double time;                                // a guess, for choices
    int bias_slabs;
    size_t bias_at, largest_at, wide_at, bytes; // places in the workspace, in floats; all of it, in bytes
};
inline GradientPlan gradient_plan(int rows, int H, int A)
{
    const long steps = (rows + 31L) / 32;
    const auto plan = [&](int symbols) {
        GradientPlan p{};
        const bool wide = symbols == 128;
        p.symbols = symbols;
        p.columns = wide ? 512 : 256;
        const long tiles = ((A + symbols - 1L) / symbols) * ((H + p.columns - 1L) / p.columns);
        // Time (us): as many rounds of workgroups as the 256 compute units take (two workgroups each where tiles are narrow), each of its share of the
        // steps of 32 rows and a few to begin and end with; every slab's sums written and read once more.
        const long at_once = wide ? 256 : 512;
        const double step = wide ? 1.7 : 1.5, slab_cost = 8.0 * A * H / 5.0e6;
        for (long s = 1; s <= 256 && s <= (steps + 3) / 4; ++s) {
            const long rounds = (tiles * s + at_once - 1) / at_once;
            const double time = static_cast<double>(rounds) * (static_cast<double>((steps + s - 1) / s) + 6.0) * step + (s > 1 ? s * slab_cost + 6.0 * step : 0.0);
            if (s == 1 || time < p.time) {
                p.time = time;
                p.slabs = static_cast<int>(s);
            }
        }
        return p;
    };
    GradientPlan p = plan(A <= 32 ? 32 : 64);
    if (A > 64) {
        // Wide tiles need a launch before theirs (the columns' largest, the rows' numbers as fp16) and are a fourth as many, each of which takes a
        // third fewer products.  (Narrow and wide, us, fp32: 514 rows, 2048 wide, 172 symbols 15 and 27, 6000 symbols 59 and 52; 4000 rows,
        // 1000 symbols 70 and 70; 12000 rows, 172 symbols 46 and 69, 1000 symbols 178 and 139, 6000 symbols 1035 and 662.)
        const GradientPlan wide = plan(128);
        if (wide.time + 20.0 <= 1.1 * p.time) p = wide;
    }
    const bool wide = p.symbols == 128;
    p.bias_slabs = wide ? kColumnSlabs : p.slabs;
    p.bias_at = p.slabs > 1 ? static_cast<size_t>(p.slabs) * A * H : 0;
    p.largest_at = p.bias_at + static_cast<size_t>(p.bias_slabs) * A;
    p.wide_at = (p.largest_at + (wide ? static_cast<size_t>(kColumnSlabs) * A : 0) + 63) / 64 * 64;
    p.bytes = (p.wide_at + (wide ? static_cast<size_t>(steps) * pitch_of(H) * 16 : 0)) * 4;
    return p;
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
