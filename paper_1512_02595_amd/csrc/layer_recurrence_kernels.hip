// Kernels of the gated linear recurrence (ctc_block.h).

#include <hip/hip_runtime.h>

#include "layer_block_internal.h"
#include "layer_gate.h"
#include "layer_rows.h"

namespace layer {
namespace {

__device__ __forceinline__ int length_of(const int32_t* lengths, int b, int T)
{
    if (!lengths) return T;
    const int n = lengths[b];
    return n < 0 ? 0 : n > T ? T : n;
}

// A channel of an utterance to a thread, frame after frame.
template <typename T> __global__ __launch_bounds__(256) void ctc_recurrence_kernel(RecurrenceArgs p)
{
    const int64_t i = group_number() * 256 + threadIdx.x;
    if (i >= static_cast<int64_t>(p.B) * p.H) return;
    const int b = static_cast<int>(i / p.H), k = static_cast<int>(i % p.H), n = length_of(p.lengths, b, p.T);
    double h = p.initial ? static_cast<double>(p.initial[i]) : 0.0;
    for (int s = 0; s < n; ++s) {
        const int64_t row = static_cast<int64_t>(k < p.forward ? s : n - 1 - s) * p.B + b;
        const T* in = static_cast<const T*>(p.inputs) + row * p.pitch + k;
        h = fma(static_cast<double>(gate_of(widen(in[0])).z), static_cast<double>(widen(in[p.H])) - h, h);
        static_cast<T*>(p.out)[row * p.H + k] = narrow<T>(static_cast<float>(h));
    }
    if (p.last) p.last[i] = static_cast<float>(h);
}

template <typename T> __global__ __launch_bounds__(256) void ctc_recurrence_backward_kernel(RecurrenceArgs p)
{
    const int64_t i = group_number() * 256 + threadIdx.x;
    if (i >= static_cast<int64_t>(p.B) * p.H) return;
    const int b = static_cast<int>(i / p.H), k = static_cast<int>(i % p.H), n = length_of(p.lengths, b, p.T);
    double d = p.dfinal ? static_cast<double>(p.dfinal[i]) : 0.0;
    for (int s = n - 1; s >= 0; --s) {
        const int64_t row = static_cast<int64_t>(k < p.forward ? s : n - 1 - s) * p.B + b;
        const int64_t before = row + (k < p.forward ? -p.B : p.B);
        const T* in = static_cast<const T*>(p.inputs) + row * p.pitch + k;
        const Gate g = gate_of(widen(in[0]));
        const float h = s ? widen(static_cast<const T*>(p.states_in)[before * p.H + k]) : p.initial ? p.initial[i] : 0.0f;
        d += static_cast<double>(widen(static_cast<const T*>(p.dstates)[row * p.H + k]));
        const float whole = static_cast<float>(d);
        T* out = static_cast<T*>(p.out) + row * p.pitch + k;
        out[0] = narrow<T>(whole * (widen(in[p.H]) - h) * (g.z * g.stays));
        out[p.H] = narrow<T>(whole * g.z);
        d *= 1.0 - static_cast<double>(g.z);
    }
    if (p.last) p.last[i] = static_cast<float>(d);
}

}  // namespace

int launch_recurrence(const RecurrenceArgs& p, bool bf16, bool backward, void* stream)
{
    hipStream_t s = static_cast<hipStream_t>(stream);
    const dim3 grid = spread(blocks(static_cast<int64_t>(p.B) * p.H, 256));
    if (backward) return bf16 ? launch(ctc_recurrence_backward_kernel<bf16_t>, grid, 256, s, p) : launch(ctc_recurrence_backward_kernel<float>, grid, 256, s, p);
    return bf16 ? launch(ctc_recurrence_kernel<bf16_t>, grid, 256, s, p) : launch(ctc_recurrence_kernel<float>, grid, 256, s, p);
}

}  // namespace layer
