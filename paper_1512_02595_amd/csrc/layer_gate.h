// Sigmoids, for the recurrence's gates and the blocks' (device code).
#ifndef LAYER_GATE_H
#define LAYER_GATE_H

#include <hip/hip_runtime.h>

namespace layer {
namespace {

// z = 1 / (1 + exp(-g)) and 1 - z, each to a few units of its own last place: from exp(-|g|), which does not overflow, both
// are a quotient without a difference.  The exponent is a product in two parts, so that it is good to a last place of the
// result, not of itself.  An infinite g gives 0 and 1, a NaN NaNs.
struct Gate {
    float z, stays;
};
__device__ __forceinline__ Gate gate_of(float g)
{
    constexpr float kLog2e = 0x1.715476p+0f, kRest = 0x1.4ae0cp-26f, kLn2 = 0x1.62e430p-1f;
    float a = fabsf(g);
    a = a > 150.0f ? 150.0f : a;                                        // (exp(-150) is 0 here; an infinity would make the rest a NaN)
    const float whole = -a * kLog2e, rest = fmaf(-a, kLog2e, -whole) - a * kRest;
    const float power = __builtin_amdgcn_exp2f(whole);
    const float t = fmaf(power, rest * kLn2, power);                    // exp(-|g|)
    const float large = __builtin_amdgcn_rcpf(1.0f + t), small = t * large;
    const bool up = g >= 0.0f;
    return {up ? large : small, up ? small : large};
}

}  // namespace
}  // namespace layer

#endif  // LAYER_GATE_H
