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

// Rows to 8 bits: so many wavefronts to a row, so many elements to a lane.  16 elements a lane, and so wavefronts by the width: more elements leave
// too few wavefronts to a compute unit for what memory takes (the norm's 27200 rows of 2048 fp32 by one wavefront with 32 a lane 137 us, by two with
// 16 125; 6000 of 3500 by two with 32 50 us, by four with 16 46).  Where rows are few, 8 a lane, for the time that one row takes (one row of 2048 bf16
// 4.1 us with 16, 3.4 with 8; 1500 rows 6.9 and 6.0; 27200 rows to 8 bits 31.3 and 35.3).
struct RowShape {
    int waves, elements;
};
inline RowShape row_shape(int rows, int H)
{
    const int pitch = pitch_of(H);
    const bool few = rows <= 2048;
    if (pitch <= 512) return {1, 8};
    if (few && pitch <= 1024) return {2, 8};
    if (few && pitch <= 2048) return {4, 8};
    if (few && pitch <= 4096) return {8, 8};
    if (pitch <= 1024) return {1, 16};
    if (pitch <= 2048) return {2, 16};
    if (pitch <= 4096) return {4, 16};
    if (pitch <= 8192) return {8, 16};
    return {8, 32};                                     // (16 wavefronts with 16 a lane: the norm's 1500 rows of 12000 bf16 38 us, eight with 32 31)
}

// Activations: rows and symbols to a workgroup; 16 by 16 is the kernel without tiles in LDS.
struct ProductTile {
    int rows, symbols;
};
inline ProductTile product_tile(int all_rows, int H, int A, bool list)
{
    // Of a list's rows, five in eight are taken to count (how many do, only the GPU knows; the workspaces' sizes above and below are for all rows, since
    // they are told without a list).
    const int64_t rows = list ? (static_cast<int64_t>(all_rows) * 5 + 7) / 8 : all_rows;
    const auto tiles = [&](int m, int n) { return (rows + m - 1) / m * ((A + n - 1) / n); };
    // Tiles of 256 by 256 read the least of memory and LDS, those of 128 by 128, two of which share a compute unit, begin and end sooner: the times
    // of a round of each (us), from K = 512 and 2048 at 3000 and 19200 rows by 6000 symbols (28.7 and 389 against 40 and 326; 5560 x 4733, K = 1152:
    // 73 against 60).
    const double steps = pitch_of(H) / 64;
    const double large = static_cast<double>((tiles(256, 256) + 255) / 256) * (13.5 + 0.85 * steps);
    const double small = static_cast<double>((tiles(128, 128) + 511) / 512) * (7.0 + 0.65 * steps);
    // (By tiles alone, whatever the rows: 1 x 6000 4.5 us against 6.0 in tiles of 64 by 64, 16 x 6000 5.9 and 6.1, 32 x 6000 7.8 and 6.3.  Few rows by
    // more than 6400 symbols have not been measured.)
    if (tiles(16, 16) <= 400) return {16, 16};
    if (A <= 64 && tiles(64, 64) > 400) return {128, 64};               // 27200 x 60 14.7 us against 15.6; 5000 x 60 8.4 against 6.8
    if (tiles(64, 64) <= 600) return {64, 64};                          // 300 x 6000 10.9 us against 13.7 in 128 by 128; 1500 x 2000 (768 tiles) 11.1 and 10.8
    return small < large ? ProductTile{128, 128} : ProductTile{256, 256};
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

// One kind of tile for A symbols of H columns, and the time (us) that so many slabs of them take for so many steps of 32 rows: as many rounds of
// workgroups as the 256 compute units take (two workgroups each where tiles are narrow), each of its share of the steps and a few to begin and
// end with; every slab's sums written and read once more.
struct GradientTiles {
    int H, A, symbols, columns;
    bool wide;
    long tiles, at_once;
    double step, slab_cost;
    GradientTiles(int H_, int A_, int symbols_) : H(H_), A(A_), symbols(symbols_), columns(symbols_ == 128 ? 512 : 256), wide(symbols_ == 128)
    {
        tiles = ((A + symbols - 1L) / symbols) * ((H + columns - 1L) / columns);
        at_once = wide ? 256 : 512;
        step = wide ? 1.7 : 1.5;
        slab_cost = 8.0 * A * H / 5.0e6;
    }
    double rounds(long s) const { return static_cast<double>((tiles * s + at_once - 1) / at_once); }
    double sums(long s) const { return s > 1 ? s * slab_cost + 6.0 * step : 0.0; }
    double time(long steps, long s) const { return rounds(s) * (static_cast<double>((steps + s - 1) / s) + 6.0) * step + sums(s); }
    static long most_slabs(long steps) { return (steps + 3) / 4 < 256 ? (steps + 3) / 4 : 256; }

    GradientPlan plan(long steps, long s) const
    {
        GradientPlan p{};
        p.symbols = symbols;
        p.columns = columns;
        p.slabs = static_cast<int>(s);
        p.time = time(steps, s);
        p.bias_slabs = wide ? kColumnSlabs : p.slabs;
        p.bias_at = s > 1 ? static_cast<size_t>(s) * A * H : 0;
        p.largest_at = p.bias_at + static_cast<size_t>(p.bias_slabs) * A;
        p.wide_at = (p.largest_at + (wide ? static_cast<size_t>(kColumnSlabs) * A : 0) + 63) / 64 * 64;
        p.bytes = (p.wide_at + (wide ? static_cast<size_t>(steps) * pitch_of(H) * 16 : 0)) * 4;
        return p;
    }
    GradientPlan quickest(long steps) const
    {
        long best = 1;
        double least = time(steps, 1);
        for (long s = 2; s <= most_slabs(steps); ++s) {
            const double t = time(steps, s);
            if (t < least) {
                least = t;
                best = s;
            }
        }
        return plan(steps, best);
    }
};

// Wide tiles need a launch before theirs (the columns' largest, the rows' numbers as fp16) and are a fourth as many, each of which takes a
// third fewer products.  (Narrow and wide, us, fp32: 514 rows, 2048 wide, 172 symbols 15 and 27, 6000 symbols 59 and 52; 4000 rows,
// 1000 symbols 70 and 70; 12000 rows, 172 symbols 46 and 69, 1000 symbols 178 and 139, 6000 symbols 1035 and 662.)
constexpr double kWideLaunch = 20.0, kWideFavour = 1.1;

inline int narrow_symbols(int A) { return A <= 32 ? 32 : 64; }

inline GradientPlan gradient_plan_of_steps(long steps, int H, int A)
{
    const GradientPlan narrow = GradientTiles(H, A, narrow_symbols(A)).quickest(steps);
    if (A <= 64) return narrow;
    const GradientPlan wide = GradientTiles(H, A, 128).quickest(steps);
    return wide.time + kWideLaunch <= kWideFavour * narrow.time ? wide : narrow;
}
inline GradientPlan gradient_plan(int rows, int H, int A) { return gradient_plan_of_steps((rows + 31L) / 32, H, A); }

// The most slabs of `mine` that are chosen for any number of steps in [from, to], or a few more; 0: none ever are.  A number of slabs is chosen only
// where its time, taken low (shares of steps not rounded up), is at most that of each smaller number, taken high, and, where there are `others` (the
// tiles of the other width), `weight` times it and `extra` at most `others_weight` times theirs: each a straight line over another, which leaves an interval of steps.
inline long most_slabs_chosen(const GradientTiles& mine, long from, long to, const GradientTiles* others, double weight, double extra, double others_weight)
{
    for (long s = GradientTiles::most_slabs(to); s >= 1; --s) {
        double low = from > 4 * s - 3 ? from : 4 * s - 3, high = to;
        const double slope = mine.rounds(s) * mine.step / s, base = mine.rounds(s) * 6.0 * mine.step + mine.sums(s);
        const auto at_most = [&](const GradientTiles& t, long u, double w, double more, double v) {       // w (slope x + base) + more <= v (time of u)
            const double a = w * slope - v * t.rounds(u) * t.step / u, top = v * (t.rounds(u) * t.step * ((u - 1.0) / u + 6.0) + t.sums(u));
            const double b = top - w * base - more + 1e-9 * (top + w * base + more);                      // (a little more than rounding takes)
            if (a > 0)
                high = b / a < high ? b / a : high;
            else if (a < 0)
                low = b / a > low ? b / a : low;
            else if (b < 0)
                high = 0;
        };
        for (long u = s - 1; u >= 1 && low <= high + 1; --u) at_most(mine, u, 1.0, 0.0, 1.0);
        if (others)
            for (long u = 1; u <= s && low <= high + 1; ++u) at_most(*others, u, weight, extra, others_weight);
        if (low <= high + 1e-6 * (high + 1)) return s;
    }
    return 0;
}

// Bytes of workspace that are enough for `rows` rows and for any fewer, so that one made for the largest minibatch serves all: slabs, and the kind of
// tile, do not always grow with the rows.  Up to 64 steps each number's plan is looked at, beyond them the most slabs of either kind.
inline size_t gradient_bytes(int rows, int H, int A)
{
    constexpr long kLookedAt = 64;
    const long steps = (rows + 31L) / 32;
    size_t most = 0;
    const auto count = [&](size_t bytes) { most = bytes > most ? bytes : most; };
    for (long x = 1; x <= steps && x <= kLookedAt; ++x) count(gradient_plan_of_steps(x, H, A).bytes);
    if (steps <= kLookedAt) return most;
    const GradientTiles narrow(H, A, narrow_symbols(A)), wide(H, A, 128);
    const bool both = A > 64;
    const long n = most_slabs_chosen(narrow, kLookedAt + 1, steps, both ? &wide : nullptr, kWideFavour, -kWideLaunch, 1.0);
    const long w = both ? most_slabs_chosen(wide, kLookedAt + 1, steps, &narrow, 1.0, kWideLaunch, kWideFavour) : 0;
    if (n) count(narrow.plan(steps, n).bytes);
    if (w) count(wide.plan(steps, w).bytes);
    return most;
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
                           int A, bool bf16, const GradientPlan& plan, float* dweight, float* dbias, float* workspace, void* stream);

}  // namespace layer

#endif  // LAYER_INTERNAL_H
