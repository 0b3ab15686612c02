// Kernels of weights in 4 bits (ctc_block.h).

#include <hip/hip_runtime.h>

#include "layer_block_internal.h"
#include "layer_rows.h"

namespace layer {
namespace {

// A row's 128 columns of one of the weights' tiles are sixteen threads': thread j has columns 4 j .. + 3, which are the low halves of its four
// bytes, and columns 64 + 4 j .. + 3, the high ones.
struct Eight {
    float low[4], high[4];
};
template <typename T> __device__ __forceinline__ Eight load_eight(const T* row, int col, int H)
{
    Eight e;
    T low[4], high[4];
    if (col + 68 <= H) {
        __builtin_memcpy(low, row + col, sizeof(low));
        __builtin_memcpy(high, row + col + 64, sizeof(high));
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            low[k] = col + k < H ? row[col + k] : narrow<T>(0.0f);
            high[k] = col + 64 + k < H ? row[col + 64 + k] : narrow<T>(0.0f);
        }
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        e.low[k] = widen(low[k]);
        e.high[k] = widen(high[k]);
    }
    return e;
}
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }
__device__ __forceinline__ uint32_t largest(const float (&v)[4])
{
    uint32_t most = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint32_t a = magnitude(v[k]);
        most = most > a ? most : a;
    }
    return most;
}
// Of sixteen threads' numbers.
__device__ __forceinline__ uint32_t largest_of_16(uint32_t v)
{
#pragma unroll
    for (int d = 8; d; d >>= 1) {
        const uint32_t o = __shfl_xor(v, d, kWave);
        v = v > o ? v : o;
    }
    return v;
}

// What rounds a group's values: its largest, lifted where that is tiny (which is exact), and seven over it.
struct Rounding {
    float lift, m, inverse;
    bool finite;
};
__device__ __forceinline__ Rounding rounding_of(uint32_t most)
{
    Rounding r;
    r.finite = most < kInfinity;
    r.lift = most < 0x20000000u ? 0x1p80f : 1.0f;
    r.m = __uint_as_float(most) * r.lift;
    r.inverse = most && r.finite ? static_cast<float>(7.0 / static_cast<double>(r.m)) : 0.0f;
    return r;
}
__device__ __forceinline__ uint32_t nibble(float v, const Rounding& r)
{
    return r.finite ? static_cast<uint32_t>(level<7>(v * r.lift, r.m, r.inverse)) & 15u : 0u;
}
__device__ __forceinline__ float scale_of(uint32_t most)
{
    return most < kInfinity ? static_cast<float>(static_cast<double>(__uint_as_float(most)) / 7.0) : __uint_as_float(0x7fc00000u);
}

// Sixteen rows, and as many columns as a scale has (128 where that is 64), to a workgroup.
template <typename T>
__global__ __launch_bounds__(256) void ctc_quantize_weights_i4_kernel(const T* __restrict__ weights, int A, int H, int group, int groups,
                                                                      int tiles, uint8_t* __restrict__ weight_q,
                                                                      float* __restrict__ weight_scales)
{
    const int r = threadIdx.x / 16, j = threadIdx.x % 16;
    const int64_t units = group == 64 ? tiles : groups;
    const int64_t at = group_number(), row_tile = at / units;
    const int unit = static_cast<int>(at % units);
    if (row_tile >= (A + 15) / 16) return;
    const int64_t a = row_tile * 16 + r;
    const int reach = group == 64 ? 1 : group / 128, first = unit * reach, last = first + reach < tiles ? first + reach : tiles;
    const T* const row = weights + a * H;
    Eight e{};
    uint32_t low = 0, high = 0;
    for (int t = first; t < last; ++t) {
        if (a < A) e = load_eight(row, t * 128 + 4 * j, H);
        const uint32_t l = largest(e.low), h = largest(e.high);
        low = low > l ? low : l;
        high = high > h ? high : h;
    }
    low = largest_of_16(low);
    high = largest_of_16(high);
    if (group != 64) low = high = low > high ? low : high;
    const Rounding by_low = rounding_of(low), by_high = rounding_of(high);
    for (int t = first; t < last; ++t) {
        if (reach > 1 && a < A) e = load_eight(row, t * 128 + 4 * j, H);           // (from the caches)
        uint32_t word = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) word |= (nibble(e.low[k], by_low) | nibble(e.high[k], by_high) << 4) << (8 * k);
        __builtin_memcpy(__builtin_assume_aligned(weight_q + ((row_tile * tiles + t) * kTileBytes + 256 * (j / 4) + 16 * r + 4 * (j % 4)), 4), &word, 4);
    }
    if (j) return;
    float* const scales = weight_scales + row_tile * groups * 16 + r;
    if (group == 64) {
        scales[static_cast<int64_t>(2 * unit) * 16] = scale_of(low);
        if (2 * unit + 1 < groups) scales[static_cast<int64_t>(2 * unit + 1) * 16] = scale_of(high);
    } else {
        scales[static_cast<int64_t>(unit) * 16] = scale_of(low);
    }
}

template <typename T>
__global__ __launch_bounds__(256) void ctc_dequantize_weights_i4_kernel(const uint8_t* __restrict__ weight_q, const float* __restrict__ weight_scales,
                                                                        int A, int H, int group, int groups, int tiles, T* __restrict__ out)
{
    const int r = threadIdx.x / 16, j = threadIdx.x % 16;
    const int64_t at = group_number(), row_tile = at / tiles;
    const int t = static_cast<int>(at % tiles);
    const int64_t a = row_tile * 16 + r;
    if (a >= A) return;
    uint32_t word;
    __builtin_memcpy(&word, __builtin_assume_aligned(weight_q + at * kTileBytes + 256 * (j / 4) + 16 * r + 4 * (j % 4), 4), 4);
    const int col = t * 128 + 4 * j;
    const float* const scales = weight_scales + row_tile * groups * 16 + r;
    const int g_low = col / group, g_high = (col + 64) / group;
    const float low = scales[static_cast<int64_t>(g_low) * 16], high = g_high < groups ? scales[static_cast<int64_t>(g_high) * 16] : 0.0f;
    T l[4], h[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        l[k] = narrow<T>(static_cast<float>(static_cast<int32_t>(word << (28 - 8 * k)) >> 28) * low);
        h[k] = narrow<T>(static_cast<float>(static_cast<int32_t>(word << (24 - 8 * k)) >> 28) * high);
    }
    T* const to = out + a * H + col;
    if (col + 68 <= H) {
        store_past<sizeof(l)>(to, l);
        store_past<sizeof(h)>(to + 64, h);
        return;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if (col + k < H) to[k] = l[k];
        if (col + 64 + k < H) to[64 + k] = h[k];
    }
}

// What a wavefront's lanes have written to LDS is there for its other lanes: its accesses are in order, if the compiler leaves them so.
__device__ __forceinline__ void in_order()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

typedef int int4v __attribute__((ext_vector_type(4)));
typedef float float4v __attribute__((ext_vector_type(4)));

// RT by ST tiles of 16 rows by 16 symbols to a workgroup, each of whose wavefronts takes every WAVES-th 128 columns of all of them, straight from memory
// into the matrix cores, the next ones asked for before these are multiplied; their sums are added in LDS.  A weight's four bits become the upper half
// of a byte, sixteen times their value: that takes one `and` (and a shift for the lower half) for four weights, and a sixteenth comes into the row's scale.
// (64 rows by 32 symbols: three wavefronts to a SIMD, by 64 symbols two; 256 x 2048 by 6144 bf16 13.7 us a pass, 16.8.)
// v_mfma_i32_16x16x64_i8: lane l gives bytes 16 (l / 16) .. of row l % 16 of either operand, and holds rows 4 (l / 16) .. + 3 of column
// l % 16 of the result.
template <typename T, int RT, int ST, int WAVES, bool BY_64>
__global__ __launch_bounds__(WAVES * kWave, RT * ST >= 8 ? 3 : 1) void ctc_linear_i4_kernel(LinearI4Args p)
{
    constexpr int kColumns = 16 * ST, kThreads = WAVES * kWave;
    constexpr bool kTurned = RT > 1;                                              // (of one tile of rows the few that count are soon read)
    constexpr int kSumBytes = WAVES * 16 * RT * kColumns * 4, kRowBytes = kTurned ? WAVES * RT * 16 * kTileColumns : 0;
    __shared__ int4v s_quads[(kSumBytes > kRowBytes ? kSumBytes : kRowBytes) / 16];
    __shared__ int s_row[16 * RT];
    float (*const s_sum)[16 * RT][kColumns] = reinterpret_cast<float (*)[16 * RT][kColumns]>(s_quads);
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const unsigned across = static_cast<unsigned>((p.A + kColumns - 1) / kColumns), group = static_cast<unsigned>(group_number());
    const int64_t m0 = static_cast<int64_t>(group / across) * (16 * RT);
    const int n0 = static_cast<int>(group % across) * ST;                         // in tiles of 16 symbols
    if (m0 >= p.rows) return;
    const int tiles = p.pitch / kTileColumns, last_tile = (p.A + 15) / 16 - 1;
    const uint8_t* w[ST];
    const float* scale[ST];
#pragma unroll
    for (int s = 0; s < ST; ++s) {
        const int64_t tile = n0 + s < last_tile ? n0 + s : last_tile;
        w[s] = p.weight_q + tile * tiles * kTileBytes + 16 * lane;
        scale[s] = p.weight_scales + tile * p.groups * 16 + lane % 16;
    }
    // A row's 128 bytes are brought by eight neighbouring lanes (16 rows' same 16 bytes, as the matrix cores take them, are 16 lines of memory to a quarter of a
    // wavefront: 256 x 2048 by 6144 bf16 17.4 us on the GPU) and turned over in the wavefront's own part of LDS, chunk c of row r at chunk c ^ r % 8.
    constexpr int kLoads = 2 * RT;
    const int8_t* q[kLoads];
    struct Columns {
        int4v q[kLoads], w[ST];
        float by[ST], by_high[ST];
    } here, next;
    const auto weights = [&](int t, Columns& to) {
        const int g = BY_64 ? 2 * t : t * kTileColumns / p.group;
#pragma unroll
        for (int s = 0; s < ST; ++s) {
            __builtin_memcpy(&to.w[s], __builtin_assume_aligned(w[s] + static_cast<int64_t>(t) * kTileBytes, 16), 16);
            to.by[s] = scale[s][static_cast<int64_t>(g) * 16];
            if constexpr (BY_64) to.by_high[s] = scale[s][static_cast<int64_t>(g + 1 < p.groups ? g + 1 : g) * 16];      // (behind the last group the weights are zeros)
        }
    };
    const auto rows = [&](int t, Columns& to) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i)
            __builtin_memcpy(&to.q[i], __builtin_assume_aligned(q[i] + t * kTileColumns + (kTurned ? 0 : 64 * i), 16), 16);
    };
    // (the weights wait for nothing, the rows for the list)
    if (wave < tiles) weights(wave, next);
    // One lane asks the list for each row.
    const int asked = row_at(p.frames, p.rows, m0 + lane % (16 * RT));
    if (wave == 0 && lane < 16 * RT) s_row[lane] = asked;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        const int r = kTurned ? __shfl(asked, 8 * i + lane / 8, kWave) : asked;
        q[i] = p.q + static_cast<int64_t>(r < 0 ? 0 : r) * p.pitch + 16 * (kTurned ? lane % 8 : lane / 16);          // (what row 0 gives instead is not written)
    }
    // (in pieces of 16 bytes, eight to a row)
    const int mine = wave * (kRowBytes / WAVES / 16), to_lds = mine + lane / 8 * 8 + (lane % 8 ^ lane / 8);
    const int from_low = mine + lane % 16 * 8 + (lane / 16 ^ lane % 8), from_high = mine + lane % 16 * 8 + ((lane / 16 + 4) ^ lane % 8);
    if (wave < tiles) rows(wave, next);
    float4v sum[RT][ST];
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int s = 0; s < ST; ++s) sum[i][s] = float4v{};
    for (int t = wave; t < tiles; t += WAVES) {
        here = next;
        if (t + WAVES < tiles) {
            weights(t + WAVES, next);
            rows(t + WAVES, next);
        }
        __builtin_amdgcn_sched_barrier(0);
        int4v low[RT], high[RT];
        if constexpr (kTurned) {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) s_quads[to_lds + i * 64] = here.q[i];
            in_order();
#pragma unroll
            for (int i = 0; i < RT; ++i) {
                low[i] = s_quads[from_low + i * 128];
                high[i] = s_quads[from_high + i * 128];
            }
            in_order();
        } else {
            low[0] = here.q[0];
            high[0] = here.q[1];
        }
#pragma unroll
        for (int s = 0; s < ST; ++s) {
            const int4v w_low = here.w[s] << 4 & static_cast<int>(0xf0f0f0f0u), w_high = here.w[s] & static_cast<int>(0xf0f0f0f0u);
#pragma unroll
            for (int i = 0; i < RT; ++i) {
                int4v a = __builtin_amdgcn_mfma_i32_16x16x64_i8(low[i], w_low, int4v{}, 0, 0, 0);
                if constexpr (BY_64) {
                    const int4v b = __builtin_amdgcn_mfma_i32_16x16x64_i8(high[i], w_high, int4v{}, 0, 0, 0);
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        sum[i][s][k] = fmaf(static_cast<float>(b[k]), here.by_high[s], fmaf(static_cast<float>(a[k]), here.by[s], sum[i][s][k]));
                } else {
                    a = __builtin_amdgcn_mfma_i32_16x16x64_i8(high[i], w_high, a, 0, 0, 0);
#pragma unroll
                    for (int k = 0; k < 4; ++k) sum[i][s][k] = fmaf(static_cast<float>(a[k]), here.by[s], sum[i][s][k]);
                }
            }
        }
    }
    if constexpr (kTurned) __syncthreads();                                       // (the sums take the rows' place)
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int s = 0; s < ST; ++s)
#pragma unroll
            for (int k = 0; k < 4; ++k) s_sum[wave][16 * i + 4 * (lane / 16) + k][16 * s + lane % 16] = sum[i][s][k];
    __syncthreads();
    for (int at = threadIdx.x; at < 16 * RT * kColumns; at += kThreads) {
        const int i = at / kColumns, j = at % kColumns, r = s_row[i];
        const int64_t a = static_cast<int64_t>(n0) * 16 + j;
        if (r < 0 || a >= p.A) continue;
        float v = s_sum[0][i][j];
#pragma unroll
        for (int o = 1; o < WAVES; ++o) v += s_sum[o][i][j];
        static_cast<T*>(p.logits)[static_cast<int64_t>(r) * p.A + a] = narrow<T>(fmaf(v, p.scales[r] * 0.0625f, p.bias ? p.bias[a] : 0.0f));
    }
}

template <typename T, int RT, int ST, int WAVES> int launch_i4_tile(const LinearI4Args& p, hipStream_t s)
{
    const dim3 grid = spread(blocks(p.rows, 16 * RT) * blocks(p.A, 16 * ST));
    return p.group == 64 ? launch(ctc_linear_i4_kernel<T, RT, ST, WAVES, true>, grid, WAVES * kWave, s, p)
                         : launch(ctc_linear_i4_kernel<T, RT, ST, WAVES, false>, grid, WAVES * kWave, s, p);
}

template <typename T> int launch_linear_of(const LinearI4Args& p, hipStream_t s)
{
    switch (i4_tile(p.rows, p.pitch, p.A)) {
    case I4Tile::k16x16: return launch_i4_tile<T, 1, 1, 4>(p, s);
    case I4Tile::k16x16Deep: return launch_i4_tile<T, 1, 1, 16>(p, s);
    case I4Tile::k32x16: return launch_i4_tile<T, 2, 1, 8>(p, s);
    case I4Tile::k64x16: return launch_i4_tile<T, 4, 1, 8>(p, s);
    default: return launch_i4_tile<T, 4, 2, 4>(p, s);
    }
}

}  // namespace

int launch_quantize_i4(const void* weights, int A, int H, int group, bool bf16, uint8_t* weight_q, float* weight_scales, void* stream)
{
    hipStream_t s = static_cast<hipStream_t>(stream);
    const int tiles = pitch_of(H) / kTileColumns, groups = groups_of(H, group);
    const dim3 grid = spread(blocks(A, 16) * static_cast<unsigned>(group == 64 ? tiles : groups));
    if (bf16) return launch(ctc_quantize_weights_i4_kernel<bf16_t>, grid, 256, s, static_cast<const bf16_t*>(weights), A, H, group, groups, tiles, weight_q, weight_scales);
    return launch(ctc_quantize_weights_i4_kernel<float>, grid, 256, s, static_cast<const float*>(weights), A, H, group, groups, tiles, weight_q, weight_scales);
}

int launch_dequantize_i4(const uint8_t* weight_q, const float* weight_scales, int A, int H, int group, bool bf16, void* out, void* stream)
{
    hipStream_t s = static_cast<hipStream_t>(stream);
    const int tiles = pitch_of(H) / kTileColumns, groups = groups_of(H, group);
    const dim3 grid = spread(blocks(A, 16) * static_cast<unsigned>(tiles));
    if (bf16) return launch(ctc_dequantize_weights_i4_kernel<bf16_t>, grid, 256, s, weight_q, weight_scales, A, H, group, groups, tiles, static_cast<bf16_t*>(out));
    return launch(ctc_dequantize_weights_i4_kernel<float>, grid, 256, s, weight_q, weight_scales, A, H, group, groups, tiles, static_cast<float*>(out));
}

int launch_linear_i4(const LinearI4Args& p, bool bf16, void* stream)
{
    hipStream_t s = static_cast<hipStream_t>(stream);
    return bf16 ? launch_linear_of<bf16_t>(p, s) : launch_linear_of<float>(p, s);
}

}  // namespace layer
