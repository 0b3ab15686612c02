// Kernels of the output layer held in 8 bits (ctc_layer.h).

#include <hip/hip_runtime.h>

#include <tuple>
#include <type_traits>

#include "layer_internal.h"

namespace layer {
namespace {

constexpr int kWave = 64;

// ---- elements ---------------------------------------------------------------------------------------------------

struct bf16_t { uint16_t bits; };

__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ float widen(bf16_t v) { return __uint_as_float(static_cast<uint32_t>(v.bits) << 16); }

// To the nearest, ties to even; a NaN stays one.
template <typename T> __device__ __forceinline__ T narrow(float v);
template <> __device__ __forceinline__ float narrow<float>(float v) { return v; }
template <> __device__ __forceinline__ bf16_t narrow<bf16_t>(float v)
{
    return {__builtin_bit_cast(uint16_t, static_cast<__bf16>(v))};
}

// Bytes of rows that nobody reads soon are written past the caches: they would take the place of what is being read, and a cache that has to let
// go of old lines to take new ones slows both.  28 900 of 48 000 rows of 2048 bf16: from 8 bits 43 us -> 27.5, the norm 91 -> 80.  (The partial sums
// of the norm's gradient take the same way, though the launch behind reads them at once; kept in the caches they have not been measured.)
template <int BYTES> __device__ __forceinline__ void store_past(void* to, const void* from)
{
    typedef uint32_t words_t __attribute__((ext_vector_type(BYTES / 4), aligned(2)));
    words_t w;
    __builtin_memcpy(&w, from, BYTES);
    __builtin_nontemporal_store(w, static_cast<words_t*>(to));
}

// 16 bytes of a row: 4 floats or 8 bf16.  Rows of odd widths begin anywhere, so these are loads and stores that ask for the
// alignment of an element only, which the hardware takes.
template <typename T> struct Vector {
    static constexpr int kElements = 16 / sizeof(T);
    T v[kElements];
};
template <typename T> __device__ __forceinline__ Vector<T> load_whole(const T* p)
{
    Vector<T> r;
    __builtin_memcpy(&r, p, 16);
    return r;
}
// Elements [col, col + kElements) of a row of H; behind the row's end zeros.
template <typename T> __device__ __forceinline__ Vector<T> load_vector(const T* row, int col, int H)
{
    constexpr int kE = Vector<T>::kElements;
    if (col + kE <= H) return load_whole(row + col);
    Vector<T> r;
#pragma unroll
    for (int i = 0; i < kE; ++i) r.v[i] = col + i < H ? row[col + i] : narrow<T>(0.0f);
    return r;
}
template <typename T> __device__ __forceinline__ void store_vector(T* row, int col, int H, const Vector<T>& r)
{
    constexpr int kE = Vector<T>::kElements;
    if (col + kE <= H) {
        store_past<16>(row + col, &r);
        return;
    }
#pragma unroll
    for (int i = 0; i < kE; ++i)
        if (col + i < H) row[col + i] = r.v[i];
}

// ---- lists of rows ----------------------------------------------------------------------------------------------

__device__ __forceinline__ int listed(const int32_t* frames, int rows)
{
    if (!frames) return rows;
    const int n = frames[0];
    return n < 0 ? 0 : n > rows ? rows : n;
}
// Row of the i-th entry, i < listed(); -1: an entry to skip.
__device__ __forceinline__ int row_of(const int32_t* frames, int rows, int i)
{
    if (!frames) return i;
    const int r = frames[1 + static_cast<int64_t>(i)];
    return r < 0 || r >= rows ? -1 : r;
}

// Row of entry i of the list, or -1 where it has none or one to skip: the list's count and its entry are asked for together.
__device__ __forceinline__ int row_at(const int32_t* frames, int rows, int64_t i)
{
    if (i >= rows) return -1;
    if (!frames) return static_cast<int>(i);
    const int n = frames[0], r = frames[1 + i];
    return i < n && r >= 0 && r < rows ? r : -1;
}

// Number of this workgroup in a grid that launch code has spread over two dimensions (spread() below).
__device__ __forceinline__ int64_t group_number() { return static_cast<int64_t>(blockIdx.y) * gridDim.x + blockIdx.x; }

// ---- sums and maxima over lanes ---------------------------------------------------------------------------------

__device__ __forceinline__ uint32_t wave_max(uint32_t v)
{
#pragma unroll
    for (int d = 32; d; d >>= 1) {
        const uint32_t o = __shfl_xor(v, d, kWave);
        v = v > o ? v : o;
    }
    return v;
}
template <typename V> __device__ __forceinline__ V wave_sum(V v)
{
#pragma unroll
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d, kWave);
    return v;
}

// ---- frames of a minibatch --------------------------------------------------------------------------------------

// Rows in ascending order: frame t's begin behind sum_b min(length_b, t) others, so a wavefront to a frame needs nobody.
__global__ __launch_bounds__(256) void ctc_pack_frames_kernel(const int32_t* __restrict__ lengths, int T, int B,
                                                              int32_t* __restrict__ frames)
{
    const int lane = threadIdx.x % kWave;
    const int64_t frame = group_number() * 4 + threadIdx.x / kWave;
    if (frame >= T) return;
    const int t = static_cast<int>(frame);
    int before = 0, all = 0;
    for (int b = lane; b < B; b += kWave) {
        int n = lengths[b];
        n = n < 0 ? 0 : n > T ? T : n;
        before += n < t ? n : t;
        all += n;
    }
    before = wave_sum(before);
    if (t == 0) {
        all = wave_sum(all);
        if (lane == 0) frames[0] = all;
    }
    int at = before;
    for (int b0 = 0; b0 < B; b0 += kWave) {
        const int b = b0 + lane;
        const bool in = b < B && lengths[b] > t;
        const uint64_t who = __ballot(in);
        if (in) frames[1 + static_cast<int64_t>(at) + __popcll(who & ((1ull << lane) - 1))] = t * B + b;
        at += __popcll(who);
    }
}

// ---- rows to 8 bits ---------------------------------------------------------------------------------------------

constexpr uint32_t kInfinity = 0x7f800000u;

// The whole number nearest to 127 |u| / m, ties to even, exactly: `inverse` is 127 / m to within half a step, so the
// product is off by less than 2^-16 (127 * 2^-23); where it comes that near to the middle between two whole numbers, 254 |u|
// is compared with (2 j + 1) m, both of which fp64 holds (32 bits).
__device__ __forceinline__ int level(float u, float m, float inverse)
{
    const float a = fabsf(u), t = a * inverse;
    int k = static_cast<int>(rintf(t));
    if (fabsf(t - static_cast<float>(k)) > 0.5f - 0x1p-15f) {
        const int j = static_cast<int>(t);
        const double twice = 254.0 * static_cast<double>(a), middle = static_cast<double>(2 * j + 1) * static_cast<double>(m);
        k = twice > middle || (twice == middle && (j & 1)) ? j + 1 : j;
    }
    return u < 0.0f ? -k : k;
}

struct NormArgs {
    const void* x;
    const void* residual;
    const float* weight;
    float eps;
    const int32_t* frames;
    int rows, H, pitch;
    void* sum;
    int8_t* q;
    float* scales;
};

// One row to a wavefront (four rows to a workgroup), or to all wavefronts of a workgroup; a row's elements stay in registers (E to a thread) from its one
// reading to its writing, its maximum and its sum of squares are formed across lanes.  Bound by the bytes.
template <typename T, int WAVES, int E, bool NORM>
__global__ __launch_bounds__(WAVES == 1 ? 256 : WAVES * kWave) void ctc_rows_to_8_bits_kernel(NormArgs p)
{
    constexpr int kE = Vector<T>::kElements, kVectors = E / kE;
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int64_t i = WAVES == 1 ? group_number() * 4 + wave : group_number();
    const int r = row_at(p.frames, p.rows, i);
    if (r < 0) return;
    const int thread = WAVES == 1 ? lane : threadIdx.x;
    const T* x = static_cast<const T*>(p.x) + static_cast<int64_t>(r) * p.H;
    const T* residual = NORM && p.residual ? static_cast<const T*>(p.residual) + static_cast<int64_t>(r) * p.H : nullptr;
    float u[E];
    double squares = 0.0;
    uint32_t most = 0;
#pragma unroll
    for (int v = 0; v < kVectors; ++v) {
        const int col = (v * WAVES * kWave + thread) * kE;
        Vector<T> z = load_vector(x, col, p.H);
        if constexpr (NORM) {
            if (residual) {
                const Vector<T> y = load_vector(residual, col, p.H);
#pragma unroll
                for (int k = 0; k < kE; ++k) z.v[k] = narrow<T>(widen(z.v[k]) + widen(y.v[k]));
            }
            if (p.sum) store_vector(static_cast<T*>(p.sum) + static_cast<int64_t>(r) * p.H, col, p.H, z);
        }
        Vector<float> w[kE / 4];
        if constexpr (NORM) {
            if (p.weight) {
#pragma unroll
                for (int k = 0; k < kE / 4; ++k) w[k] = load_vector(p.weight, col + 4 * k, p.H);
            }
        }
#pragma unroll
        for (int k = 0; k < kE; ++k) {
            const float f = widen(z.v[k]);
            if constexpr (NORM) squares += static_cast<double>(f) * static_cast<double>(f);
            const float g = NORM && p.weight ? f * w[k / 4].v[k % 4] : f;
            const uint32_t a = __float_as_uint(g) & 0x7fffffffu;
            most = most > a ? most : a;
            u[v * kE + k] = g;
        }
    }
    most = wave_max(most);
    if constexpr (NORM) squares = wave_sum(squares);
    if constexpr (WAVES > 1) {
        __shared__ uint32_t s_most[WAVES];
        __shared__ double s_squares[WAVES];
        if (lane == 0) {
            s_most[wave] = most;
            if constexpr (NORM) s_squares[wave] = squares;
        }
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WAVES; ++w) most = most > s_most[w] ? most : s_most[w];
        if constexpr (NORM) {
            squares = 0.0;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) squares += s_squares[w];
        }
    }
    // A row that is not finite: zeros, and a scale that says so.  Rows of tiny values are lifted, which is exact.
    const bool finite = most < kInfinity;
    const float lift = most < 0x20000000u ? 0x1p80f : 1.0f;
    const float m = __uint_as_float(most), m_lifted = m * lift;
    const float inverse = most && finite ? static_cast<float>(127.0 / static_cast<double>(m_lifted)) : 0.0f;
    int8_t* q = p.q + static_cast<int64_t>(r) * p.pitch;
#pragma unroll
    for (int v = 0; v < kVectors; ++v) {
        const int col = (v * WAVES * kWave + thread) * kE;
        if (col >= p.pitch) break;
        uint32_t word[kE / 4];
#pragma unroll
        for (int k = 0; k < kE; ++k) {
            const int l = finite ? level(u[v * kE + k] * lift, m_lifted, inverse) : 0;
            if (k % 4 == 0) word[k / 4] = 0;
            word[k / 4] |= (static_cast<uint32_t>(l) & 0xffu) << (8 * (k % 4));
        }
        __builtin_memcpy(__builtin_assume_aligned(q + col, kE), word, kE);
    }
    if (thread == 0) {
        double scale = static_cast<double>(m) / 127.0;
        if constexpr (NORM) scale /= sqrt(squares / p.H + static_cast<double>(p.eps));
        p.scales[r] = !finite ? __uint_as_float(0x7fc00000u) : most ? static_cast<float>(scale) : 0.0f;
    }
}

template <typename T>
__global__ __launch_bounds__(256) void ctc_rows_from_8_bits_kernel(const int8_t* __restrict__ q, const float* __restrict__ scales,
                                                                   const int32_t* __restrict__ frames, int rows, int H, int pitch,
                                                                   T* __restrict__ out)
{
    constexpr int kE = Vector<T>::kElements;
    const int lane = threadIdx.x % kWave;
    const int64_t i = group_number() * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int r = row_at(frames, rows, i);
    if (r < 0) return;
    const float scale = scales[r];
    const int8_t* from = q + static_cast<int64_t>(r) * pitch;
    T* to = out + static_cast<int64_t>(r) * H;
    constexpr int kStep = kWave * kE, kVectors = 4;
    for (int first = lane * kE; first < H; first += kVectors * kStep) {
        int8_t b[kVectors][kE];
#pragma unroll
        for (int i = 0; i < kVectors; ++i)                                   // (a row's bytes reach to its pitch)
            if (first + i * kStep < pitch) __builtin_memcpy(b[i], __builtin_assume_aligned(from + first + i * kStep, kE), kE);
#pragma unroll
        for (int i = 0; i < kVectors; ++i) {
            const int col = first + i * kStep;
            if (col >= H) break;
            Vector<T> v;
#pragma unroll
            for (int k = 0; k < kE; ++k) v.v[k] = narrow<T>(static_cast<float>(b[i][k]) * scale);
            store_vector(to, col, H, v);
        }
    }
}

// ---- the norm's backward pass -----------------------------------------------------------------------------------

struct NormBackArgs {
    const void* dy;
    const void* sum;
    const float* weight;
    float eps;
    const void* dresidual;
    const int32_t* frames;
    int rows, H;
    void* dsum;
    float* partials;             // [groups, H], or null
};

// A row to a wavefront (four rows to a workgroup) or to all wavefronts of a workgroup; workgroups take rows in turn and
// keep the sum over theirs of what each of their columns adds to dweight.
template <typename T, int WAVES, int E>
__global__ __launch_bounds__(WAVES == 1 ? 256 : WAVES * kWave) void ctc_norm_backward_kernel(NormBackArgs p)
{
    constexpr int kE = Vector<T>::kElements, kVectors = E / kE, kWidth = WAVES * kWave, kRows = WAVES == 1 ? 4 : 1;
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int thread = WAVES == 1 ? lane : threadIdx.x;
    const int n = listed(p.frames, p.rows);
    float w[E], dw[E];
#pragma unroll
    for (int v = 0; v < kVectors; ++v)
#pragma unroll
        for (int k = 0; k < kE; k += 4) {
            const int col = (v * kWidth + thread) * kE + k;
            Vector<float> four = {{1.0f, 1.0f, 1.0f, 1.0f}};
            if (p.weight) four = load_vector(p.weight, col, p.H);
#pragma unroll
            for (int j = 0; j < 4; ++j) w[v * kE + k + j] = four.v[j];
        }
#pragma unroll
    for (int k = 0; k < E; ++k) dw[k] = 0.0f;
    int turn = 0;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * kRows + (WAVES == 1 ? wave : 0); i < n;
         i += static_cast<int64_t>(gridDim.x) * kRows) {
        const int r = row_of(p.frames, p.rows, static_cast<int>(i));
        if (r < 0) continue;
        const int64_t row = static_cast<int64_t>(r) * p.H;
        Vector<T> z[kVectors], dy[kVectors], d[kVectors];
#pragma unroll
        for (int v = 0; v < kVectors; ++v) {
            const int col = (v * kWidth + thread) * kE;
            z[v] = load_vector(static_cast<const T*>(p.sum) + row, col, p.H);
            dy[v] = load_vector(static_cast<const T*>(p.dy) + row, col, p.H);
            d[v] = Vector<T>{};
            if (p.dresidual) d[v] = load_vector(static_cast<const T*>(p.dresidual) + row, col, p.H);
        }
        double squares = 0.0, along = 0.0;
#pragma unroll
        for (int v = 0; v < kVectors; ++v)
#pragma unroll
            for (int k = 0; k < kE; ++k) {
                const double f = static_cast<double>(widen(z[v].v[k]));
                squares += f * f;
                along += static_cast<double>(widen(dy[v].v[k]) * w[v * kE + k]) * f;
            }
        squares = wave_sum(squares);
        along = wave_sum(along);
        if constexpr (WAVES > 1) {
            // (two buffers by turns: who writes one again has passed the barrier that its readers of two turns ago came to)
            __shared__ double s_sums[2][2][WAVES];
            if (lane == 0) {
                s_sums[turn][0][wave] = squares;
                s_sums[turn][1][wave] = along;
            }
            __syncthreads();
            squares = along = 0.0;
#pragma unroll
            for (int o = 0; o < WAVES; ++o) {
                squares += s_sums[turn][0][o];
                along += s_sums[turn][1][o];
            }
            turn ^= 1;
        }
        const double variance = squares / p.H + static_cast<double>(p.eps);
        // (the mean's share without the factor: with it, it would vanish in fp32 for rows of 1e20 and more)
        const float f = static_cast<float>(1.0 / sqrt(variance)), c = static_cast<float>(along / p.H / variance);
#pragma unroll
        for (int v = 0; v < kVectors; ++v) {
#pragma unroll
            for (int k = 0; k < kE; ++k) {
                const float g = widen(dy[v].v[k]), zk = widen(z[v].v[k]);
                dw[v * kE + k] += g * (zk * f);
                d[v].v[k] = narrow<T>((g * w[v * kE + k] - zk * c) * f + widen(d[v].v[k]));
            }
            store_vector(static_cast<T*>(p.dsum) + row, (v * kWidth + thread) * kE, p.H, d[v]);
        }
    }
    if (!p.partials) return;
    if constexpr (WAVES == 1) {
        // The four wavefronts' sums, one after another.
        __shared__ float s_dw[E][kWave];
        for (int o = 0; o < 4; ++o) {
            if (wave == o) {
#pragma unroll
                for (int k = 0; k < E; ++k) {
                    if (o) dw[k] += s_dw[k][lane];
                    s_dw[k][lane] = dw[k];
                }
            }
            __syncthreads();
        }
        if (wave != 3) return;
    }
    float* out = p.partials + static_cast<int64_t>(blockIdx.x) * p.H;
#pragma unroll
    for (int v = 0; v < kVectors; ++v)
#pragma unroll
        for (int k = 0; k < kE; k += 4) {
            Vector<float> four;
#pragma unroll
            for (int j = 0; j < 4; ++j) four.v[j] = dw[v * kE + k + j];
            store_vector(out, (v * kWidth + thread) * kE + k, p.H, four);
        }
}

// out[k] = sum over p of partials[p * stride + k], in fp64; 64 rows by 16 columns to a workgroup at once, so that few columns make enough workgroups
// and a thread's loads are under way together (16 rows by 64 columns: the norm's gradient of 1500 rows of 1024 bf16 11.4 us, so 9.9).
__global__ __launch_bounds__(1024) void ctc_sum_partials_kernel(const float* __restrict__ partials, int count, int64_t stride,
                                                                int64_t width, float* __restrict__ out)
{
    __shared__ double s_sum[16][16];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int64_t col = static_cast<int64_t>(blockIdx.x) * 16 + lane % 16;
    double sum = 0.0;
    if (col < width)
#pragma unroll 16
        for (int p = wave * 4 + lane / 16; p < count; p += 64) sum += static_cast<double>(partials[p * stride + col]);
    sum += __shfl_xor(sum, 16, kWave);
    sum += __shfl_xor(sum, 32, kWave);
    if (lane < 16) s_sum[wave][lane] = sum;
    __syncthreads();
    if (threadIdx.x < 16 && col < width) {
#pragma unroll
        for (int g = 1; g < 16; ++g) sum += s_sum[g][lane];
        out[col] = static_cast<float>(sum);
    }
}

// ---- activations ------------------------------------------------------------------------------------------------

typedef int int4v __attribute__((ext_vector_type(4)));

struct LinearArgs {
    const int8_t* q;
    const float* scales;
    const int8_t* weight_q;
    const float* weight_scales;
    const float* bias;
    const int32_t* frames;
    int rows, A, pitch;
    void* logits;
};

// What a sum becomes: the scales' product, the sum times it, the bias; then one rounding to T.
template <typename T> __device__ __forceinline__ T activation(int sum, float scale, float weight_scale, float bias)
{
    return narrow<T>(fmaf(static_cast<float>(sum), scale * weight_scale, bias));
}

// Few rows and symbols: 16 by 16 to a workgroup, straight from memory into the matrix cores, each of the four wavefronts with every fourth 128
// bytes of the rows; their sums are added in LDS.  The larger operand is read once, with nothing between a wavefront's loads.
// v_mfma_i32_16x16x64_i8: lane l gives bytes 16 (l / 16) .. of row l % 16 of either operand, and holds rows 4 (l / 16) .. + 3 of column
// l % 16 of the result.
template <typename T>
__global__ __launch_bounds__(256) void ctc_linear_direct_kernel(LinearArgs p)
{
    __shared__ int4v s_sum[4][kWave];
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const unsigned columns = static_cast<unsigned>((p.A + 15) / 16);
    const int64_t m0 = static_cast<int64_t>(blockIdx.x / columns) * 16;
    const int a = static_cast<int>(blockIdx.x % columns) * 16 + lane % 16;
    // All loads of 2048 bytes of the rows before the first product; the weights', which wait for nothing, before the list's.
    const int begin = wave * 128 + lane / 16 * 16;
    const int8_t* const column = p.weight_q + static_cast<int64_t>(a < p.A ? a : p.A - 1) * p.pitch + begin;
    int4v x[8], w[8];
    const auto load = [&](int4v (&to)[8], const int8_t* from, int k0) {
#pragma unroll
        for (int h = 0; h < 8; ++h) {
            const int k = k0 + h / 2 * 512 + h % 2 * 64;
            to[h] = k + wave * 128 < p.pitch ? *reinterpret_cast<const int4v*>(from + k) : int4v{};
        }
    };
    load(w, column, 0);
    const int mine = row_at(p.frames, p.rows, m0 + lane % 16);
    // (a row that does not count gives the first symbol's weights: any bytes will do)
    const int8_t* const row = (mine < 0 ? p.weight_q : p.q + static_cast<int64_t>(mine) * p.pitch) + begin;
    if (m0 >= listed(p.frames, p.rows)) return;
    const float weight_scale = a < p.A ? p.weight_scales[a] : 0.0f, bias = a < p.A && p.bias ? p.bias[a] : 0.0f;
    int4v sum = {};
    for (int k0 = 0; k0 < p.pitch; k0 += 2048) {
        load(x, row, k0);
#pragma unroll
        for (int h = 0; h < 8; ++h) sum = __builtin_amdgcn_mfma_i32_16x16x64_i8(x[h], w[h], sum, 0, 0, 0);
        if (k0 + 2048 < p.pitch) load(w, column, k0 + 2048);
    }
    s_sum[wave][lane] = sum;
    __syncthreads();
    // One of a lane's four rows to each wavefront.
    const int r = __shfl(mine, lane / 16 * 4 + wave, kWave);
    if (r < 0 || a >= p.A) return;
    const int total = s_sum[0][lane][wave] + s_sum[1][lane][wave] + s_sum[2][lane][wave] + s_sum[3][lane][wave];
    static_cast<T*>(p.logits)[static_cast<int64_t>(r) * p.A + a] = activation<T>(total, p.scales[r], weight_scale, bias);
}

typedef int int16v __attribute__((ext_vector_type(16)));

// 16 bytes a lane from memory to LDS, lane after lane from `to` on.
__device__ __forceinline__ void to_lds(const int8_t* from, int8_t* to)
{
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from,
                                     (__attribute__((address_space(3))) void*)to, 16, 0, 0);
}

// Waits until at most N of this wavefront's requests to memory are under way and none to LDS, then for the workgroup's others.
template <int N> __device__ __forceinline__ void wait_and_meet()
{
    static_assert(N < 64);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0070 | (N & 15) | (N >> 4) << 14);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// Many rows by many symbols: 64 WM rows by 64 WN symbols to a workgroup, 32 WM by 32 WN to each of its four wavefronts, 64 bytes of
// every row at a time in LDS, in kStages buffers: while the matrix cores work on one, memory fills the others.  A wavefront
// holds the operands of the next 32 bytes in registers while it multiplies these; the barrier comes before a buffer's last 32, whose
// operands are in registers by then, so that the next buffer's first are fetched beside them.
// LDS holds a row's four 16-byte pieces in the order piece ^ (row / 4 % 4): eight lanes that read one piece of eight rows then
// meet eight places of 16 bytes, a different one each modulo the banks.
// v_mfma_i32_32x32x32_i8: lane l gives bytes 16 (l / 32) .. of row l % 32 of either operand and holds rows
// 8 (v / 4) + 4 (l / 32) + v % 4, v < 16, of column l % 32 of the result; with the weights first those are symbols, and the lane's
// column is a row of the states.  The sums go through LDS once more, 32 rows at a time, so that rows of activations are written in
// vectors.
template <typename T, int WM, int WN>
__global__ __launch_bounds__(256) void ctc_linear_tiles_kernel(LinearArgs p)
{
    constexpr int kBM = 64 * WM, kBN = 64 * WN, kGroup = 8, kStages = 4, kLoads = WM + WN, kBytes = (kBM + kBN) * 64;
    __shared__ __align__(1024) int8_t s_buffer[kStages][kBytes];
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int n = listed(p.frames, p.rows);
    // Workgroups go to the 8 dies in turn: each die takes a contiguous run of tiles, which go down kGroup tiles of rows before
    // they go on to the next symbols, so that a die's workgroups share rows and weights in its cache.
    const unsigned down = static_cast<unsigned>((n + kBM - 1) / kBM), across = static_cast<unsigned>((p.A + kBN - 1) / kBN);
    const unsigned tiles = down * across, per_die = (tiles + 7) / 8;
    if (blockIdx.x / 8 >= per_die) return;
    const unsigned tile = blockIdx.x % 8 * per_die + blockIdx.x / 8;
    if (tile >= tiles) return;
    const unsigned group = tile / (kGroup * across), in_group = tile % (kGroup * across);
    const unsigned high = down - group * kGroup < kGroup ? down - group * kGroup : kGroup;
    const int m0 = static_cast<int>(group * kGroup + in_group % high) * kBM, a0 = static_cast<int>(in_group / high) * kBN;

    // Thread i will say where the tile's row i begins among the activations (-1: it does not count), and its scale.
    struct Row { int64_t at; float scale; };
    Row mine = {-1, 0.0f};
    if (threadIdx.x < kBM && static_cast<int64_t>(m0) + threadIdx.x < n) {
        const int r = row_of(p.frames, p.rows, m0 + static_cast<int>(threadIdx.x));
        if (r >= 0) mine = {static_cast<int64_t>(r) * p.A, p.scales[r]};
    }
    const int8_t* from[kLoads];
    const int piece = (lane % 4 ^ lane / 16) * 16;
#pragma unroll
    for (int j = 0; j < WM; ++j) {
        const int64_t i = static_cast<int64_t>(m0) + (j * 4 + wave) * 16 + lane / 4;
        const int r = i < n ? row_of(p.frames, p.rows, static_cast<int>(i)) : -1;
        from[j] = (r < 0 ? p.weight_q : p.q + static_cast<int64_t>(r) * p.pitch) + piece;    // (any bytes for a row that does not count)
    }
#pragma unroll
    for (int j = 0; j < WN; ++j) {
        const int a = a0 + (j * 4 + wave) * 16 + lane / 4;
        from[WM + j] = p.weight_q + static_cast<int64_t>(a < p.A ? a : p.A - 1) * p.pitch + piece;
    }
    // The bytes of step t; behind the last one those of the last again, which nobody reads, so that the number of requests under
    // way is the same in every step.
    const int steps = p.pitch / 64;
    const auto fill = [&](int8_t* buffer, int t) {
        const int on = t + 1 < steps ? 64 : 0;
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            to_lds(from[j], buffer + (j * 4 + wave) * 1024);
            from[j] += on;
        }
    };
    const int at_row = (wave / 2 * 32 * WM + lane % 32) * 64, at_column = (kBM + wave % 2 * 32 * WN + lane % 32) * 64;
    const int first_piece = lane / 32 ^ lane / 4 % 4;
    int4v x[2][WM], w[2][WN];
    const auto fetch = [&](const int8_t* buffer, int half) {
        const int at = (first_piece ^ half * 2) * 16;
#pragma unroll
        for (int i = 0; i < WM; ++i) x[half][i] = *reinterpret_cast<const int4v*>(buffer + at_row + i * 2048 + at);
#pragma unroll
        for (int i = 0; i < WN; ++i) w[half][i] = *reinterpret_cast<const int4v*>(buffer + at_column + i * 2048 + at);
    };
    int16v sum[WM][WN] = {};
    const auto multiply = [&](int half) {
#pragma unroll
        for (int i = 0; i < WM; ++i)
#pragma unroll
            for (int j = 0; j < WN; ++j) sum[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(w[half][j], x[half][i], sum[i][j], 0, 0, 0);
    };
    // A product, a read of LDS and so on; the products that are left hide the last reads (left alone the compiler puts the reads right
    // before their use).
    const auto interleave = [&]() {
#pragma unroll
        for (int i = 0; i < WM + WN; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, WM * WN > WM + WN ? WM * WN - WM - WN : 0, 0);
        __builtin_amdgcn_sched_barrier(0);
    };
    // One buffer's products.  The next one's bytes were asked for kStages - 1 steps ago; behind the barrier every wavefront has what
    // it needs of this one, which is filled again.
    const auto step = [&](int stage, int t) {
        int8_t* const now = s_buffer[stage];
        fetch(now, 1);
        multiply(0);
        interleave();
        wait_and_meet<(kStages - 2) * kLoads>();
        fill(now, t + kStages);
        fetch(s_buffer[(stage + 1) % kStages], 0);      // (behind the last step what nobody multiplies)
        multiply(1);
        interleave();
    };
#pragma unroll
    for (int t = 0; t < kStages; ++t) fill(s_buffer[t], t);
    wait_and_meet<(kStages - 1) * kLoads>();
    fetch(s_buffer[0], 0);
    int t = 0;
    for (; t + kStages <= steps; t += kStages) {
#pragma unroll
        for (int i = 0; i < kStages; ++i) step(i, t + i);
    }
#pragma unroll
    for (int i = 0; i + 1 < kStages; ++i)
        if (t + i < steps) step(i, t + i);
    // (From here on memory is asked for nothing but to write: a wait for a load behind the writes would wait for them too.)
    constexpr int kAcross = 8 * WN, kDown = kWave / kAcross, kLine = 32 * WN + 4;       // lanes to a row, rows at once, ints from row to row
    const int a = a0 + wave % 2 * 32 * WN + lane % kAcross * 4;
    float weight_scale[4], bias[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int b = a + k < p.A ? a + k : p.A - 1;
        weight_scale[k] = p.weight_scales[b];
        bias[k] = p.bias ? p.bias[b] : 0.0f;
    }
    wait_and_meet<0>();
    static_assert(kBM <= 256 && kBM * sizeof(Row) + 4 * 32 * kLine * 4 <= kStages * kBytes);
    Row* const s_row = reinterpret_cast<Row*>(&s_buffer[0][0]);
    int* const s_sum = reinterpret_cast<int*>(s_row + kBM) + wave * 32 * kLine;
    if (threadIdx.x < kBM) s_row[threadIdx.x] = mine;
    wait_and_meet<0>();
    T* const logits = static_cast<T*>(p.logits) + a;
#pragma unroll
    for (int i = 0; i < WM; ++i) {
#pragma unroll
        for (int j = 0; j < WN; ++j)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *reinterpret_cast<int4v*>(s_sum + lane % 32 * kLine + j * 32 + g * 8 + lane / 32 * 4) =
                    int4v{sum[i][j][g * 4], sum[i][j][g * 4 + 1], sum[i][j][g * 4 + 2], sum[i][j][g * 4 + 3]};
        const auto write = [&](auto whole) {
#pragma unroll
            for (int b0 = 0; b0 < 32 / kDown; b0 += 4) {
                int4v four[4];
                Row row[4];
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    const int at = (b0 + b) * kDown + lane / kAcross;
                    four[b] = *reinterpret_cast<const int4v*>(s_sum + at * kLine + lane % kAcross * 4);
                    row[b] = s_row[(wave / 2 * WM + i) * 32 + at];
                }
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    T value[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) value[k] = activation<T>(four[b][k], row[b].scale, weight_scale[k], bias[k]);
                    if (decltype(whole)::value) {
                        if (row[b].at >= 0) __builtin_memcpy(logits + row[b].at, value, sizeof(value));
                    } else {
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            if (row[b].at >= 0 && a + k < p.A) logits[row[b].at + k] = value[k];
                    }
                }
            }
        };
        if (a0 + kBN <= p.A)
            write(std::true_type{});
        else
            write(std::false_type{});
    }
}

// ---- gradient of the weights ------------------------------------------------------------------------------------

// dweight = G^T Q is a product whose inner index, the row, is the slow one of both operands: memory gives 4 symbols' or
// columns' worth of a row at a time, the matrix cores take 8 rows of one symbol or column.  So the operands pass through registers, where
// gradients take their scale and are split, and whole numbers become floats, and are laid down in LDS with the rows innermost.
//
// A product of gradient and scale, an fp32 number c, enters the matrix cores
//   as three bf16 numbers, the leading 8 bits, the next 8 and the last (exact from 2^-110 on; below, bits under 2^-133, where bf16 ends, are
//   lost): narrow tiles, whose gradients' work is done as they come, or
//   as two fp16 numbers, each rounded to nearest (22 bits and a sign; c is off by at most half its last bit or 2^-39 of its column's
//   largest), after a power of two that puts the column's largest in [2^14, 2^15): wide tiles, which the matrix cores bind.  The columns' largest
//   take one more reading of the gradients, a launch of its own, which also forms the bias's gradient.
// The whole numbers are exact in either type.

struct GradientArgs {
    const void* grads;
    const int8_t* q;
    const float* scales;
    const int32_t* frames;
    int rows, H, A, pitch, slabs;
    float* out;                  // [slabs, A, H]
    float* bias;                 // [slabs, A]: sums of the gradients; null: not wanted
    const uint32_t* largest;     // [kColumnSlabs, A]: bits of the largest |gradient * scale|
};

typedef float float16v __attribute__((ext_vector_type(16)));
typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t uint4v __attribute__((ext_vector_type(4)));
typedef uint32_t uint2v __attribute__((ext_vector_type(2)));

// The power of two that brings numbers of at most `largest` (bits) below 2^15, as an exponent.
__device__ __forceinline__ int lift_of(uint32_t largest)
{
    const int e = static_cast<int>(largest >> 23);
    return e == 255 ? 0 : e < 14 ? 127 : 141 - e;
}

// [first, last) of the list's entries for slab `slab` of `slabs`; slabs begin at multiples of 32.
struct Range { int first, last; };
__device__ __forceinline__ Range slab_of(int n, int slab, int slabs)
{
    const int64_t per = ((n + 31LL) / 32 + slabs - 1) / slabs * 32, first = slab * per;
    return {static_cast<int>(first < n ? first : n), static_cast<int>(first + per < n ? first + per : n)};
}

// Waits for this wavefront's requests to LDS, then for the workgroup's others; requests to memory stay under way.
__device__ __forceinline__ void meet()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xc07f);                 // lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// A step's rows, as the list has them; -1: does not count.  (Steps behind the last have rows that do not count; every index is one of the
// list's, every address a row's.)  The entry is asked for early and looked at late.
struct StepRows {
    const int32_t* entries;
    bool list;
    int rows;
    Range range;
    int place;                   // which of a step's 32 this lane has
    __device__ __forceinline__ StepRows(const GradientArgs& p, Range r, int which)
        : entries(p.frames ? p.frames + 1 : reinterpret_cast<const int32_t*>(p.scales)), list(p.frames), rows(p.rows), range(r), place(which) {}
    __device__ __forceinline__ int ask(int step) const
    {
        const int i = range.first + step * 32 + place;
        return entries[i < range.last ? i : range.last - 1];
    }
    __device__ __forceinline__ int row(int step, int entry) const
    {
        const int i = range.first + step * 32 + place;
        const int r = list ? entry : i;
        return i < range.last && r >= 0 && r < rows ? r : -1;
    }
};

// Largest |gradient * scale| and sum of the gradients of each symbol, over the rows of a slab: two symbols to a lane, the rows dealt out to
// four wavefronts, eight at a time.
template <typename T> __device__ __forceinline__ void look_at_columns(const GradientArgs& p, uint32_t* largest, int block, int slab)
{
    __shared__ uint32_t s_most[4][2 * kWave];
    __shared__ double s_sum[4][2 * kWave];
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int a = block * (2 * kWave) + 2 * lane;
    const Range range = slab_of(listed(p.frames, p.rows), slab, kColumnSlabs);
    const int at = a + 1 < p.A ? a : a < p.A ? a - 1 : 0;                    // (A is at least 2 here; the last symbol of an odd number is the upper of a pair)
    uint32_t most[2] = {};
    double sum[2] = {};
    const int steps = (range.last - range.first + 31) / 32;
    const StepRows list(p, range, wave * 8 + lane % 8);
    int entry = steps > 0 ? list.ask(0) : 0;
    for (int t = 0; t < steps; ++t) {
        const int row = list.row(t, entry);
        const float scales = row < 0 ? 0.0f : p.scales[row];
        entry = list.ask(t + 1);
        T g[8][2];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int r = __builtin_amdgcn_readlane(row, j);
            __builtin_memcpy(g[j], static_cast<const T*>(p.grads) + static_cast<int64_t>(r < 0 ? 0 : r) * p.A + at, sizeof(g[j]));
        }
        float eight[2] = {};
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (__builtin_amdgcn_readlane(row, j) < 0) continue;
            const float scale = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(scales), j));
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const float v = widen(g[j][k]);
                const uint32_t bits = __float_as_uint(v * scale) & 0x7fffffffu;
                most[k] = most[k] > bits ? most[k] : bits;
                eight[k] += v;
            }
        }
        sum[0] += static_cast<double>(eight[0]);
        sum[1] += static_cast<double>(eight[1]);
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        s_most[wave][2 * lane + k] = most[k];
        s_sum[wave][2 * lane + k] = sum[k];
    }
    __syncthreads();
    const int mine = block * (2 * kWave) + threadIdx.x;
    if (threadIdx.x >= 2 * kWave || mine >= p.A) return;
    const int from = mine == p.A - 1 && mine % 2 == 0 ? threadIdx.x + 1 : threadIdx.x;
    uint32_t m = 0;
    double total = 0.0;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        m = m > s_most[w][from] ? m : s_most[w][from];
        total += s_sum[w][from];
    }
    largest[static_cast<int64_t>(slab) * p.A + mine] = m;
    if (p.bias) p.bias[static_cast<int64_t>(slab) * p.A + mine] = static_cast<float>(total);
}

// What lies `at` bytes behind an address that is the same in all lanes and stays in scalar registers, as `at` stays 32 bits if it comes from here():
// left alone the compiler adds a lane's place to the address before it multiplies the row by its pitch, with a vector instruction of
// quarter rate for each load (27200 rows of 2048, 29 symbols: 33.3 us, so, with a step's rows in the same lanes of every wavefront, 31.7).
template <typename V> __device__ __forceinline__ V load_from(const void* row, uint32_t at)
{
    typedef const __attribute__((address_space(1))) char* Global;
    const uint64_t whole = reinterpret_cast<uint64_t>(row);
    const uint32_t low = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(whole)), high = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(whole >> 32));
    const Global from = reinterpret_cast<Global>(static_cast<uint64_t>(high) << 32 | low);
    return *(const __attribute__((address_space(1))) V*)(from + at);
}

// `at`, as far as the compiler knows another one for each `row`.
__device__ __forceinline__ uint32_t here(uint32_t at, int row)
{
    asm("" : "+v"(at) : "v"(row));
    return at;
}

// Gradients of one symbol in eight rows, as they are in memory; the rows, and their scales, in lanes 0 to 7 (and again in 8 to 15 and so on).
struct Eight {
    int row;
    float scale;
    uint32_t g[8];
};
// Row `row`'s gradient of the symbol at `at` bytes.
template <typename T> __device__ __forceinline__ uint32_t gradient_of(const GradientArgs& p, int row, uint32_t at)
{
    const char* from = static_cast<const char*>(p.grads) + static_cast<uint64_t>(row < 0 ? 0 : row) * static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(p.A * static_cast<int>(sizeof(T))));
    if constexpr (sizeof(T) == 2)
        return load_from<uint16_t>(from, at);
    else
        return load_from<uint32_t>(from, at);
}
template <typename T> __device__ __forceinline__ float gradient_in(uint32_t bits) { return __uint_as_float(sizeof(T) == 2 ? bits << 16 : bits); }
// Gradients and scales of rows that do not count: 0, whatever is there.
__device__ __forceinline__ void clear(Eight& e)
{
    if (__ballot(e.row >= 0) == ~0ull) return;
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (__builtin_amdgcn_readlane(e.row, j) < 0) e.g[j] = 0;
    if (e.row < 0) e.scale = 0.0f;
}
__device__ __forceinline__ float scale_of(const Eight& e, int lane) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(e.scale), lane)); }

// Narrow tiles: 32 NA symbols by 256 columns to a workgroup of eight wavefronts, 32 NA by 32 to each; 32 rows a step, in two buffers of
// LDS: in a step a wavefront lays down the next step's operands, asks memory for what it will lay down kAhead steps later, and multiplies.
// LDS: symbol a's 8-row piece j (16 bytes) lies at 64 a + 16 (j ^ a / 4 % 4); column k's at 64 (64 (k % 4) + k / 4) + 16 (j ^ k % 4 ^ k / 16 % 4):
// what lanes write or read at once then falls on different banks.
// v_mfma_f32_32x32x16_{f16,bf16}: lane l gives numbers 8 (l / 32) .. of row l % 32 of either operand, and holds rows
// 8 (v / 4) + 4 (l / 32) + v % 4, v < 16, of column l % 32 of the result.
template <typename T, int NA>
__global__ __launch_bounds__(512) void ctc_weight_gradient_narrow_kernel(GradientArgs p)
{
    constexpr int kTA = 32 * NA, kPartBytes = kTA * 64, kNumbers = 3 * kPartBytes, kBytes = kNumbers + 256 * 64, kAhead = 2;
    __shared__ __align__(1024) int8_t s_buffer[2][kBytes];
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int a0 = blockIdx.x * kTA, k0 = blockIdx.y * 256, slab = blockIdx.z, chunk = wave % 4 * 8;
    const Range range = slab_of(listed(p.frames, p.rows), slab, p.slabs);
    const int steps = (range.last - range.first + 31) / 32;
    // (wavefronts w and w + 4 have the same eight rows, the second with its four of whole numbers in front)
    const StepRows list(p, range, chunk + (lane % 8 ^ wave / 4 * 4));
    // What this lane brings: symbol a0 + lane of rows `chunk` .. (four wavefronts), columns 4 lane .. of half of these rows.  (Symbols behind the
    // last and columns behind a row's bytes are others' once more: what becomes of them is not written.)
    const bool brings = wave < 4 && lane < kTA;
    const uint32_t at = static_cast<uint32_t>(a0 + lane < p.A ? a0 + lane : p.A - 1) * static_cast<uint32_t>(sizeof(T));
    const uint32_t column = static_cast<uint32_t>(k0 + 4 * lane < p.pitch ? k0 + 4 * lane : 0);
    struct Raw {
        Eight e;
        uint32_t q[4];
    };
    const auto ask = [&](Raw& to, int row) {
        to.e.row = row;
        to.e.scale = p.scales[row < 0 ? 0 : row];
        const uint32_t from = here(column, row);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int r = __builtin_amdgcn_readlane(row, j);
            to.q[j] = load_from<uint32_t>(p.q + static_cast<uint64_t>(r < 0 ? 0 : r) * static_cast<uint32_t>(p.pitch), from);
        }
        if (brings) {
            const uint32_t mine = here(at, row);
#pragma unroll
            for (int j = 0; j < 8; ++j) to.e.g[j] = gradient_of<T>(p, __builtin_amdgcn_readlane(row, j), mine);
        }
    };
    double bias = 0.0;
    const bool sums = p.bias && blockIdx.y == 0;
    const auto lay_down = [&](Raw& from, int8_t* buffer) {
        clear(from.e);
        if (brings) {
            uint4v part[3];
            float eight = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; j += 2) {
                float c[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const float g = gradient_in<T>(from.e.g[j + i]);
                    eight += g;
                    c[i] = g * scale_of(from.e, j + i);
                }
#pragma unroll
                for (int b = 0; b < 3; ++b) {
                    const uint32_t u = __float_as_uint(c[0]), v = __float_as_uint(c[1]);
                    part[b][j / 2] = __builtin_amdgcn_perm(v, u, 0x07060302);                 // the leading halves of both
                    c[0] -= __uint_as_float(u & 0xffff0000u);
                    c[1] -= __uint_as_float(v & 0xffff0000u);
                }
            }
            if (sums) bias += static_cast<double>(eight);
#pragma unroll
            for (int b = 0; b < 3; ++b)
                *reinterpret_cast<uint4v*>(buffer + b * kPartBytes + lane * 64 + ((wave % 4 ^ lane / 4 % 4) * 16)) = part[b];
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            uint2v four;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float u = static_cast<float>(static_cast<int8_t>(from.q[2 * j] >> 8 * k));
                const float v = static_cast<float>(static_cast<int8_t>(from.q[2 * j + 1] >> 8 * k));
                four[j] = __builtin_amdgcn_perm(__float_as_uint(v), __float_as_uint(u), 0x07060302);
            }
            *reinterpret_cast<uint2v*>(buffer + kNumbers + (k * 64 + lane) * 64 + ((wave % 4 ^ k ^ lane / 4 % 4) * 16) + wave / 4 * 8) = four;
        }
    };
    float16v sum[NA] = {};
    const auto multiply = [&](const int8_t* buffer) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int piece = (h * 2 + lane / 32) ^ lane % 4 ^ (wave % 2 * 2 + lane % 32 / 16);
            const bf16x8 q = *reinterpret_cast<const bf16x8*>(buffer + kNumbers + (lane % 4 * 64 + wave * 8 + lane % 32 / 4) * 64 + piece * 16);
            bf16x8 g[3][NA];
#pragma unroll
            for (int b = 0; b < 3; ++b)
#pragma unroll
                for (int i = 0; i < NA; ++i)
                    g[b][i] = *reinterpret_cast<const bf16x8*>(buffer + b * kPartBytes + (i * 32 + lane % 32) * 64 + (((h * 2 + lane / 32) ^ lane / 4 % 4) * 16));
#pragma unroll
            for (int b = 2; b >= 0; --b)
#pragma unroll
                for (int i = 0; i < NA; ++i) sum[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(g[b][i], q, sum[i], 0, 0, 0);
        }
    };
    if (steps > 0) {
        // A step's rows' numbers are asked for kAhead steps before its rows, these kAhead steps before they are laid down: nothing is waited for
        // that has not been under way as long.
        // (The first steps' are asked for together: three round trips to memory before the loop, and not five.)
        Raw first, raw[kAhead];
        int early[1 + kAhead], entry[kAhead];
#pragma unroll
        for (int j = 0; j <= kAhead; ++j) early[j] = list.ask(j);
#pragma unroll
        for (int j = 0; j < kAhead; ++j) entry[j] = list.ask(1 + kAhead + j);
        ask(first, list.row(0, early[0]));
#pragma unroll
        for (int j = 0; j < kAhead; ++j) ask(raw[j], list.row(1 + j, early[1 + j]));
        lay_down(first, s_buffer[0]);
        meet();
        for (int t0 = 0; t0 < steps; t0 += kAhead) {
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                const int t = t0 + j;
                if (t >= steps) break;
                lay_down(raw[j], s_buffer[j % 2 ^ 1]);
                ask(raw[j], list.row(t + 1 + kAhead, entry[j]));
                entry[j] = list.ask(t + 1 + 2 * kAhead);
                multiply(s_buffer[j % 2]);
                meet();
            }
        }
    }
    if (sums) {
        // The four wavefronts that brought the gradients, one after another.
        double* const s_bias = reinterpret_cast<double*>(&s_buffer[0][0]);
        for (int w = 0; w < 4; ++w) {
            if (wave == w && lane < kTA) {
                if (w) bias += s_bias[lane];
                s_bias[lane] = bias;
            }
            __syncthreads();
        }
        if (wave == 3 && lane < kTA && a0 + lane < p.A) p.bias[static_cast<int64_t>(slab) * p.A + a0 + lane] = static_cast<float>(bias);
    }
    float* const out = p.out + static_cast<int64_t>(slab) * p.A * p.H;
    const int k = k0 + wave * 32 + lane % 32;
#pragma unroll
    for (int i = 0; i < NA; ++i)
#pragma unroll
        for (int v = 0; v < 16; ++v) {
            const int a = a0 + i * 32 + 8 * (v / 4) + 4 * (lane / 32) + v % 4;
            if (a < p.A && k < p.H) out[static_cast<int64_t>(a) * p.H + k] = sum[i][v];
        }
}

// For wide tiles: the whole numbers of the listed rows as fp16, once for all symbols' workgroups.  32 listed rows at a time (a step), for each
// column k 64 bytes, its 8-row pieces in the order j ^ k / 4 % 4: as the kernel below wants them in LDS.  256 columns to a workgroup.
__device__ __forceinline__ void widen_rows(const GradientArgs& p, uint16_t* wide, int step, int k0)
{
    __shared__ __align__(16) int8_t s_row[32][256 + 4];
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int n = listed(p.frames, p.rows);
    if (step * 32 >= n) return;
    const StepRows list(p, {0, n}, wave * 8 + lane % 8);
    const int row = list.row(step, list.ask(step));
    if (k0 + 4 * lane < p.pitch) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int r = __builtin_amdgcn_readlane(row, j);
            *reinterpret_cast<uint32_t*>(&s_row[wave * 8 + j][4 * lane]) =
                *reinterpret_cast<const uint32_t*>(p.q + static_cast<uint64_t>(r < 0 ? 0 : r) * static_cast<uint32_t>(p.pitch) + k0 + 4 * lane);
        }
    }
    __syncthreads();
    const int k = threadIdx.x;
    if (k0 + k >= p.pitch) return;
    uint16_t* const to = wide + (static_cast<int64_t>(step) * p.pitch + k0 + k) * 32;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        half8 piece;
#pragma unroll
        for (int i = 0; i < 8; ++i) piece[i] = static_cast<_Float16>(static_cast<float>(s_row[j * 8 + i][k]));
        *reinterpret_cast<half8*>(to + (j ^ k / 4 % 4) * 8) = piece;
    }
}

// Both in one launch: the columns' workgroups first.
template <typename T>
__global__ __launch_bounds__(256) void ctc_gradient_prepare_kernel(GradientArgs p, uint32_t* largest, uint16_t* wide, unsigned column_blocks)
{
    const unsigned columns = column_blocks * kColumnSlabs, group = static_cast<unsigned>(group_number());
    if (group < columns) {
        look_at_columns<T>(p, largest, group % column_blocks, group / column_blocks);
    } else {
        const unsigned across = static_cast<unsigned>((p.pitch + 255) / 256), i = group - columns;
        widen_rows(p, wide, static_cast<int>(i / across), static_cast<int>(i % across) * 256);
    }
}

// 128 symbols by 512 columns to a workgroup of eight wavefronts, 64 by 128 to each; 32 rows a step, in three buffers of LDS.  The barrier is in
// a step's middle, when every wavefront has the operands of its second half in registers: behind it the step's buffer of whole numbers is filled, from
// memory, for three steps on, and the next step's first operands are fetched.  Gradients pass through registers: asked for three steps before they
// are split and laid down, two steps before they are multiplied.
// LDS: piece j of symbol a lies at 64 a + 16 (j ^ a / 4 % 4), and so for columns: eight lanes' reads of a piece meet different banks.
template <typename T>
__global__ __launch_bounds__(512) void ctc_weight_gradient_wide_kernel(GradientArgs p, const uint16_t* wide)
{
    constexpr int kTA = 128, kTK = 512, kPartBytes = kTA * 64;
    // (six arrays and not one: the compiler waits for what fills an array from memory before it lets anybody use it)
    __shared__ __align__(1024) int8_t s_g0[2 * kPartBytes];
    __shared__ __align__(1024) int8_t s_g1[2 * kPartBytes];
    __shared__ __align__(1024) int8_t s_g2[2 * kPartBytes];
    __shared__ __align__(1024) int8_t s_q0[kTK * 64];
    __shared__ __align__(1024) int8_t s_q1[kTK * 64];
    __shared__ __align__(1024) int8_t s_q2[kTK * 64];
    int8_t* const s_g[3] = {s_g0, s_g1, s_g2};
    int8_t* const s_q[3] = {s_q0, s_q1, s_q2};
    __shared__ int s_lift[kTA];
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int a0 = blockIdx.x * kTA, k0 = blockIdx.y * kTK, slab = blockIdx.z, chunk = wave % 4 * 8;
    const Range range = slab_of(listed(p.frames, p.rows), slab, p.slabs);
    const int steps = (range.last - range.first + 31) / 32;
    const StepRows list(p, range, chunk + lane % 8);
    if (static_cast<int>(threadIdx.x) < kTA) {
        uint32_t most = 0;
        if (a0 + static_cast<int>(threadIdx.x) < p.A)
#pragma unroll 16
            for (int b = 0; b < kColumnSlabs; ++b) {
                const uint32_t m = p.largest[static_cast<int64_t>(b) * p.A + a0 + threadIdx.x];
                most = most > m ? most : m;
            }
        s_lift[threadIdx.x] = lift_of(most);
    }
    __syncthreads();
    // What this lane brings: symbol `symbol` of rows `chunk` .., and a sixty-fourth of four KiB of whole numbers.  (Symbols behind the last and
    // columns behind a row's bytes are others' once more: what becomes of them is not written.)
    const int symbol = wave / 4 * 64 + lane;
    const float lift = ldexpf(1.0f, s_lift[symbol]);
    const uint32_t at = static_cast<uint32_t>(a0 + symbol < p.A ? a0 + symbol : p.A - 1) * static_cast<uint32_t>(sizeof(T));
    const int8_t* numbers = reinterpret_cast<const int8_t*>(wide) + static_cast<int64_t>(range.first / 32) * p.pitch * 64;
    const uint32_t step_bytes = static_cast<uint32_t>(p.pitch) * 64, lane_bytes = lane * 16;
    // (behind a slab's last step that step's once more: multiplied by gradients that are 0, or by nobody)
    const auto fill = [&](int buffer, int step, int j) {
        const int k = k0 + (j * 8 + wave) * 16;
        to_lds(numbers + (k < p.pitch ? k : 0) * 64 + lane_bytes, s_q[buffer] + (j * 8 + wave) * 1024);
        if (j == 3) numbers += step + 1 < steps ? step_bytes : 0;
    };
    uint4v part[2];
    // Two rows' gradients, split, and the write of eight rows' parts with the last of them.
    const auto split = [&](const Eight& e, int buffer, int j) {
        const float c[2] = {gradient_in<T>(e.g[j]) * scale_of(e, j) * lift, gradient_in<T>(e.g[j + 1]) * scale_of(e, j + 1) * lift};
        const half2 high = {static_cast<_Float16>(c[0]), static_cast<_Float16>(c[1])};
        const half2 low = {static_cast<_Float16>(c[0] - static_cast<float>(high[0])), static_cast<_Float16>(c[1] - static_cast<float>(high[1]))};
        part[0][j / 2] = __builtin_bit_cast(uint32_t, high);
        part[1][j / 2] = __builtin_bit_cast(uint32_t, low);
        if (j != 6) return;
#pragma unroll
        for (int b = 0; b < 2; ++b) *reinterpret_cast<uint4v*>(s_g[buffer] + b * kPartBytes + symbol * 64 + ((wave % 4 ^ lane / 4 % 4) * 16)) = part[b];
    };
    const int wave_a = wave / 4, wave_k = wave % 4;
    float16v sum[2][4] = {};
    half8 g[2][2][2], q[2][4];
    const auto fetch = [&](int buffer, int h, int n) {                       // (the n-th of a half's eight reads, in the order of the products)
        const int piece = ((h * 2 + lane / 32) ^ lane / 4 % 4) * 16;
        if (n < 4)
            q[h][n] = *reinterpret_cast<const half8*>(s_q[buffer] + ((wave_k * 4 + n) * 32 + lane % 32) * 64 + piece);
        else
            g[h][1 - (n - 4) / 2][n % 2] = *reinterpret_cast<const half8*>(s_g[buffer] + (1 - (n - 4) / 2) * kPartBytes + ((wave_a * 2 + n % 2) * 32 + lane % 32) * 64 + piece);
    };
    const auto product = [&](int n) {
        const int h = n / 16, b = 1 - n / 8 % 2, i = n / 4 % 2, k = n % 4;
        sum[i][k] = __builtin_amdgcn_mfma_f32_32x32x16_f16(g[h][b][i], q[h][k], sum[i][k], 0, 0, 0);
    };
    if (steps > 0) {
        // (A step's rows' numbers are asked for three steps before its rows.)
        Eight raw[3];
        int entry[3];
        uint32_t mine_at = at;
        const auto ask = [&](Eight& e, int j) { e.g[j] = gradient_of<T>(p, __builtin_amdgcn_readlane(e.row, j), mine_at); };
        const auto rows = [&](Eight& e, int row) { e.row = row, e.scale = p.scales[row < 0 ? 0 : row], mine_at = here(at, row); };
#pragma unroll
        for (int t = 0; t < 3; ++t) {
#pragma unroll
            for (int j = 0; j < 4; ++j) fill(t, t, j);
            if (t == 2) break;
            rows(raw[t], list.row(t, list.ask(t)));
#pragma unroll
            for (int j = 0; j < 8; ++j) ask(raw[t], j);
            clear(raw[t]);
#pragma unroll
            for (int j = 0; j < 8; j += 2) split(raw[t], t, j);
        }
#pragma unroll
        for (int j = 0; j < 3; ++j) {
            rows(raw[j], list.row(2 + j, list.ask(2 + j)));
#pragma unroll
            for (int i = 0; i < 8; ++i) ask(raw[j], i);
            entry[j] = list.ask(5 + j);
        }
        wait_and_meet<0>();
#pragma unroll
        for (int n = 0; n < 8; ++n) fetch(0, 0, n);
        for (int t0 = 0; t0 < steps; t0 += 3) {
#pragma unroll
            for (int s = 0; s < 3; ++s) {
                const int t = t0 + s;
                if (t >= steps) break;
                const int now = s, next = (s + 1) % 3, down = (s + 2) % 3;
                Eight& mine = raw[s];
                clear(mine);
                const int row = list.row(t + 5, entry[s]);
                // A wavefront's products and its other instructions run beside each other only if they come in turns, and LDS serves eight wavefronts'
                // reads beside the products only if they are spread over them.
#pragma unroll
                for (int n = 0; n < 32; ++n) {
                    __builtin_amdgcn_sched_barrier(0);
                    product(n);
                    if (n >= 2 && n < 10) fetch(now, 1, n - 2);
                    if (n >= 2 && n < 18 && n % 4 == 2) split(mine, down, n / 2 - 1);
                    if (n == 13) wait_and_meet<24>();   // (the next step's numbers are there: 24 requests came after theirs, 14 in each step)
                    if (n >= 14 && n < 18) fill(now, t + 3, n - 14);
                    if (n == 18) rows(mine, row);
                    if (n >= 20 && n < 28) fetch(next, 0, n - 20), ask(mine, n - 20);
                    if (n == 28) entry[s] = list.ask(t + 8);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    }
    float* const out = p.out + static_cast<int64_t>(slab) * p.A * p.H;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int v = 0; v < 16; ++v) {
            const int a = (wave_a * 2 + i) * 32 + 8 * (v / 4) + 4 * (lane / 32) + v % 4;
            const int lower = -s_lift[a];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int c = k0 + (wave_k * 4 + k) * 32 + lane % 32;
                if (a0 + a < p.A && c < p.H) out[static_cast<int64_t>(a0 + a) * p.H + c] = ldexpf(sum[i][k][v], lower);
            }
        }
}

// The slabs' sums, in order: of the weights' gradient, four to a thread (none where there is one slab), and, in the workgroups behind, of the bias's.
__global__ __launch_bounds__(256) void ctc_sum_slabs_kernel(const float* __restrict__ partials, int slabs, int64_t width, float* __restrict__ out,
                                                            unsigned blocks, const float* __restrict__ bias, int bias_slabs, int A,
                                                            float* __restrict__ dbias)
{
    if (blockIdx.x >= blocks) {
        const int a = static_cast<int>(blockIdx.x - blocks) * 256 + threadIdx.x;
        if (a >= A) return;
        double sum = 0.0;
#pragma unroll 16
        for (int s = 0; s < bias_slabs; ++s) sum += static_cast<double>(bias[static_cast<int64_t>(s) * A + a]);
        dbias[a] = static_cast<float>(sum);
        return;
    }
    const int64_t i = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) * 4;
    if (i >= width) return;
    if (i + 4 <= width) {
        float sum[4] = {};
#pragma unroll 8
        for (int s = 0; s < slabs; ++s) {
            const Vector<float> v = load_whole(partials + s * width + i);
#pragma unroll
            for (int k = 0; k < 4; ++k) sum[k] += v.v[k];
        }
        __builtin_memcpy(out + i, sum, sizeof(sum));
        return;
    }
    for (int64_t k = i; k < width; ++k) {
        float sum = 0.0f;
        for (int s = 0; s < slabs; ++s) sum += partials[s * width + k];
        out[k] = sum;
    }
}

unsigned blocks(int64_t items, int per_block) { return static_cast<unsigned>((items + per_block - 1) / per_block); }

// A grid of `groups` workgroups and some: a dimension has fewer than 2^32 threads, rows may be 2^30.
dim3 spread(unsigned groups)
{
    constexpr unsigned kAcross = 1u << 22;
    return groups <= kAcross ? dim3(groups) : dim3(kAcross, (groups + kAcross - 1) / kAcross);
}

// Enqueues a kernel and returns this launch's own error: hipGetLastError's could be one that the caller has met and dealt with long ago.
template <typename... P, typename... Args> int launch(void (*kernel)(P...), dim3 grid, int threads, hipStream_t s, const Args&... args)
{
    std::tuple<P...> held(args...);
    const hipError_t err = std::apply([&](auto&... p) {
        void* at[] = {const_cast<void*>(static_cast<const void*>(&p))...};
        return hipLaunchKernel(reinterpret_cast<const void*>(kernel), grid, dim3(threads), at, 0, s);
    }, held);
    if (err != hipSuccess) (void)hipGetLastError();     // (told by status, and by nothing else)
    return static_cast<int>(err);
}

template <typename T, bool NORM, int WAVES, int E> int launch_rows(const NormArgs& p, hipStream_t s)
{
    const unsigned groups = WAVES == 1 ? blocks(p.rows, 4) : static_cast<unsigned>(p.rows);
    return launch(ctc_rows_to_8_bits_kernel<T, WAVES, E, NORM>, spread(groups), WAVES == 1 ? 256 : WAVES * kWave, s, p);
}
template <typename T, bool NORM> int launch_to_8_bits(const NormArgs& p, hipStream_t s)
{
    const RowShape shape = row_shape(p.rows, p.H);
    switch (shape.waves) {
    case 1: return shape.elements == 8 ? launch_rows<T, NORM, 1, 8>(p, s) : launch_rows<T, NORM, 1, 16>(p, s);
    case 2: return shape.elements == 8 ? launch_rows<T, NORM, 2, 8>(p, s) : launch_rows<T, NORM, 2, 16>(p, s);
    case 4: return shape.elements == 8 ? launch_rows<T, NORM, 4, 8>(p, s) : launch_rows<T, NORM, 4, 16>(p, s);
    default:
        return shape.elements == 8    ? launch_rows<T, NORM, 8, 8>(p, s)
               : shape.elements == 16 ? launch_rows<T, NORM, 8, 16>(p, s)
                                      : launch_rows<T, NORM, 8, 32>(p, s);
    }
}

template <typename T> int launch_backward(const NormBackArgs& p, unsigned groups, hipStream_t s)
{
    const dim3 grid(groups);
    // As few wavefronts to a row as hold it in registers, for each wavefront more is one more to wait for in the row's sums (27200 rows
    // of 1024 bf16: one wavefront with 16 a lane 39 us, two with 8 50, four with 8 67; 5556 of 3204 fp32: four with 16 54.7, eight with 8 58.6),
    // until registers are what a compute unit runs out of (5600 of 1999 fp32: two with 16 37.3, four with 8 35.1; 4000 of 5000: eight with
    // 16 66, sixteen with 8 62).
    if (p.H <= 512) return launch(ctc_norm_backward_kernel<T, 1, 8>, grid, 256, s, p);
    if (p.H <= 1024) return launch(ctc_norm_backward_kernel<T, 1, 16>, grid, 256, s, p);
    if (p.H <= 2048) return launch(ctc_norm_backward_kernel<T, 4, 8>, grid, 256, s, p);
    if (p.H <= 4096) return launch(ctc_norm_backward_kernel<T, 4, 16>, grid, 256, s, p);
    if (p.H <= 8192) return launch(ctc_norm_backward_kernel<T, 16, 8>, grid, 1024, s, p);
    return launch(ctc_norm_backward_kernel<T, 8, 32>, grid, 512, s, p);
}

template <typename T, int WM, int WN> int launch_tiles(const LinearArgs& p, hipStream_t s)
{
    const int64_t tiles = static_cast<int64_t>(blocks(p.rows, 64 * WM)) * blocks(p.A, 64 * WN);
    return launch(ctc_linear_tiles_kernel<T, WM, WN>, dim3(blocks(tiles, 8) * 8), 256, s, p);
}
template <typename T> int launch_direct(const LinearArgs& p, hipStream_t s)
{
    return launch(ctc_linear_direct_kernel<T>, dim3(blocks(p.rows, 16) * blocks(p.A, 16)), 256, s, p);
}
template <typename T> int launch_product(const LinearArgs& p, ProductTile tile, hipStream_t s)
{
    if (tile.rows == 16) return launch_direct<T>(p, s);
    if (tile.symbols == 64) return tile.rows == 128 ? launch_tiles<T, 2, 1>(p, s) : launch_tiles<T, 1, 1>(p, s);
    return tile.symbols == 128 ? launch_tiles<T, 2, 2>(p, s) : launch_tiles<T, 4, 4>(p, s);
}

template <typename T> int launch_gradient(const GradientArgs& p, const GradientPlan& plan, float* workspace, hipStream_t s)
{
    const dim3 grid(blocks(p.A, plan.symbols), blocks(p.H, plan.columns), static_cast<unsigned>(p.slabs));
    if (plan.symbols == 32) return launch(ctc_weight_gradient_narrow_kernel<T, 1>, grid, 512, s, p);
    if (plan.symbols == 64) return launch(ctc_weight_gradient_narrow_kernel<T, 2>, grid, 512, s, p);
    uint16_t* const wide = reinterpret_cast<uint16_t*>(workspace + plan.wide_at);
    const unsigned columns = blocks(p.A, 2 * kWave);
    const int err = launch(ctc_gradient_prepare_kernel<T>, spread(columns * kColumnSlabs + blocks(p.rows, 32) * blocks(p.pitch, 256)), 256, s, p,
                           reinterpret_cast<uint32_t*>(workspace + plan.largest_at), wide, columns);
    return err ? err : launch(ctc_weight_gradient_wide_kernel<T>, grid, 512, s, p, wide);
}

}  // namespace

int launch_pack_frames(const int32_t* lengths, int T, int B, int32_t* frames, void* stream)
{
    return launch(ctc_pack_frames_kernel, spread(blocks(T, 4)), 256, static_cast<hipStream_t>(stream), lengths, T, B, frames);
}

int launch_quantize(const void* x, const int32_t* frames, int rows, int H, bool bf16, int8_t* q, float* scales, void* stream)
{
    const NormArgs p = {x, nullptr, nullptr, 0.0f, frames, rows, H, pitch_of(H), nullptr, q, scales};
    hipStream_t s = static_cast<hipStream_t>(stream);
    return bf16 ? launch_to_8_bits<bf16_t, false>(p, s) : launch_to_8_bits<float, false>(p, s);
}

int launch_norm(const void* x, const void* residual, const float* weight, float eps, const int32_t* frames, int rows, int H,
                bool bf16, void* sum, int8_t* q, float* scales, void* stream)
{
    const NormArgs p = {x, residual, weight, eps, frames, rows, H, pitch_of(H), sum, q, scales};
    hipStream_t s = static_cast<hipStream_t>(stream);
    return bf16 ? launch_to_8_bits<bf16_t, true>(p, s) : launch_to_8_bits<float, true>(p, s);
}

int launch_dequantize(const int8_t* q, const float* scales, const int32_t* frames, int rows, int H, bool bf16, void* out,
                      void* stream)
{
    const dim3 grid = spread(blocks(rows, 4));
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (bf16) return launch(ctc_rows_from_8_bits_kernel<bf16_t>, grid, 256, s, q, scales, frames, rows, H, pitch_of(H), static_cast<bf16_t*>(out));
    return launch(ctc_rows_from_8_bits_kernel<float>, grid, 256, s, q, scales, frames, rows, H, pitch_of(H), static_cast<float*>(out));
}

int launch_norm_backward(const void* dy, const void* sum, const float* weight, float eps, const void* dresidual,
                         const int32_t* frames, int rows, int H, bool bf16, void* dsum, float* dweight, float* partials,
                         void* stream)
{
    hipStream_t s = static_cast<hipStream_t>(stream);
    const int groups = norm_partials(rows, H);
    const NormBackArgs p = {dy, sum, weight, eps, dresidual, frames, rows, H, dsum, dweight ? partials : nullptr};
    const int err = bf16 ? launch_backward<bf16_t>(p, static_cast<unsigned>(groups), s) : launch_backward<float>(p, static_cast<unsigned>(groups), s);
    if (err || !dweight) return err;
    return launch(ctc_sum_partials_kernel, dim3(blocks(H, 16)), 1024, s, partials, groups, static_cast<int64_t>(H), static_cast<int64_t>(H), dweight);
}

int launch_linear(const int8_t* q, const float* scales, const int8_t* weight_q, const float* weight_scales, const float* bias,
                  const int32_t* frames, int rows, int H, int A, bool bf16, void* logits, void* stream)
{
    const LinearArgs p = {q, scales, weight_q, weight_scales, bias, frames, rows, A, pitch_of(H), logits};
    const ProductTile tile = product_tile(rows, H, A, frames != nullptr);
    hipStream_t s = static_cast<hipStream_t>(stream);
    return bf16 ? launch_product<bf16_t>(p, tile, s) : launch_product<float>(p, tile, s);
}

int launch_weight_gradient(const void* grads, const int8_t* q, const float* scales, const int32_t* frames, int rows, int H,
                           int A, bool bf16, const GradientPlan& plan, float* dweight, float* dbias, float* workspace, void* stream)
{
    hipStream_t s = static_cast<hipStream_t>(stream);
    const int64_t weights = static_cast<int64_t>(A) * H;
    float* const bias = workspace + plan.bias_at;
    const GradientArgs p = {grads, q, scales, frames, rows, H, A, pitch_of(H), plan.slabs,
                            plan.slabs > 1 ? workspace : dweight, dbias ? bias : nullptr,
                            reinterpret_cast<const uint32_t*>(workspace + plan.largest_at)};
    const int err = bf16 ? launch_gradient<bf16_t>(p, plan, workspace, s) : launch_gradient<float>(p, plan, workspace, s);
    const unsigned weight_blocks = plan.slabs > 1 ? blocks(weights, 1024) : 0, bias_blocks = dbias ? blocks(A, 256) : 0;
    if (err || weight_blocks + bias_blocks == 0) return err;
    return launch(ctc_sum_slabs_kernel, dim3(weight_blocks + bias_blocks), 256, s, workspace, plan.slabs, weights, dweight, weight_blocks, bias,
                  plan.bias_slabs, A, dbias);
}

}  // namespace layer
