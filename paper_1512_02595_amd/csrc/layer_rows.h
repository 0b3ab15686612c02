// What the kernels of the layers share: elements of a row and vectors of them, lists of rows, sums over lanes, whole numbers, launches.
#ifndef LAYER_ROWS_H
#define LAYER_ROWS_H

#include <hip/hip_runtime.h>

#include <cstdint>
#include <tuple>

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

// ---- whole numbers ----------------------------------------------------------------------------------------------

constexpr uint32_t kInfinity = 0x7f800000u;

// The whole number nearest to LEVELS |u| / m, ties to even, exactly: `inverse` is LEVELS / m to within half a step, so the
// product is off by less than 2^-16 (127 * 2^-23); where it comes that near to the middle between two whole numbers, 2 LEVELS |u|
// is compared with (2 j + 1) m, both of which fp64 holds (32 bits).
template <int LEVELS = 127> __device__ __forceinline__ int level(float u, float m, float inverse)
{
    const float a = fabsf(u), t = a * inverse;
    int k = static_cast<int>(rintf(t));
    if (fabsf(t - static_cast<float>(k)) > 0.5f - 0x1p-15f) {
        const int j = static_cast<int>(t);
        const double twice = 2.0 * LEVELS * static_cast<double>(a), middle = static_cast<double>(2 * j + 1) * static_cast<double>(m);
        k = twice > middle || (twice == middle && (j & 1)) ? j + 1 : j;
    }
    return u < 0.0f ? -k : k;
}

// ---- launches ---------------------------------------------------------------------------------------------------

inline unsigned blocks(int64_t items, int per_block) { return static_cast<unsigned>((items + per_block - 1) / per_block); }

// A grid of `groups` workgroups and some: a dimension has fewer than 2^32 threads, rows may be 2^30.
inline dim3 spread(unsigned groups)
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

}  // namespace
}  // namespace layer

#endif  // LAYER_ROWS_H
