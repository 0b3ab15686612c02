// Kernels of the norms around a block (ctc_block.h).

#include <hip/hip_runtime.h>

#include "layer_block_internal.h"
#include "layer_gate.h"
#include "layer_rows.h"

namespace layer {
namespace {

// Four of a weight's floats, ones where there is no weight.
__device__ __forceinline__ Vector<float> weights_at(const float* w, int col, int H)
{
    if (w) return load_vector(w, col, H);
    return {{1.0f, 1.0f, 1.0f, 1.0f}};
}

// A wavefront's sum in every lane, without LDS: lanes one and two apart, the other four of eight, the other eight of sixteen, the neighbouring sixteen, the
// other half.  (The swap of sixteens, or halves, of a number with itself leaves the one in the first result, the other in the second.)
template <int CONTROL> __device__ __forceinline__ double from_lane(double v)
{
    const uint64_t bits = __builtin_bit_cast(uint64_t, v);
    const int low = __builtin_amdgcn_mov_dpp(static_cast<int>(bits), CONTROL, 0xf, 0xf, true);
    const int high = __builtin_amdgcn_mov_dpp(static_cast<int>(bits >> 32), CONTROL, 0xf, 0xf, true);
    return __builtin_bit_cast(double, static_cast<uint64_t>(static_cast<uint32_t>(high)) << 32 | static_cast<uint32_t>(low));
}
template <typename F> __device__ __forceinline__ double both_of(double v, F swap)
{
    const uint64_t bits = __builtin_bit_cast(uint64_t, v);
    const auto low = swap(static_cast<uint32_t>(bits)), high = swap(static_cast<uint32_t>(bits >> 32));
    return __builtin_bit_cast(double, static_cast<uint64_t>(high[0]) << 32 | low[0]) + __builtin_bit_cast(double, static_cast<uint64_t>(high[1]) << 32 | low[1]);
}
__device__ __forceinline__ double lanes_sum(double v)
{
    v += from_lane<0xB1>(v);                        // quad_perm 1 0 3 2
    v += from_lane<0x4E>(v);                        // quad_perm 2 3 0 1
    v += from_lane<0x141>(v);                       // row_half_mirror
    v += from_lane<0x140>(v);                       // row_mirror
    v = both_of(v, [](uint32_t w) { return __builtin_amdgcn_permlane16_swap(w, w, false, false); });
    return both_of(v, [](uint32_t w) { return __builtin_amdgcn_permlane32_swap(w, w, false, false); });
}

// Sums over a row's threads: a wavefront's, or those of all wavefronts of the workgroup through LDS.  `s_sums` is one of two buffers that a row's
// reductions take by turns, so that one barrier each is enough: who writes a buffer again has passed the barrier that its readers came to.
template <int WAVES, int N> __device__ __forceinline__ void row_sums(double (&v)[N], double (*s_sums)[WAVES], int lane, int wave)
{
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = lanes_sum(v[i]);
    if constexpr (WAVES > 1) {
        if (lane == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) s_sums[i][wave] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            v[i] = 0.0;
#pragma unroll
            for (int o = 0; o < WAVES; ++o) v[i] += s_sums[i][o];
        }
    }
}

// A row to a wavefront (four rows to a workgroup) or to all wavefronts of a workgroup, which take rows in turn; a row stays in registers (E elements
// a thread) from its one reading to its writing.
template <typename T, int WAVES, int E>
__global__ __launch_bounds__(WAVES == 1 ? 256 : WAVES * kWave) void ctc_block_norm_kernel(BlockNormArgs p)
{
    constexpr int kE = Vector<T>::kElements, kVectors = E / kE, kWidth = WAVES * kWave, kRows = WAVES == 1 ? 4 : 1;
    __shared__ double s_sums[2][1][WAVES];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int thread = WAVES == 1 ? lane : threadIdx.x;
    const int n = listed(p.frames, p.rows);
    float after[E], before[E];
#pragma unroll
    for (int v = 0; v < E / 4; ++v) {
        const int col = ((v * 4 / kE) * kWidth + thread) * kE + v * 4 % kE;
        const Vector<float> a = weights_at(p.weight_after, col, p.H), s = weights_at(p.scale, col, p.H), w = weights_at(p.weight_before, col, p.H);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            after[4 * v + j] = a.v[j] * s.v[j];
            before[4 * v + j] = w.v[j];
        }
    }
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * kRows + (WAVES == 1 ? wave : 0); i < n; i += static_cast<int64_t>(gridDim.x) * kRows) {
        const int r = row_of(p.frames, p.rows, static_cast<int>(i));
        if (r < 0) continue;
        const int64_t row = static_cast<int64_t>(r) * p.H;
        Vector<T> x[kVectors], g[kVectors], z[kVectors];
#pragma unroll
        for (int v = 0; v < kVectors; ++v) {
            const int col = (v * kWidth + thread) * kE;
            x[v] = load_vector(static_cast<const T*>(p.x) + row, col, p.H);
            if (p.gate) g[v] = load_vector(static_cast<const T*>(p.gate) + r * p.gate_pitch, col, p.H);
            z[v] = Vector<T>{};
            if (p.residual) z[v] = load_vector(static_cast<const T*>(p.residual) + row, col, p.H);
        }
        double sum[1] = {};
#pragma unroll
        for (int k = 0; k < E; ++k) {
            const double f = static_cast<double>(widen(x[k / kE].v[k % kE]));
            sum[0] += f * f;
        }
        row_sums<WAVES, 1>(sum, s_sums[0], lane, wave);
        float f = static_cast<float>(1.0 / sqrt(sum[0] / p.H + static_cast<double>(p.eps)));
        sum[0] = 0.0;
#pragma unroll
        for (int k = 0; k < E; ++k) {
            float y = widen(x[k / kE].v[k % kE]) * f * after[k];
            if (p.gate) {
                const float gate = widen(g[k / kE].v[k % kE]);
                y *= gate * share_of<sizeof(T) == 4>(gate);
            }
            const T rounded = narrow<T>(y + widen(z[k / kE].v[k % kE]));
            z[k / kE].v[k % kE] = rounded;
            const double d = static_cast<double>(widen(rounded));
            sum[0] += d * d;
        }
        if (p.sum)
#pragma unroll
            for (int v = 0; v < kVectors; ++v) store_vector(static_cast<T*>(p.sum) + row, (v * kWidth + thread) * kE, p.H, z[v]);
        if (!p.normed) {
            if constexpr (WAVES > 1) __syncthreads();                   // (the buffer is written again for the next row)
            continue;
        }
        row_sums<WAVES, 1>(sum, s_sums[1], lane, wave);
        f = static_cast<float>(1.0 / sqrt(sum[0] / p.H + static_cast<double>(p.eps)));
#pragma unroll
        for (int v = 0; v < kVectors; ++v) {
#pragma unroll
            for (int k = 0; k < kE; ++k) z[v].v[k] = narrow<T>(widen(z[v].v[k]) * f * before[v * kE + k]);
            store_vector(static_cast<T*>(p.normed) + row, (v * kWidth + thread) * kE, p.H, z[v]);
        }
    }
}

template <typename T, int WAVES, int E>
__global__ __launch_bounds__(WAVES == 1 ? 256 : WAVES * kWave) void ctc_block_norm_backward_kernel(BlockNormBackArgs p)
{
    constexpr int kE = Vector<T>::kElements, kVectors = E / kE, kWidth = WAVES * kWave, kRows = WAVES == 1 ? 4 : 1;
    __shared__ double s_first[3][WAVES], s_second[1][WAVES];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int thread = WAVES == 1 ? lane : threadIdx.x;
    const int n = listed(p.frames, p.rows);
    float after[E], before[E], sum_before[E], sum_q[E];
#pragma unroll
    for (int v = 0; v < E / 4; ++v) {
        const int col = ((v * 4 / kE) * kWidth + thread) * kE + v * 4 % kE;
        const Vector<float> a = weights_at(p.weight_after, col, p.H), s = weights_at(p.scale, col, p.H), w = weights_at(p.weight_before, col, p.H);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            after[4 * v + j] = a.v[j] * s.v[j];
            before[4 * v + j] = w.v[j];
        }
    }
#pragma unroll
    for (int k = 0; k < E; ++k) sum_before[k] = sum_q[k] = 0.0f;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * kRows + (WAVES == 1 ? wave : 0); i < n; i += static_cast<int64_t>(gridDim.x) * kRows) {
        const int r = row_of(p.frames, p.rows, static_cast<int>(i));
        if (r < 0) continue;
        const int64_t row = static_cast<int64_t>(r) * p.H;
        Vector<T> x[kVectors], g[kVectors], z[kVectors], dy[kVectors], dz[kVectors];
#pragma unroll
        for (int v = 0; v < kVectors; ++v) {
            const int col = (v * kWidth + thread) * kE;
            x[v] = load_vector(static_cast<const T*>(p.x) + row, col, p.H);
            if (p.gate) g[v] = load_vector(static_cast<const T*>(p.gate) + r * p.gate_pitch, col, p.H);
            z[v] = dy[v] = dz[v] = Vector<T>{};
            if (p.dnormed) {
                z[v] = load_vector(static_cast<const T*>(p.sum) + row, col, p.H);
                dy[v] = load_vector(static_cast<const T*>(p.dnormed) + row, col, p.H);
            }
            if (p.dsum) dz[v] = load_vector(static_cast<const T*>(p.dsum) + row, col, p.H);
        }
        double sums[3] = {};
#pragma unroll
        for (int k = 0; k < E; ++k) {
            const double a = static_cast<double>(widen(x[k / kE].v[k % kE])), b = static_cast<double>(widen(z[k / kE].v[k % kE]));
            sums[0] += a * a;
            sums[1] += b * b;
            sums[2] += static_cast<double>(widen(dy[k / kE].v[k % kE]) * before[k]) * b;
        }
        row_sums<WAVES, 3>(sums, s_first, lane, wave);
        const double v1 = sums[0] / p.H + static_cast<double>(p.eps), v2 = sums[1] / p.H + static_cast<double>(p.eps);
        // (the mean's share without the factor: with it, it would vanish in fp32 for rows of 1e20 and more)
        const float f1 = static_cast<float>(1.0 / sqrt(v1)), f2 = static_cast<float>(1.0 / sqrt(v2)), c2 = static_cast<float>(sums[2] / p.H / v2);
        double along[1] = {};
        float e[E];
#pragma unroll
        for (int k = 0; k < E; ++k) {
            const float dyk = widen(dy[k / kE].v[k % kE]), zk = widen(z[k / kE].v[k % kE]), xk = widen(x[k / kE].v[k % kE]);
            const float d = (dyk * before[k] - zk * c2) * f2 + widen(dz[k / kE].v[k % kE]);
            sum_before[k] += dyk * (zk * f2);
            dz[k / kE].v[k % kE] = narrow<T>(d);
            float a = 1.0f;
            const float normed = xk * f1;
            if (p.gate) {
                const float gate = widen(g[k / kE].v[k % kE]);
                const Gate s = gate_of<sizeof(T) == 4>(gate);
                a = gate * s.z;
                g[k / kE].v[k % kE] = narrow<T>(d * after[k] * normed * (s.z + a * s.stays));
            }
            sum_q[k] += d * a * normed;
            e[k] = d * a * after[k];
            along[0] += static_cast<double>(e[k]) * static_cast<double>(xk);
        }
        row_sums<WAVES, 1>(along, s_second, lane, wave);
        const float c1 = static_cast<float>(along[0] / p.H / v1);
#pragma unroll
        for (int v = 0; v < kVectors; ++v) {
            const int col = (v * kWidth + thread) * kE;
#pragma unroll
            for (int k = 0; k < kE; ++k) x[v].v[k] = narrow<T>((e[v * kE + k] - widen(x[v].v[k]) * c1) * f1);
            store_vector(static_cast<T*>(p.dx) + row, col, p.H, x[v]);
            if (p.gate) store_vector(static_cast<T*>(p.dgate) + r * p.gate_pitch, col, p.H, g[v]);
            if (p.dresidual) store_vector(static_cast<T*>(p.dresidual) + row, col, p.H, dz[v]);
        }
    }
    if (!p.partials) return;
    float* out = p.partials + static_cast<int64_t>(blockIdx.x) * 2 * p.H;
    if constexpr (WAVES == 1) {
        // The four wavefronts' sums, one after another.
        __shared__ float s_dw[2 * E][kWave];
        for (int o = 0; o < 4; ++o) {
            if (wave == o) {
#pragma unroll
                for (int k = 0; k < E; ++k) {
                    if (o) {
                        sum_before[k] += s_dw[k][lane];
                        sum_q[k] += s_dw[E + k][lane];
                    }
                    s_dw[k][lane] = sum_before[k];
                    s_dw[E + k][lane] = sum_q[k];
                }
            }
            __syncthreads();
        }
        if (wave != 3) return;
    }
#pragma unroll
    for (int v = 0; v < E / 4; ++v) {
        const int col = ((v * 4 / kE) * kWidth + thread) * kE + v * 4 % kE;
        Vector<float> a, b;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            a.v[j] = sum_before[4 * v + j];
            b.v[j] = sum_q[4 * v + j];
        }
        store_vector(out, col, p.H, a);
        store_vector(out + p.H, col, p.H, b);
    }
}

// Rows of more than 4096, whose tensors a compute unit's registers do not hold beside the sums: a workgroup to a row, which reads it twice from memory and once more from the
// caches, and adds to its own partial sums there.
template <typename T> __global__ __launch_bounds__(1024) void ctc_block_norm_backward_wide_kernel(BlockNormBackArgs p)
{
    constexpr int kE = Vector<T>::kElements, kStep = 1024 * kE;
    __shared__ double s_first[3][16], s_second[1][16];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int n = listed(p.frames, p.rows);
    float* const sums_out = p.partials ? p.partials + static_cast<int64_t>(blockIdx.x) * 2 * p.H : nullptr;
    if (sums_out)
        for (int col = threadIdx.x * kE; col < p.H; col += kStep)
            for (int k = 0; k < kE && col + k < p.H; ++k) sums_out[col + k] = sums_out[p.H + col + k] = 0.0f;
    for (int64_t i = blockIdx.x; i < n; i += gridDim.x) {
        const int r = row_of(p.frames, p.rows, static_cast<int>(i));
        if (r < 0) continue;
        const int64_t row = static_cast<int64_t>(r) * p.H;
        const T* const at_x = static_cast<const T*>(p.x) + row;
        const T* const at_z = static_cast<const T*>(p.sum) + row;
        const T* const at_dy = static_cast<const T*>(p.dnormed) + row;
        double sums[3] = {};
        for (int col = threadIdx.x * kE; col < p.H; col += kStep) {
            const Vector<T> x = load_vector(at_x, col, p.H);
            Vector<T> z{}, dy{};
            if (p.dnormed) {
                z = load_vector(at_z, col, p.H);
                dy = load_vector(at_dy, col, p.H);
            }
#pragma unroll
            for (int v = 0; v < kE; v += 4) {
                const Vector<float> w = weights_at(p.weight_before, col + v, p.H);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const double a = static_cast<double>(widen(x.v[v + j])), b = static_cast<double>(widen(z.v[v + j]));
                    sums[0] += a * a;
                    sums[1] += b * b;
                    sums[2] += static_cast<double>(widen(dy.v[v + j]) * w.v[j]) * b;
                }
            }
        }
        row_sums<16, 3>(sums, s_first, lane, wave);
        const double v1 = sums[0] / p.H + static_cast<double>(p.eps), v2 = sums[1] / p.H + static_cast<double>(p.eps);
        const float f1 = static_cast<float>(1.0 / sqrt(v1)), f2 = static_cast<float>(1.0 / sqrt(v2)), c2 = static_cast<float>(sums[2] / p.H / v2);
        double along[1] = {};
        float c1 = 0.0f;
        // Twice: for the sum along x and what needs no such sum but the partial sums, then for what is written, which may be in the inputs' place.
#pragma unroll 1
        for (int pass = 0; pass < 2; ++pass) {
            for (int col = threadIdx.x * kE; col < p.H; col += kStep) {
                const Vector<T> x = load_vector(at_x, col, p.H);
                Vector<T> g{}, z{}, dy{}, dz{};
                if (p.gate) g = load_vector(static_cast<const T*>(p.gate) + r * p.gate_pitch, col, p.H);
                if (p.dnormed) {
                    z = load_vector(at_z, col, p.H);
                    dy = load_vector(at_dy, col, p.H);
                }
                if (p.dsum) dz = load_vector(static_cast<const T*>(p.dsum) + row, col, p.H);
                Vector<T> dx;
#pragma unroll
                for (int v = 0; v < kE; v += 4) {
                    const Vector<float> wa = weights_at(p.weight_after, col + v, p.H), ws = weights_at(p.scale, col + v, p.H);
                    const Vector<float> wb = weights_at(p.weight_before, col + v, p.H);
                    Vector<float> more[2] = {};
                    if (sums_out && !pass) {
                        more[0] = load_vector(sums_out, col + v, p.H);
                        more[1] = load_vector(sums_out + p.H, col + v, p.H);
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float dyk = widen(dy.v[v + j]), zk = widen(z.v[v + j]), xk = widen(x.v[v + j]), after = wa.v[j] * ws.v[j];
                        const float d = (dyk * wb.v[j] - zk * c2) * f2 + widen(dz.v[v + j]);
                        float a = 1.0f;
                        const float normed = xk * f1;
                        if (p.gate) {
                            const float gate = widen(g.v[v + j]);
                            const Gate s = gate_of<sizeof(T) == 4>(gate);
                            a = gate * s.z;
                            g.v[v + j] = narrow<T>(d * after * normed * (s.z + a * s.stays));
                        }
                        const float e = d * a * after;
                        along[0] += pass ? 0.0 : static_cast<double>(e) * static_cast<double>(xk);
                        more[0].v[j] += dyk * (zk * f2);
                        more[1].v[j] += d * a * normed;
                        dx.v[v + j] = narrow<T>((e - xk * c1) * f1);
                        dz.v[v + j] = narrow<T>(d);
                    }
                    if (sums_out && !pass) {
                        for (int j = 0; j < 4 && col + v + j < p.H; ++j) {
                            sums_out[col + v + j] = more[0].v[j];
                            sums_out[p.H + col + v + j] = more[1].v[j];
                        }
                    }
                }
                if (!pass) continue;
                store_vector(static_cast<T*>(p.dx) + row, col, p.H, dx);
                if (p.gate) store_vector(static_cast<T*>(p.dgate) + r * p.gate_pitch, col, p.H, g);
                if (p.dresidual) store_vector(static_cast<T*>(p.dresidual) + row, col, p.H, dz);
            }
            if (pass) break;
            row_sums<16, 1>(along, s_second, lane, wave);
            c1 = static_cast<float>(along[0] / p.H / v1);
        }
    }
}

// The weights' gradients from the workgroups' sums, added in fp64: of the two sums a column has, one is dweight_before, of the other the two weights
// that it meets as a product each have their share.  64 rows by 16 columns to a workgroup at once.
__global__ __launch_bounds__(1024) void ctc_block_norm_weights_kernel(const float* __restrict__ partials, int count, int H,
                                                                      const float* __restrict__ weight_after, const float* __restrict__ scale,
                                                                      float* __restrict__ dweight_after, float* __restrict__ dscale,
                                                                      float* __restrict__ dweight_before)
{
    __shared__ double s_sum[16][16];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int col = blockIdx.x * 16 + lane % 16;
    double sum = 0.0;
    if (col < 2 * H)
#pragma unroll 16
        for (int p = wave * 4 + lane / 16; p < count; p += 64) sum += static_cast<double>(partials[static_cast<int64_t>(p) * 2 * H + col]);
    sum += __shfl_xor(sum, 16, kWave);
    sum += __shfl_xor(sum, 32, kWave);
    if (lane < 16) s_sum[wave][lane] = sum;
    __syncthreads();
    if (threadIdx.x >= 16 || col >= 2 * H) return;
#pragma unroll
    for (int g = 1; g < 16; ++g) sum += s_sum[g][lane];
    if (col < H) {
        if (dweight_before) dweight_before[col] = static_cast<float>(sum);
        return;
    }
    const int k = col - H;
    if (dweight_after) dweight_after[k] = static_cast<float>(scale ? sum * static_cast<double>(scale[k]) : sum);
    if (dscale) dscale[k] = static_cast<float>(weight_after ? sum * static_cast<double>(weight_after[k]) : sum);
}

template <typename T> int launch_norm_of(const BlockNormArgs& p, hipStream_t s)
{
    const int per_group = p.H <= 1024 ? 4 : 1;
    const int64_t groups = (static_cast<int64_t>(p.rows) + per_group - 1) / per_group;
    const dim3 grid(static_cast<unsigned>(groups < 8192 ? groups : 8192));
    if (p.H <= 512) return launch(ctc_block_norm_kernel<T, 1, 8>, grid, 256, s, p);
    if (p.H <= 1024) return launch(ctc_block_norm_kernel<T, 1, 16>, grid, 256, s, p);
    if (p.H <= 2048) return launch(ctc_block_norm_kernel<T, 4, 8>, grid, 256, s, p);
    if (p.H <= 4096) return launch(ctc_block_norm_kernel<T, 4, 16>, grid, 256, s, p);
    if (p.H <= 8192) return launch(ctc_block_norm_kernel<T, 16, 8>, grid, 1024, s, p);
    return launch(ctc_block_norm_kernel<T, 16, 16>, grid, 1024, s, p);
}

template <typename T> int launch_backward_of(const BlockNormBackArgs& p, unsigned groups, hipStream_t s)
{
    const dim3 grid(groups);
    if (p.H <= 512) return launch(ctc_block_norm_backward_kernel<T, 1, 8>, grid, 256, s, p);
    if (p.H <= 1024) return launch(ctc_block_norm_backward_kernel<T, 2, 8>, grid, 128, s, p);
    if (p.H <= 2048) return launch(ctc_block_norm_backward_kernel<T, 4, 8>, grid, 256, s, p);
    if (p.H <= 4096) return launch(ctc_block_norm_backward_kernel<T, 8, 8>, grid, 512, s, p);
    return launch(ctc_block_norm_backward_wide_kernel<T>, grid, 1024, s, p);
}

}  // namespace

int launch_block_norm(const BlockNormArgs& p, bool bf16, void* stream)
{
    hipStream_t s = static_cast<hipStream_t>(stream);
    return bf16 ? launch_norm_of<bf16_t>(p, s) : launch_norm_of<float>(p, s);
}

int launch_block_norm_backward(const BlockNormBackArgs& p, bool bf16, float* dweight_after, float* dscale, float* dweight_before, void* stream)
{
    hipStream_t s = static_cast<hipStream_t>(stream);
    const int groups = block_norm_groups(p.rows, p.H);
    const int err = bf16 ? launch_backward_of<bf16_t>(p, static_cast<unsigned>(groups), s) : launch_backward_of<float>(p, static_cast<unsigned>(groups), s);
    if (err || !p.partials) return err;
    return launch(ctc_block_norm_weights_kernel, dim3(blocks(2 * static_cast<int64_t>(p.H), 16)), 1024, s, p.partials, groups, p.H, p.weight_after,
                  p.scale, dweight_after, dscale, dweight_before);
}

}  // namespace layer
