// Device code of the root-mean-square norm (sm_100a).
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "checkpoint.cuh"

namespace star {

struct NormArgs {
    const void *x;
    const void *residual;    // may be null
    void *total;             // may be null
    void *y;
    const void *gain;        // may be null
    float *rstd;             // may be null
    Kept kept;               // codes may be null
    int64_t ld_x, ld_residual, ld_total, ld_y;
    int64_t rows;
    int cols;
    float eps, inv_cols;
    int wide;                // every row of every matrix is 32-byte aligned
};

struct NormGradArgs {
    void *dx;
    const void *dy;
    const void *total;       // or null, and then kept
    Kept kept;
    const void *gain;        // may be null
    const float *rstd;
    const void *d_total;     // may be null
    int64_t ld_dx, ld_dy, ld_total, ld_d_total;
    int64_t rows;
    int cols;
    float inv_cols;
    int wide;
    float *partial;          // a row of cols sums for each block; null: the gain has no gradient
};

// 1 / sqrt(mean of squares + eps), NaN where the squares' sum is none of binary32.
__device__ __forceinline__ float norm_factor(float squares, float inv_cols, float eps)
{
    if (!(squares < INFINITY)) return NAN;
    return __fdiv_rn(1.0f, __fsqrt_rn(__fmaf_rn(squares, inv_cols, eps)));
}

__device__ __forceinline__ float rounded_to(float x, const GradF32 *) { return x; }
__device__ __forceinline__ float rounded_to(float x, const GradBF16 *) { return __uint_as_float(pack_bf16(x, 0.0f) << 16); }
// x as a buffer of type G holds it.
template <typename G> __device__ __forceinline__ float as_stored(float x) { return rounded_to(x, static_cast<const G *>(nullptr)); }

// The sum over a block's threads, in every thread, in a fixed order.  `part` holds a
// number for each warp and is free again after the next barrier.
template <int THREADS> __device__ __forceinline__ float block_total(float x, float *part)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x = __fadd_rn(x, __shfl_xor_sync(0xffffffffu, x, o));
    if constexpr (THREADS > 32) {
        if (threadIdx.x % 32 == 0) part[threadIdx.x / 32] = x;
        __syncthreads();
        x = threadIdx.x % 32 < THREADS / 32 ? part[threadIdx.x % 32] : 0.0f;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) x = __fadd_rn(x, __shfl_xor_sync(0xffffffffu, x, o));
    }
    return x;
}

// ---------------------------------------------------------------------------
// Any alignment: a block to a row, a warp on blocks of 32 columns, a lane to a
// column; the row is read again for its results.
// ---------------------------------------------------------------------------
constexpr int kNormThreads = 256;

template <typename G, typename W>
__global__ void __launch_bounds__(kNormThreads) star_rms_norm_loose_kernel(const __grid_constant__ NormArgs a)
{
    __shared__ float part[2][kNormThreads / 32];
    wait_for_primary();
    int parity = 0;
    const int padded = (a.cols + 31) / 32 * 32;
    for (int64_t t = blockIdx.x; t < a.rows; t += gridDim.x, parity ^= 1) {
        const char *x = static_cast<const char *>(a.x) + t * a.ld_x * G::kBytes;
        const char *residual = static_cast<const char *>(a.residual) + t * a.ld_residual * G::kBytes;
        char *total = static_cast<char *>(a.total) + t * a.ld_total * G::kBytes;
        const auto stream = [&](int c) {
            const float v = load_value<G>(x, c);
            return a.residual ? as_stored<G>(__fadd_rn(v, load_value<G>(residual, c))) : v;
        };
        float squares = 0.0f;
        for (int c = threadIdx.x; c < a.cols; c += kNormThreads) {
            const float s = stream(c);
            if (a.total) store_value<G>(total, c, s);
            squares = __fmaf_rn(s, s, squares);
        }
        const float r = norm_factor(block_total<kNormThreads>(squares, part[parity]), a.inv_cols, a.eps);
        if (threadIdx.x == 0 && a.rstd) a.rstd[t] = r;
        char *y = static_cast<char *>(a.y) + t * a.ld_y * G::kBytes;
        // What was written to `total` is read back by the thread that wrote it.
        for (int c = threadIdx.x; c < padded; c += kNormThreads) {
            float v = 0.0f;
            if (c < a.cols) {
                v = __fmul_rn(a.total ? load_value<G>(total, c) : stream(c), r);
                if (a.gain) v = __fmul_rn(v, load_value<W>(a.gain, c));
                v = as_stored<G>(v);
                store_value<G>(y, c, v);
            }
            if (a.kept.codes) {
                const int s = scale_byte(__reduce_max_sync(0xffffffffu, __float_as_uint(v) & 0x7fffffffu));
                if (c < a.kept.pitch) a.kept.codes[t * a.kept.pitch + c] = s == 255 ? 0 : static_cast<int8_t>(code_bits(v, scale_inverse(s)) & 0xffu);
                if (c % 32 == 0) a.kept.scales[scale_at(a.kept, t, c / 32)] = static_cast<uint8_t>(s);
            }
        }
    }
}

// The backward pass: with n = total * rstd,
//     dx = d_total + rstd (gain dy - n mean(gain dy n)),   dgain = sum over rows of dy n.
// Each block adds its rows' dy n to a row of `partial`.
template <typename G, typename W>
__global__ void __launch_bounds__(kNormThreads) star_rms_norm_backward_loose_kernel(const __grid_constant__ NormGradArgs a)
{
    __shared__ float part[2][kNormThreads / 32];
    launch_dependents();
    wait_for_primary();
    int parity = 0;
    float *sums = a.partial ? a.partial + static_cast<int64_t>(blockIdx.x) * a.cols : nullptr;
    for (int64_t t = blockIdx.x; t < a.rows; t += gridDim.x, parity ^= 1) {
        const char *dy = static_cast<const char *>(a.dy) + t * a.ld_dy * G::kBytes;
        const char *total = static_cast<const char *>(a.total) + t * a.ld_total * G::kBytes;
        const char *d_total = static_cast<const char *>(a.d_total) + t * a.ld_d_total * G::kBytes;
        const float r = a.rstd[t];
        const auto normal = [&](int c) {
            const float s = a.total ? load_value<G>(total, c)
                                    : __fmul_rn(static_cast<float>(a.kept.codes[t * a.kept.pitch + c]), scale_value(a.kept.scales[scale_at(a.kept, t, c / 32)]));
            return __fmul_rn(s, r);
        };
        const auto scaled = [&](int c, float d) { return a.gain ? __fmul_rn(d, load_value<W>(a.gain, c)) : d; };
        float inner = 0.0f;
        for (int c = threadIdx.x; c < a.cols; c += kNormThreads) inner = __fmaf_rn(scaled(c, load_value<G>(dy, c)), normal(c), inner);
        const float mean = __fmul_rn(block_total<kNormThreads>(inner, part[parity]), a.inv_cols);
        char *dx = static_cast<char *>(a.dx) + t * a.ld_dx * G::kBytes;
        for (int c = threadIdx.x; c < a.cols; c += kNormThreads) {
            const float d = load_value<G>(dy, c), n = normal(c);
            float v = __fmul_rn(r, __fmaf_rn(-n, mean, scaled(c, d)));
            if (a.d_total) v = __fadd_rn(v, load_value<G>(d_total, c));
            store_value<G>(dx, c, v);
            if (sums) sums[c] = t == blockIdx.x ? __fmul_rn(d, n) : __fmaf_rn(d, n, sums[c]);
        }
    }
}

// dgain from the blocks' sums: 32 columns to a block, 32 warps that share the rows.
constexpr int kGainThreads = 1024;

template <typename W>
__global__ void __launch_bounds__(kGainThreads) star_rms_norm_gain_kernel(const float *partial, int64_t parts, int cols, void *dgain, int accumulate)
{
    __shared__ float part[32][33];
    wait_for_primary();
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    for (int base = blockIdx.x * 32; base < cols; base += gridDim.x * 32) {
        const int c = base + lane;
        float x = 0.0f;
        if (c < cols)
            for (int64_t q = warp; q < parts; q += 32) x = __fadd_rn(x, partial[q * cols + c]);
        part[warp][lane] = x;
        __syncthreads();
        if (warp == 0 && c < cols) {
            double sum = accumulate ? static_cast<double>(load_value<W>(dgain, c)) : 0.0;
            for (int w = 0; w < 32; ++w) sum += part[w][lane];
            store_value<W>(dgain, c, static_cast<float>(sum));
        }
        __syncthreads();
    }
}

}  // namespace star
