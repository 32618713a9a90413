// Device code of the root-mean-square norm (sm_100a).
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "checkpoint.cuh"
#include "rows.cuh"

namespace star {

struct NormArgs {
    const void *x;
    const void *residual;    // may be null
    void *total;             // may be null
    void *y;
    const void *gain;        // may be null
    int gain_wide;           // binary32, else bf16
    float *rstd;             // may be null
    Kept kept;               // codes may be null
    int64_t ld_x, ld_residual, ld_total, ld_y;
    int64_t rows;
    int cols;
    float eps;
    double inv_cols;
    int wide;                // every row of every matrix is 32-byte aligned
};

struct NormGradArgs {
    void *dx;
    const void *dy;
    const void *total;       // or null, and then kept
    Kept kept;
    const void *gain;        // may be null
    int gain_wide;
    const float *rstd;
    const void *d_total;     // may be null
    int64_t ld_dx, ld_dy, ld_total, ld_d_total;
    int64_t rows;
    int cols;
    double inv_cols;
    int wide;
    float *partial;          // a row of cols sums for each block; null: the gain has no gradient
};

// 1 / sqrt(mean of squares + eps) as the sum of two binary32 numbers, so that a result
// made with it has little more than its own rounding; NaN where the squares' sum is
// none of binary32.
struct NormFactor {
    float high, low;
};
__device__ __forceinline__ NormFactor norm_factor(double squares, double inv_cols, float eps)
{
    if (!(static_cast<float>(squares) < INFINITY)) return NormFactor{NAN, 0.0f};
    const double r = rsqrt(fma(squares, inv_cols, static_cast<double>(eps)));
    const float high = static_cast<float>(r);
    return NormFactor{high, static_cast<float>(r - static_cast<double>(high))};
}
__device__ __forceinline__ float scaled(float x, NormFactor r) { return __fmaf_rn(x, r.high, __fmul_rn(x, r.low)); }
__device__ __forceinline__ float gain_at(const void *gain, int wide, int64_t c)
{
    return gain == nullptr ? 1.0f : wide ? load_value<GradF32>(gain, c) : load_value<GradBF16>(gain, c);
}

__device__ __forceinline__ float rounded_to(float x, const GradF32 *) { return x; }
__device__ __forceinline__ float rounded_to(float x, const GradBF16 *) { return __uint_as_float(pack_bf16(x, 0.0f) << 16); }
// x as a buffer of type G holds it.
template <typename G> __device__ __forceinline__ float as_stored(float x) { return rounded_to(x, static_cast<const G *>(nullptr)); }

// The THREADS that share a row, one of several such groups in a block (or the block).
template <int THREADS, int BLOCK> __device__ __forceinline__ void group_sync()
{
    if constexpr (THREADS == 32)
        __syncwarp();
    else if constexpr (THREADS == BLOCK)
        __syncthreads();
    else
        asm volatile("bar.sync %0, %1;" :: "r"(static_cast<int>(threadIdx.x) / THREADS + 1), "n"(THREADS) : "memory");
}

// The sum over a group's threads, in every thread, in a fixed order.  `part` holds a
// number for each warp of the block and is free again after the group's next sum
// but one.
template <int THREADS, int BLOCK, typename T> __device__ __forceinline__ T group_total(T x, T *part)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    if constexpr (THREADS > 32) {
        constexpr int kWarps = THREADS / 32;
        if (threadIdx.x % 32 == 0) part[threadIdx.x / 32] = x;
        group_sync<THREADS, BLOCK>();
        x = part[threadIdx.x / THREADS * kWarps + threadIdx.x % kWarps];
#pragma unroll
        for (int o = kWarps / 2; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    }
    return x;
}

// ---------------------------------------------------------------------------
// Rows longer than a block's registers hold: a block to a row, a warp on blocks of 32
// columns, a lane to a column; the row is read again for its results.  A thread
// counts its steps: a column beyond the last of up to 2^31 - 65 has no number.
//
// Bound by the latency of single elements: 4096 x 20000 bf16 with residual and 8 bits 451 us,
// backward 596; 2048 x 32768 fp32 521 and 568 (3 to 6 times what their bytes take).
// ---------------------------------------------------------------------------
constexpr int kNormThreads = 256;
__device__ __forceinline__ int long_column(int step) { return step * kNormThreads + static_cast<int>(threadIdx.x); }
__device__ __forceinline__ int long_steps(int cols) { return (cols - static_cast<int>(threadIdx.x) - 1) / kNormThreads + 1; }    // cols >= threads

// The sum of f(c) over a thread's columns: runs of 16 in binary32, added up in binary64.  In
// binary32 alone a million columns of one value, 4096 to a thread, are off by 3e-5.
template <typename F> __device__ __forceinline__ double sum_of_runs(int steps, F f)
{
    double sum = 0.0;
    for (int i = 0; i < steps;) {
        float run = 0.0f;
#pragma unroll 4
        for (const int end = min(steps, i + 16); i < end; ++i) run = f(long_column(i), run);
        sum += static_cast<double>(run);
    }
    return sum;
}

template <typename G>
__global__ void __launch_bounds__(kNormThreads) star_rms_norm_long_kernel(const __grid_constant__ NormArgs a)
{
    __shared__ double part[2][kNormThreads / 32];
    wait_for_primary();
    int parity = 0;
    const int steps = long_steps(a.cols), padded_steps = long_steps((a.cols + 31) / 32 * 32);
    for (int64_t t = blockIdx.x; t < a.rows; t += gridDim.x, parity ^= 1) {
        const char *x = static_cast<const char *>(a.x) + t * a.ld_x * G::kBytes;
        const char *residual = static_cast<const char *>(a.residual) + t * a.ld_residual * G::kBytes;
        char *total = static_cast<char *>(a.total) + t * a.ld_total * G::kBytes;
        const auto stream = [&](int c) {
            const float v = load_value<G>(x, c);
            return a.residual ? as_stored<G>(__fadd_rn(v, load_value<G>(residual, c))) : v;
        };
        const double squares = sum_of_runs(steps, [&](int c, float run) {
            const float s = stream(c);
            if (a.total) store_value<G>(total, c, s);
            return __fmaf_rn(s, s, run);
        });
        const NormFactor r = norm_factor(group_total<kNormThreads, kNormThreads>(squares, part[parity]), a.inv_cols, a.eps);
        if (threadIdx.x == 0 && a.rstd) a.rstd[t] = r.high;
        char *y = static_cast<char *>(a.y) + t * a.ld_y * G::kBytes;
        // What was written to `total` is read back by the thread that wrote it.
        for (int i = 0; i < padded_steps; ++i) {
            const int c = long_column(i);
            float v = 0.0f;
            if (c < a.cols) {
                v = a.total ? load_value<G>(total, c) : stream(c);
                v = as_stored<G>(scaled(__fmul_rn(v, gain_at(a.gain, a.gain_wide, c)), r));
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
template <typename G>
__global__ void __launch_bounds__(kNormThreads) star_rms_norm_backward_long_kernel(const __grid_constant__ NormGradArgs a)
{
    __shared__ double part[2][kNormThreads / 32];
    launch_dependents();
    wait_for_primary();
    int parity = 0;
    float *sums = a.partial ? a.partial + static_cast<int64_t>(blockIdx.x) * a.cols : nullptr;
    const int steps = long_steps(a.cols);
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
        const auto weighted = [&](int c, float d) { return __fmul_rn(d, gain_at(a.gain, a.gain_wide, c)); };
        const double inner = sum_of_runs(steps, [&](int c, float run) { return __fmaf_rn(weighted(c, load_value<G>(dy, c)), normal(c), run); });
        const float mean = static_cast<float>(group_total<kNormThreads, kNormThreads>(inner, part[parity]) * a.inv_cols);
        char *dx = static_cast<char *>(a.dx) + t * a.ld_dx * G::kBytes;
        for (int i = 0; i < steps; ++i) {
            const int c = long_column(i);
            const float d = load_value<G>(dy, c), n = normal(c);
            float v = __fmul_rn(r, __fmaf_rn(-n, mean, weighted(c, d)));
            if (a.d_total) v = __fadd_rn(v, load_value<G>(d_total, c));
            store_value<G>(dx, c, v);
            if (sums) sums[c] = t == blockIdx.x ? __fmul_rn(d, n) : __fmaf_rn(d, n, sums[c]);
        }
    }
}

// ---------------------------------------------------------------------------
// Rows whose values start on 16-byte boundaries: the row stays in registers, 16
// columns (half a block of 32, whose other half the neighbouring lane has) to a
// thread, EACH times.  THREADS share a row, several rows are in a block's hands at once
// where they are short.  One barrier to a row.
//
// Bound by memory: 16384 x 4096 bf16 with residual and 8 bits (9.03 bytes an element) in
// 93.6 us, 6.5 TB/s; element by element with a second reading 380.
// ---------------------------------------------------------------------------
__host__ __device__ constexpr int norm_block(int threads) { return threads < 256 ? 256 : threads; }

// 16 values of the gain from column c on, 1 where there is none.
__device__ __forceinline__ void load_gain(const void *gain, int wide, int64_t c, int64_t cols, int aligned, float (&g)[16])
{
    if (gain == nullptr) {
#pragma unroll
        for (int e = 0; e < 16; ++e) g[e] = 1.0f;
    } else if (!aligned) {
#pragma unroll
        for (int e = 0; e < 16; ++e) g[e] = c + e < cols ? gain_at(gain, wide, c + e) : 0.0f;
    } else if (wide) {
        uint32_t w[Sixteen<GradF32>::kWords];
        Sixteen<GradF32>::load(gain, c, cols, 0, w);
        Sixteen<GradF32>::widen(w, g);
    } else {
        uint32_t w[Sixteen<GradBF16>::kWords];
        Sixteen<GradBF16>::load(gain, c, cols, 0, w);
        Sixteen<GradBF16>::widen(w, g);
    }
}

template <typename G, int THREADS, int EACH>
__global__ void __launch_bounds__(norm_block(THREADS)) star_rms_norm_kernel(const __grid_constant__ NormArgs a)
{
    using S = Sixteen<G>;
    constexpr int kBlock = norm_block(THREADS), kGroups = kBlock / THREADS;
    __shared__ double part[2][kBlock / 32];
    const int at = threadIdx.x % THREADS;
    const int aligned = reinterpret_cast<uintptr_t>(a.gain) % 16 == 0;
    launch_dependents();
    wait_for_primary();
    int parity = 0;
    for (int64_t t = static_cast<int64_t>(blockIdx.x) * kGroups + threadIdx.x / THREADS; t < a.rows; t += static_cast<int64_t>(gridDim.x) * kGroups, parity ^= 1) {
        uint32_t w[EACH][S::kWords];
        float squares = 0.0f;
#pragma unroll
        for (int q = 0; q < EACH; ++q) {
            const int64_t c = static_cast<int64_t>(q * THREADS + at) * 16;
            if (c < a.cols) S::load(static_cast<const char *>(a.x) + t * a.ld_x * G::kBytes, c, a.cols, a.wide, w[q]);
        }
        if (a.residual) {
            uint32_t r[EACH][S::kWords];
#pragma unroll
            for (int q = 0; q < EACH; ++q) {
                const int64_t c = static_cast<int64_t>(q * THREADS + at) * 16;
                if (c < a.cols) S::load(static_cast<const char *>(a.residual) + t * a.ld_residual * G::kBytes, c, a.cols, a.wide, r[q]);
            }
#pragma unroll
            for (int q = 0; q < EACH; ++q) {
                float f[16], g[16];
                S::widen(w[q], f);
                S::widen(r[q], g);
#pragma unroll
                for (int e = 0; e < 16; ++e) f[e] = __fadd_rn(f[e], g[e]);
                S::narrow(f, w[q]);
            }
        }
#pragma unroll
        for (int q = 0; q < EACH; ++q) {
            const int64_t c = static_cast<int64_t>(q * THREADS + at) * 16;
            if (c < a.cols) {
                if (a.total) S::store(static_cast<char *>(a.total) + t * a.ld_total * G::kBytes, c, a.cols, a.wide, w[q]);
                float f[16];
                S::widen(w[q], f);
#pragma unroll
                for (int e = 0; e < 16; ++e) squares = __fmaf_rn(f[e], f[e], squares);
            }
        }
        const NormFactor r = norm_factor(group_total<THREADS, kBlock>(static_cast<double>(squares), part[parity]), a.inv_cols, a.eps);
        if (at == 0 && a.rstd) a.rstd[t] = r.high;
#pragma unroll
        for (int q = 0; q < EACH; ++q) {
            const int64_t c = static_cast<int64_t>(q * THREADS + at) * 16;
            const bool in = c < a.cols;
            uint32_t largest = 0;
            float f[16];
            if (in) {
                float g[16];
                load_gain(a.gain, a.gain_wide, c, a.cols, aligned, g);
                S::widen(w[q], f);
#pragma unroll
                for (int e = 0; e < 16; ++e) f[e] = scaled(__fmul_rn(f[e], g[e]), r);
                S::narrow(f, w[q]);
                S::store(static_cast<char *>(a.y) + t * a.ld_y * G::kBytes, c, a.cols, a.wide, w[q]);
                largest = S::largest(w[q]);
            }
            if (a.kept.codes) {
                largest = max(largest, __shfl_xor_sync(0xffffffffu, largest, 1));
                if (in) {
                    const int s = scale_byte(largest);
                    S::widen(w[q], f);
                    *reinterpret_cast<uint4 *>(a.kept.codes + t * a.kept.pitch + c) = codes_of(f, s);
                    if (at % 2 == 0) a.kept.scales[scale_at(a.kept, t, c / 32)] = static_cast<uint8_t>(s);
                }
            }
        }
    }
}

// ---------------------------------------------------------------------------
// Rows of any alignment that a block's registers hold: a lane to a column, a warp on
// blocks of 32 neighbouring columns, THREADS to a row and EACH columns to one of them.
// Every access is one element to a lane, so that a row's phase does not matter.
// Bound by instructions (two thirds of the issue slots): 4096 x 4095 bf16 with residual
// and 8 bits 69 us, 4096 x 4096 as whole pieces 25.
// ---------------------------------------------------------------------------
template <typename G, int THREADS, int EACH>
__global__ void __launch_bounds__(norm_block(THREADS)) star_rms_norm_columns_kernel(const __grid_constant__ NormArgs a)
{
    constexpr int kBlock = norm_block(THREADS), kGroups = kBlock / THREADS;
    __shared__ double part[2][kBlock / 32];
    const int at = threadIdx.x % THREADS;
    launch_dependents();
    wait_for_primary();
    int parity = 0;
    for (int64_t t = static_cast<int64_t>(blockIdx.x) * kGroups + threadIdx.x / THREADS; t < a.rows; t += static_cast<int64_t>(gridDim.x) * kGroups, parity ^= 1) {
        const char *x = static_cast<const char *>(a.x) + t * a.ld_x * G::kBytes;
        float v[EACH];
#pragma unroll
        for (int q = 0; q < EACH; ++q) v[q] = q * THREADS + at < a.cols ? load_value<G>(x, q * THREADS + at) : 0.0f;
        if (a.residual) {
            const char *residual = static_cast<const char *>(a.residual) + t * a.ld_residual * G::kBytes;
            float r[EACH];
#pragma unroll
            for (int q = 0; q < EACH; ++q) r[q] = q * THREADS + at < a.cols ? load_value<G>(residual, q * THREADS + at) : 0.0f;
#pragma unroll
            for (int q = 0; q < EACH; ++q) v[q] = as_stored<G>(__fadd_rn(v[q], r[q]));
        }
        float squares = 0.0f;
#pragma unroll
        for (int q = 0; q < EACH; ++q) squares = __fmaf_rn(v[q], v[q], squares);
        if (a.total) {
            char *total = static_cast<char *>(a.total) + t * a.ld_total * G::kBytes;
#pragma unroll
            for (int q = 0; q < EACH; ++q)
                if (q * THREADS + at < a.cols) store_value<G>(total, q * THREADS + at, v[q]);
        }
        const NormFactor r = norm_factor(group_total<THREADS, kBlock>(static_cast<double>(squares), part[parity]), a.inv_cols, a.eps);
        if (at == 0 && a.rstd) a.rstd[t] = r.high;
        float g[EACH];
        if (a.gain == nullptr) {
#pragma unroll
            for (int q = 0; q < EACH; ++q) g[q] = 1.0f;
        } else if (a.gain_wide) {
#pragma unroll
            for (int q = 0; q < EACH; ++q) g[q] = q * THREADS + at < a.cols ? load_value<GradF32>(a.gain, q * THREADS + at) : 0.0f;
        } else {
#pragma unroll
            for (int q = 0; q < EACH; ++q) g[q] = q * THREADS + at < a.cols ? load_value<GradBF16>(a.gain, q * THREADS + at) : 0.0f;
        }
        char *y = static_cast<char *>(a.y) + t * a.ld_y * G::kBytes;
#pragma unroll
        for (int q = 0; q < EACH; ++q) {
            v[q] = as_stored<G>(scaled(__fmul_rn(v[q], g[q]), r));
            if (q * THREADS + at < a.cols) store_value<G>(y, q * THREADS + at, v[q]);
        }
        if (a.kept.codes) {
            int8_t *codes = a.kept.codes + t * a.kept.pitch + at;
            const int pitch = static_cast<int>(a.kept.pitch), first = at / 32 * 32;
#pragma unroll
            for (int q = 0; q < EACH; ++q) {
                if (q * THREADS + first < a.cols) {              // not a warp's 32 columns beyond the row
                    const float w = q * THREADS + at < a.cols ? v[q] : 0.0f;
                    const int s = scale_byte(__reduce_max_sync(0xffffffffu, __float_as_uint(w) & 0x7fffffffu));
                    if (q * THREADS + at < pitch) codes[q * THREADS] = s == 255 ? 0 : static_cast<int8_t>(code_bits(w, scale_inverse(s)) & 0xffu);
                    if (at % 32 == 0) a.kept.scales[scale_at(a.kept, t, (q * THREADS + at) / 32)] = static_cast<uint8_t>(s);
                }
            }
        }
    }
}

template <typename G, bool KEPT, int THREADS, int EACH>
__global__ void __launch_bounds__(norm_block(THREADS)) star_rms_norm_backward_columns_kernel(const __grid_constant__ NormGradArgs a)
{
    constexpr int kBlock = norm_block(THREADS), kGroups = kBlock / THREADS;
    __shared__ float part[2][kBlock / 32];
    __shared__ float group_sums[kGroups > 1 ? (kGroups - 1) * THREADS * EACH : 1];
    const int at = threadIdx.x % THREADS, group = threadIdx.x / THREADS;
    launch_dependents();
    wait_for_primary();
    float sums[EACH], gain[EACH];
#pragma unroll
    for (int q = 0; q < EACH; ++q) {
        sums[q] = 0.0f;
        gain[q] = q * THREADS + at < a.cols ? gain_at(a.gain, a.gain_wide, q * THREADS + at) : 0.0f;
    }
    int parity = 0;
    for (int64_t t = static_cast<int64_t>(blockIdx.x) * kGroups + group; t < a.rows; t += static_cast<int64_t>(gridDim.x) * kGroups, parity ^= 1) {
        const char *dy = static_cast<const char *>(a.dy) + t * a.ld_dy * G::kBytes;
        const char *total = static_cast<const char *>(a.total) + t * a.ld_total * G::kBytes;
        const char *d_total = static_cast<const char *>(a.d_total) + t * a.ld_d_total * G::kBytes;
        const float r = a.rstd[t];
        float d[EACH], n[EACH], x[EACH];
#pragma unroll
        for (int q = 0; q < EACH; ++q) {
            const int c = q * THREADS + at;
            const bool in = c < a.cols;
            d[q] = in ? load_value<G>(dy, c) : 0.0f;
            if constexpr (KEPT)
                n[q] = in ? __fmul_rn(static_cast<float>(a.kept.codes[t * a.kept.pitch + c]), scale_value(a.kept.scales[scale_at(a.kept, t, c / 32)])) : 0.0f;
            else
                n[q] = in ? load_value<G>(total, c) : 0.0f;
            x[q] = in && a.d_total ? load_value<G>(d_total, c) : 0.0f;
        }
        float inner = 0.0f;
#pragma unroll
        for (int q = 0; q < EACH; ++q) {
            n[q] = __fmul_rn(n[q], r);
            sums[q] = __fmaf_rn(d[q], n[q], sums[q]);
            d[q] = __fmul_rn(d[q], gain[q]);
            inner = __fmaf_rn(d[q], n[q], inner);
        }
        const float mean = static_cast<float>(group_total<THREADS, kBlock>(inner, part[parity]) * a.inv_cols), back = -__fmul_rn(r, mean);
        char *dx = static_cast<char *>(a.dx) + t * a.ld_dx * G::kBytes;
#pragma unroll
        for (int q = 0; q < EACH; ++q)
            if (q * THREADS + at < a.cols) store_value<G>(dx, q * THREADS + at, __fmaf_rn(n[q], back, __fmaf_rn(d[q], r, x[q])));
    }
    if (!a.partial) return;
    if constexpr (kGroups > 1) {
        if (group > 0) {
#pragma unroll
            for (int q = 0; q < EACH; ++q) group_sums[((group - 1) * EACH + q) * THREADS + at] = sums[q];
        }
        __syncthreads();
        if (group > 0) return;
        for (int other = 0; other < kGroups - 1; ++other)
#pragma unroll
            for (int q = 0; q < EACH; ++q) sums[q] = __fadd_rn(sums[q], group_sums[(other * EACH + q) * THREADS + at]);
    }
    float *out = a.partial + static_cast<int64_t>(blockIdx.x) * a.cols;
#pragma unroll
    for (int q = 0; q < EACH; ++q)
        if (q * THREADS + at < a.cols) out[q * THREADS + at] = sums[q];
}

// ---------------------------------------------------------------------------
// The backward pass of such rows.  A thread takes EACH granules of 16 bytes of a row
// and keeps their columns' sums for the gain over all its rows, so blocks stay and go
// round the rows.  What it needs of its next STAGES rows is on its way into its own
// slots of shared memory meanwhile (asynchronous copies, which nobody else reads: no
// barrier but the one of the row's sum), since registers for rows in flight cost more
// threads than they gain.  16384 x 4096 bf16 with d_total 88 us, 6.1 TB/s (loads when a
// row's turn comes 104, the next row in registers 134; all blocks that fit 64 registers a
// thread, four to an SM, 116).
// ---------------------------------------------------------------------------
// SIZE bytes, of which `bytes` are there; the rest reads as 0.
template <int SIZE> __device__ __forceinline__ void copy_async(void *to, const void *from, int bytes)
{
    if constexpr (SIZE == 16)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" :: "r"(smem_address(to)), "l"(from), "r"(bytes) : "memory");
    else
        asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" :: "r"(smem_address(to)), "l"(from), "n"(SIZE), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" :: "n"(LEFT) : "memory"); }

// E codes as numbers: they become the low bytes of numbers near 2^23 first.
template <int E> __device__ __forceinline__ void widen_codes(const uint32_t *codes, Pair (&f)[E / 2])
{
    const Pair off = pair_of(-8388736.0f);
#pragma unroll
    for (int w = 0; w < E / 4; ++w) {
        const uint32_t u = codes[w] ^ 0x80808080u;
        f[2 * w] = pair_add(make_pair(__uint_as_float(__byte_perm(u, 0x4b000000u, 0x7650)), __uint_as_float(__byte_perm(u, 0x4b000000u, 0x7651))), off);
        f[2 * w + 1] = pair_add(make_pair(__uint_as_float(__byte_perm(u, 0x4b000000u, 0x7652)), __uint_as_float(__byte_perm(u, 0x4b000000u, 0x7653))), off);
    }
}

template <typename G, bool KEPT, int EACH, int STAGES> struct NormRing {
    static constexpr int E = 16 / G::kBytes, P = E / 2, kCodeWords = E / 4;
    // Bytes of one thread's slots.
    static constexpr int kThread = STAGES * (EACH * (16 + 16 + (KEPT ? E + 4 : 16)) + 4);
};

template <typename G, bool KEPT, int THREADS, int EACH, int STAGES>
__global__ void __launch_bounds__(norm_block(THREADS), 768 / norm_block(THREADS) < 1 ? 1 : 768 / norm_block(THREADS))
star_rms_norm_backward_kernel(const __grid_constant__ NormGradArgs a)
{
    using Ring = NormRing<G, KEPT, EACH, STAGES>;
    constexpr int E = Ring::E, P = Ring::P, kBlock = norm_block(THREADS), kGroups = kBlock / THREADS;
    // The sum's type decides how the blocks' phases fall: 16384 x 4096 bf16 88.2 us with binary64 and 94.6 with binary32,
    // from the stream in 8 bits 97.0 and 93.7.
    using Sum = std::conditional_t<KEPT, float, double>;
    __shared__ Sum part[2][kBlock / 32];
    extern __shared__ uint4 slots[];
    uint4 *const own = slots + threadIdx.x;                      // dy, d_total and the stream: one column of slots each
    constexpr int kDTotal = STAGES * EACH, kStream = 2 * STAGES * EACH;
    // Neighbouring lanes share 16 bytes of codes, and the four scales of 128 columns; the first of them copies.
    constexpr int kCodeLanes = 16 / E, kScaleLanes = 128 / E;
    uint32_t *const words = reinterpret_cast<uint32_t *>(slots + (KEPT ? 2 : 3) * STAGES * EACH * kBlock);
    uint32_t *const own_codes = words + threadIdx.x * Ring::kCodeWords;                  // KEPT: [slot][thread][word]
    uint32_t *const own_scales = words + (KEPT ? STAGES * EACH * kBlock * Ring::kCodeWords : 0) + threadIdx.x / kScaleLanes;
    float *const own_rstd = reinterpret_cast<float *>(words + (KEPT ? STAGES * EACH * kBlock * (Ring::kCodeWords + 1) : 0)) + threadIdx.x;
    const int at = threadIdx.x % THREADS, group = threadIdx.x / THREADS;
    launch_dependents();
    wait_for_primary();
    Pair sums[EACH][P], gain[EACH][P];
#pragma unroll
    for (int q = 0; q < EACH; ++q)
#pragma unroll
        for (int e = 0; e < P; ++e) {
            const int c = (q * THREADS + at) * E + 2 * e;
            sums[q][e] = pair_of(0.0f);
            gain[q][e] = make_pair(c < a.cols ? gain_at(a.gain, a.gain_wide, c) : 0.0f, c + 1 < a.cols ? gain_at(a.gain, a.gain_wide, c + 1) : 0.0f);
        }
    const int64_t step = static_cast<int64_t>(gridDim.x) * kGroups;
    const auto fetch = [&](int64_t t, int stage) {
        if (t < a.rows) {
#pragma unroll
            for (int q = 0; q < EACH; ++q) {
                const int64_t c = static_cast<int64_t>(q * THREADS + at) * E;
                const int slot = stage * EACH + q;
                if (c < a.cols) {
                    const int bytes = static_cast<int>(min(a.cols - c, int64_t{E})) * G::kBytes;
                    copy_async<16>(own + slot * kBlock, static_cast<const char *>(a.dy) + (t * a.ld_dy + c) * G::kBytes, bytes);
                    if (a.d_total) copy_async<16>(own + (kDTotal + slot) * kBlock, static_cast<const char *>(a.d_total) + (t * a.ld_d_total + c) * G::kBytes, bytes);
                    if constexpr (KEPT) {
                        if (at % kCodeLanes == 0) copy_async<16>(own_codes + slot * kBlock * Ring::kCodeWords, a.kept.codes + t * a.kept.pitch + c, 16);
                        if (at % kScaleLanes == 0) copy_async<4>(own_scales + slot * kBlock, a.kept.scales + scale_at(a.kept, t, c / 128 * 4), 4);
                    } else {
                        copy_async<16>(own + (kStream + slot) * kBlock, static_cast<const char *>(a.total) + (t * a.ld_total + c) * G::kBytes, bytes);
                    }
                }
            }
            copy_async<4>(own_rstd + stage * kBlock, a.rstd + t, 4);
        }
        copies_commit();
    };
    const auto normal = [&](int slot, int64_t c, float r, Pair (&n)[P]) {
        if constexpr (KEPT) {
            uint32_t codes[Ring::kCodeWords];
#pragma unroll
            for (int w = 0; w < Ring::kCodeWords; ++w) codes[w] = own_codes[slot * kBlock * Ring::kCodeWords + w];
            widen_codes<E>(codes, n);
            r = __fmul_rn(scale_value(own_scales[slot * kBlock] >> (c / 32 % 4 * 8) & 0xffu), r);        // a power of two: exact
        } else {
            Granule<G>::widen(own[(kStream + slot) * kBlock], n);
        }
#pragma unroll
        for (int e = 0; e < P; ++e) n[e] = pair_mul(n[e], pair_of(r));
    };
    int64_t t = static_cast<int64_t>(blockIdx.x) * kGroups + group;
#pragma unroll
    for (int q = 0; q < STAGES; ++q) fetch(t + q * step, q);
    int parity = 0, stage = 0;
    for (; t < a.rows; t += step, parity ^= 1) {
        copies_wait<STAGES - 1>();
        if constexpr (KEPT) __syncwarp();                        // the neighbours' copies
        const float r = own_rstd[stage * kBlock];
        Pair inner = pair_of(0.0f);
#pragma unroll
        for (int q = 0; q < EACH; ++q) {
            const int64_t c = static_cast<int64_t>(q * THREADS + at) * E;
            if (c < a.cols) {
                Pair d[P], n[P];
                Granule<G>::widen(own[(stage * EACH + q) * kBlock], d);
                normal(stage * EACH + q, c, r, n);
#pragma unroll
                for (int e = 0; e < P; ++e) {
                    inner = pair_fma(pair_mul(d[e], gain[q][e]), n[e], inner);
                    sums[q][e] = pair_fma(d[e], n[e], sums[q][e]);
                }
            }
        }
        float lo, hi;
        split_pair(inner, &lo, &hi);
        const float mean = static_cast<float>(group_total<THREADS, kBlock>(static_cast<Sum>(__fadd_rn(lo, hi)), part[parity]) * a.inv_cols);
        const Pair rr = pair_of(r), back = pair_of(-__fmul_rn(r, mean));
#pragma unroll
        for (int q = 0; q < EACH; ++q) {
            const int64_t c = static_cast<int64_t>(q * THREADS + at) * E;
            if (c < a.cols) {
                Pair d[P], n[P], x[P];
                Granule<G>::widen(own[(stage * EACH + q) * kBlock], d);
                normal(stage * EACH + q, c, r, n);
#pragma unroll
                for (int e = 0; e < P; ++e) x[e] = pair_of(0.0f);
                if (a.d_total) Granule<G>::widen(own[(kDTotal + stage * EACH + q) * kBlock], x);
#pragma unroll
                for (int e = 0; e < P; ++e) x[e] = pair_fma(n[e], back, pair_fma(pair_mul(d[e], gain[q][e]), rr, x[e]));
                char *out = static_cast<char *>(a.dx) + (t * a.ld_dx + c) * G::kBytes;
                if (c + E <= a.cols) {
                    *reinterpret_cast<uint4 *>(out) = Granule<G>::narrow(x);
                } else {
#pragma unroll
                    for (int e = 0; e < P; ++e) {
                        split_pair(x[e], &lo, &hi);
                        if (c + 2 * e < a.cols) store_value<G>(out, 2 * e, lo);
                        if (c + 2 * e + 1 < a.cols) store_value<G>(out, 2 * e + 1, hi);
                    }
                }
            }
        }
        if constexpr (KEPT) __syncwarp();
        fetch(t + STAGES * step, stage);                         // into the slots just read
        stage = stage + 1 == STAGES ? 0 : stage + 1;
    }
    if (!a.partial) return;
    // The groups' sums join, and the block's go out.
    if constexpr (kGroups > 1) {
        constexpr int kSums = THREADS * EACH * P;
        static_assert((kGroups - 1) * kSums * 8 <= kBlock * STAGES * EACH * 32, "the slots hold the sums");
        Pair *group_sums = reinterpret_cast<Pair *>(slots);
        copies_wait<0>();
        __syncthreads();                                         // nobody's slots are in use
        if (group > 0) {
#pragma unroll
            for (int q = 0; q < EACH; ++q)
#pragma unroll
                for (int e = 0; e < P; ++e) group_sums[(group - 1) * kSums + (q * P + e) * THREADS + at] = sums[q][e];
        }
        __syncthreads();
        if (group > 0) return;
        for (int other = 0; other < kGroups - 1; ++other)
#pragma unroll
            for (int q = 0; q < EACH; ++q)
#pragma unroll
                for (int e = 0; e < P; ++e) sums[q][e] = pair_add(sums[q][e], group_sums[other * kSums + (q * P + e) * THREADS + at]);
    }
    float *out = a.partial + static_cast<int64_t>(blockIdx.x) * a.cols;
#pragma unroll
    for (int q = 0; q < EACH; ++q) {
        const int c = (q * THREADS + at) * E;
#pragma unroll
        for (int e = 0; e < P; ++e) {
            float lo, hi;
            split_pair(sums[q][e], &lo, &hi);
            if (c + 2 * e < a.cols) out[c + 2 * e] = lo;
            if (c + 2 * e + 1 < a.cols) out[c + 2 * e + 1] = hi;
        }
    }
}

// dgain from the blocks' sums: 32 columns to a block, up to 32 warps that share the rows.
constexpr int kGainThreads = 1024;

template <typename W>
__global__ void __launch_bounds__(kGainThreads) star_rms_norm_gain_kernel(const float *partial, int64_t parts, int cols, void *dgain, int accumulate)
{
    __shared__ float part[32][33];
    wait_for_primary();
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, warps = blockDim.x / 32;
    for (int64_t base = blockIdx.x * 32; base < cols; base += gridDim.x * 32) {
        const int64_t c = base + lane;
        float x = 0.0f;
        if (c < cols)
            for (int64_t q = warp; q < parts; q += warps) x = __fadd_rn(x, partial[q * cols + c]);
        part[warp][lane] = x;
        __syncthreads();
        if (warp == 0 && c < cols) {
            double sum = accumulate ? static_cast<double>(load_value<W>(dgain, c)) : 0.0;
            for (int w = 0; w < warps; ++w) sum += part[w][lane];
            store_value<W>(dgain, c, static_cast<float>(sum));
        }
        __syncthreads();
    }
}

}  // namespace star
