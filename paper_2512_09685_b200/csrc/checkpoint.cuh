// Device code of activations kept in 8 bits: the format, and the elementwise
// kernels that write and read it (sm_100a).
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "device.cuh"
#include "star.h"

namespace star {

// Where a checkpoint lies; see star.h for the format.
struct Kept {
    int8_t *codes;
    uint8_t *scales;
    int64_t rows, cols;
    int64_t pitch;       // bytes from row to row of codes
    int64_t tall;        // rows rounded up to 64
};

__device__ __forceinline__ int64_t scale_at(const Kept &k, int64_t t, int64_t block)
{
    return ((block >> 2) * k.tall + t) * 4 + (block & 3);
}

// The scale byte of a block from the bits of its largest magnitude.  With
// largest = f 2^k, 1 <= f < 2, the codes of scale 2^(k-6) reach f * 64; they
// round to at most 127 iff f < 127.5 / 64, i.e. unless the seven upper mantissa
// bits are all ones -- adding one at the seventh carries into the exponent
// exactly then.  255 marks a block without finite values.
constexpr int kScaleMost = 104 + 127;
__device__ __forceinline__ int scale_byte(uint32_t largest_bits)
{
    const int b = static_cast<int>((largest_bits + 0x00010000u) >> 23) - 6;
    return b > kScaleMost ? 255 : max(b, 1);
}

// 2^e and 2^-e of a scale byte (255: infinity, so that a code of 0 is NaN; 0).
__device__ __forceinline__ float scale_value(int b) { return __int_as_float(b << 23); }
__device__ __forceinline__ float scale_inverse(int b) { return b == 255 ? 0.0f : __int_as_float((254 - b) << 23); }

// round(x 2^-e) in the low byte: adding 1.5 * 2^23 rounds to an integer,
// nearest even, and leaves it in the low mantissa bits.
constexpr float kRoundMagic = 12582912.0f;
__device__ __forceinline__ uint32_t code_bits(float x, float inverse)
{
    return __float_as_uint(__fmaf_rn(x, inverse, kRoundMagic));
}

template <int ACT> __device__ __forceinline__ float activation(float x);
template <int ACT> __device__ __forceinline__ float activation_slope(float x);

__device__ __forceinline__ float sigmoid(float x)
{
    return __fdividef(1.0f, __fadd_rn(1.0f, exp2_fast(__fmul_rn(-kLog2e, x))));
}

// 0.5 (1 + tanh(y)) = sigmoid(2 y).
constexpr float kGeluB = 0.79788456080286536f * 2.0f;           // 2 sqrt(2 / pi)
constexpr float kGeluC = kGeluB * 0.044715f;
constexpr float kSqrtHalf = 0.70710678118654752f;
constexpr float kInvSqrt2Pi = 0.39894228040143268f;

template <> __device__ __forceinline__ float activation<STAR_ACT_NONE>(float x) { return x; }
template <> __device__ __forceinline__ float activation_slope<STAR_ACT_NONE>(float) { return 1.0f; }

template <> __device__ __forceinline__ float activation<STAR_ACT_GELU_TANH>(float x)
{
    return __fmul_rn(x, sigmoid(__fmul_rn(x, __fmaf_rn(kGeluC, __fmul_rn(x, x), kGeluB))));
}
template <> __device__ __forceinline__ float activation_slope<STAR_ACT_GELU_TANH>(float x)
{
    const float x2 = __fmul_rn(x, x);
    const float q = sigmoid(__fmul_rn(x, __fmaf_rn(kGeluC, x2, kGeluB)));
    const float inner = __fmul_rn(x, __fmaf_rn(3.0f * kGeluC, x2, kGeluB));      // x times the inner derivative
    const float w = __fmul_rn(q, __fsub_rn(1.0f, q));
    return w == 0.0f ? q : __fmaf_rn(w, inner, q);       // inner overflows where w is long 0
}

template <> __device__ __forceinline__ float activation<STAR_ACT_SILU>(float x) { return __fmul_rn(x, sigmoid(x)); }
template <> __device__ __forceinline__ float activation_slope<STAR_ACT_SILU>(float x)
{
    const float q = sigmoid(x);
    return __fmaf_rn(__fmul_rn(q, __fsub_rn(1.0f, q)), x, q);
}

template <> __device__ __forceinline__ float activation<STAR_ACT_GELU_ERF>(float x)
{
    return __fmul_rn(__fmul_rn(0.5f, x), __fadd_rn(1.0f, erff(__fmul_rn(x, kSqrtHalf))));
}
template <> __device__ __forceinline__ float activation_slope<STAR_ACT_GELU_ERF>(float x)
{
    const float cdf = __fmaf_rn(0.5f, erff(__fmul_rn(x, kSqrtHalf)), 0.5f);
    const float pdf = __fmul_rn(kInvSqrt2Pi, exp2_fast(__fmul_rn(-0.5f * kLog2e, __fmul_rn(x, x))));
    return __fmaf_rn(x, pdf, cdf);
}

struct PackArgs {
    Kept kept;
    const void *x;
    int64_t ld;
    void *act_out;       // may be null
    int64_t ld_act;
};

constexpr int kPackThreads = 256;

// One warp per block of 32 columns, one lane per element.
template <typename G, int ACT> __global__ void __launch_bounds__(kPackThreads) star_checkpoint_pack_kernel(const __grid_constant__ PackArgs a)
{
    const int lane = threadIdx.x % 32;
    const int64_t blocks = (a.kept.cols + 31) / 32, n = a.kept.rows * blocks;
    for (int64_t i = blockIdx.x * static_cast<int64_t>(kPackThreads / 32) + threadIdx.x / 32; i < n;
         i += gridDim.x * static_cast<int64_t>(kPackThreads / 32)) {
        const int64_t t = i / blocks, b = i % blocks, c = b * 32 + lane;
        const bool in = c < a.kept.cols;
        const float x = in ? load_value<G>(a.x, t * a.ld + c) : 0.0f;
        const uint32_t largest = __reduce_max_sync(0xffffffffu, __float_as_uint(x) & 0x7fffffffu);
        const int s = scale_byte(largest);
        if (c < a.kept.pitch)
            a.kept.codes[t * a.kept.pitch + c] = s == 255 ? 0 : static_cast<int8_t>(code_bits(x, scale_inverse(s)) & 0xffu);
        if (lane == 0) a.kept.scales[scale_at(a.kept, t, b)] = static_cast<uint8_t>(s);
        if (a.act_out && in) store_value<G>(a.act_out, t * a.ld_act + c, activation<ACT>(x));
    }
}

__device__ __forceinline__ float kept_value(const Kept &k, int64_t t, int64_t c)
{
    return __fmul_rn(static_cast<float>(k.codes[t * k.pitch + c]), scale_value(k.scales[scale_at(k, t, c / 32)]));
}

struct UnpackArgs {
    Kept kept;
    void *out;
    int64_t ld;
    const void *dy;      // BACKWARD only
    int64_t ld_dy;
};

// out = act(value), or dy * act'(value).
template <typename G, int ACT, bool BACKWARD>
__global__ void __launch_bounds__(kPackThreads) star_checkpoint_read_kernel(const __grid_constant__ UnpackArgs a)
{
    const int64_t n = a.kept.rows * a.kept.cols;
    for (int64_t i = blockIdx.x * static_cast<int64_t>(kPackThreads) + threadIdx.x; i < n;
         i += gridDim.x * static_cast<int64_t>(kPackThreads)) {
        const int64_t t = i / a.kept.cols, c = i % a.kept.cols;
        const float x = kept_value(a.kept, t, c);
        float y;
        if constexpr (BACKWARD)
            y = __fmul_rn(load_value<G>(a.dy, t * a.ld_dy + c), activation_slope<ACT>(x));
        else
            y = activation<ACT>(x);
        store_value<G>(a.out, t * a.ld + c, y);
    }
}

struct WeightGradArgs {
    Kept kept;
    const void *dy;
    int64_t ld_dy;
    void *dw;
    int64_t stride_o, stride_c;      // elements of dw between neighbouring outputs and columns
    int64_t outs;
    int accumulate;
};

// 32 x 32 outputs per block, 32 rows at a time.
template <typename GY, typename GW> __global__ void __launch_bounds__(256) star_weight_grad_kernel(const __grid_constant__ WeightGradArgs a)
{
    __shared__ float xs[32][33], ys[32][33];
    const int64_t c0 = static_cast<int64_t>(blockIdx.x) * 32, tiles = (a.outs + 31) / 32;
    const int lane = threadIdx.x % 32, w = threadIdx.x / 32;
    for (int64_t tile = blockIdx.y; tile < tiles; tile += gridDim.y) {
        const int64_t o0 = tile * 32;
        float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int64_t t0 = 0; t0 < a.kept.rows; t0 += 32) {
            for (int r = w; r < 32; r += 8) {
                const int64_t t = t0 + r;
                xs[r][lane] = t < a.kept.rows && c0 + lane < a.kept.cols ? kept_value(a.kept, t, c0 + lane) : 0.0f;
                ys[r][lane] = t < a.kept.rows && o0 + lane < a.outs ? load_value<GY>(a.dy, t * a.ld_dy + o0 + lane) : 0.0f;
            }
            __syncthreads();
            for (int r = 0; r < 32; ++r)
#pragma unroll
                for (int q = 0; q < 4; ++q) sum[q] = __fmaf_rn(ys[r][w + 8 * q], xs[r][lane], sum[q]);
            __syncthreads();
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int64_t o = o0 + w + 8 * q, c = c0 + lane;
            if (o < a.outs && c < a.kept.cols) {
                const int64_t at = o * a.stride_o + c * a.stride_c;
                if (a.accumulate) sum[q] = __fadd_rn(sum[q], load_value<GW>(a.dw, at));
                store_value<GW>(a.dw, at, sum[q]);
            }
        }
    }
}

}  // namespace star
