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

// ---------------------------------------------------------------------------
// Activations and their slopes, two values at a time: an exponential (2 ulp) and a
// reciprocal (1 ulp) each, the rest in packed binary32.  SiLU in fp32 4.2e-8 in norm
// against 3.7e-8 with binary32's own exp and division.
// ---------------------------------------------------------------------------
constexpr float kGeluB = 0.79788456080286536f * 2.0f;           // 2 sqrt(2 / pi)
constexpr float kGeluC = kGeluB * 0.044715f;
constexpr float kInvSqrt2Pi = 0.39894228040143268f;

// 1 / (1 + 2^y): the sigmoid of x for y = -log2(e) x.
__device__ __forceinline__ Pair sigmoid_exp2(Pair y) { return pair_reciprocal(pair_add(pair_exp2(y), pair_of(1.0f))); }

// x^2, at most 1e4: beyond |x| = 100 every sigmoid here is 0 or 1, and what
// multiplies its slope of 0 must stay finite.
__device__ __forceinline__ Pair bounded_square(Pair x)
{
    float lo, hi;
    split_pair(pair_mul(x, x), &lo, &hi);
    return make_pair(fminf(lo, 1e4f), fminf(hi, 1e4f));
}
__device__ __forceinline__ Pair pair_negate(Pair x) { return x ^ 0x8000000080000000ull; }

// q + q (1 - q) inner: the slope of x sigmoid(g(x)), with inner = x g'(x).
__device__ __forceinline__ Pair gated_slope(Pair q, Pair inner)
{
    return pair_fma(pair_mul(q, pair_add(pair_of(1.0f), pair_negate(q))), inner, q);
}

template <int N> __device__ __forceinline__ Pair polynomial(const float (&c)[N], Pair x)
{
    Pair y = pair_of(c[N - 1]);
#pragma unroll
    for (int i = N - 2; i >= 0; --i) y = pair_fma(x, y, pair_of(c[i]));
    return y;
}

// Phi(x), with a bound on its error relative to itself: x Phi(x) and its slope live in
// the tail too.  The tail is Phi(-|x|) = t P(t) exp(-x^2 / 2) with t = 1 / (1 + p |x|)
// and P of degree 6, a minimax fit of the relative error for |x| <= 14.
//   not FINE, for bf16 results: one P for all x, off by 9e-7, a 2000th of their rounding.
//   FINE, for fp32: P for |x| >= 1, off by 9e-8, and below 1/2 + x S(x^2) with S of degree
//   5, fitted to (Phi(x) - 1/2) / x, 3e-8.  In norm, on Gaussian values, 3.6e-8 for x Phi(x)
//   and 4.9e-8 for the slope, as of binary32's erf and exp.
// Both for both, us, with GELU forward / backward: 16384 x 4096 bf16 60 / 56 not FINE, 73 / 70
// FINE (issue-bound); 8192 x 4096 fp32 46 / 45 FINE, bound by memory either way.
// *power = exp(-x^2 / 2), which the slope needs too.
template <bool FINE> __device__ __forceinline__ Pair normal_cdf(Pair x, Pair *power)
{
    constexpr float kNear[6] = {0.3989422917366028f, -0.06649035960435867f, 0.009973322972655296f, -0.0011863299878314137f,
                                0.00011348637053743005f, -7.65420827519847e-06f};
    constexpr float kTail[7] = {0.159595787525177f, 0.1590999811887741f, 0.13900233805179596f, 0.055540427565574646f,
                                0.10536342114210129f, -0.1864282488822937f, 0.06812146306037903f};
    constexpr float kWhole[7] = {0.1437130570411682f, 0.14177247881889343f, 0.13971911370754242f, 0.026549765840172768f,
                                 0.18095333874225616f, -0.17976419627666473f, 0.04705614596605301f};
    const Pair size = x & 0x7fffffff7fffffffull, x2 = pair_mul(x, x);
    const Pair t = pair_reciprocal(pair_fma(pair_of(FINE ? 0.4f : 0.36f), size, pair_of(1.0f)));
    *power = pair_exp2(pair_mul(pair_of(-0.5f * kLog2e), x2));
    const Pair tail = pair_mul(pair_mul(t, polynomial(FINE ? kTail : kWhole, t)), *power);
    float x0, x1, q0, q1, n0 = 0.0f, n1 = 0.0f;
    split_pair(x, &x0, &x1);
    split_pair(tail, &q0, &q1);
    q0 = x0 > 0.0f ? __fsub_rn(1.0f, q0) : q0;
    q1 = x1 > 0.0f ? __fsub_rn(1.0f, q1) : q1;
    if constexpr (FINE) {
        split_pair(pair_fma(x, polynomial(kNear, x2), pair_of(0.5f)), &n0, &n1);
        q0 = fabsf(x0) < 1.0f ? n0 : q0;
        q1 = fabsf(x1) < 1.0f ? n1 : q1;
    }
    return make_pair(q0, q1);
}

template <int ACT, bool FINE> __device__ __forceinline__ Pair activation(Pair x)
{
    if constexpr (ACT == STAR_ACT_GELU_TANH) {           // 0.5 (1 + tanh(y)) = sigmoid(2 y)
        const Pair g = pair_fma(pair_of(-kLog2e * kGeluC), pair_mul(x, x), pair_of(-kLog2e * kGeluB));
        return pair_mul(x, sigmoid_exp2(pair_mul(x, g)));
    } else if constexpr (ACT == STAR_ACT_GELU_ERF) {
        Pair power;
        return pair_mul(x, normal_cdf<FINE>(x, &power));
    } else if constexpr (ACT == STAR_ACT_SILU) {
        return pair_mul(x, sigmoid_exp2(pair_mul(x, pair_of(-kLog2e))));
    } else {
        return x;
    }
}

template <int ACT, bool FINE> __device__ __forceinline__ Pair activation_slope(Pair x)
{
    if constexpr (ACT == STAR_ACT_GELU_TANH) {
        const Pair x2 = bounded_square(x);
        const Pair q = sigmoid_exp2(pair_mul(x, pair_fma(pair_of(-kLog2e * kGeluC), x2, pair_of(-kLog2e * kGeluB))));
        return gated_slope(q, pair_mul(x, pair_fma(pair_of(3.0f * kGeluC), x2, pair_of(kGeluB))));
    } else if constexpr (ACT == STAR_ACT_GELU_ERF) {
        Pair power;
        const Pair cdf = normal_cdf<FINE>(x, &power);
        return pair_fma(x, pair_mul(pair_of(kInvSqrt2Pi), power), cdf);
    } else if constexpr (ACT == STAR_ACT_SILU) {
        return gated_slope(sigmoid_exp2(pair_mul(x, pair_of(-kLog2e))), x);
    } else {
        return pair_of(1.0f);
    }
}

// One value.
template <int ACT, bool FINE> __device__ __forceinline__ float activation(float x)
{
    float lo, hi;
    split_pair(activation<ACT, FINE>(make_pair(x, 0.0f)), &lo, &hi);
    return lo;
}
template <int ACT, bool FINE> __device__ __forceinline__ float activation_slope(float x)
{
    float lo, hi;
    split_pair(activation_slope<ACT, FINE>(make_pair(x, 0.0f)), &lo, &hi);
    return lo;
}

struct PackArgs {
    Kept kept;
    const void *x;
    int64_t ld;
    void *act_out;       // may be null
    int64_t ld_act;
};

struct ReadArgs {
    Kept kept;
    void *out;
    int64_t ld;
    const void *dy;      // BACKWARD only
    int64_t ld_dy;
};

constexpr int kKeepThreads = 256;

// ---------------------------------------------------------------------------
// Rows whose values start on 16-byte boundaries: a thread takes half a block, 16
// columns, and its neighbour the other half; all accesses are 16 or 32 bytes.  The
// work is numbered row by row, an even number of halves to a row, so that two
// neighbouring lanes always share a block.
//
// Bound by memory: 16384 x 4096 bf16, kept with GELU forward (5.03 bytes an
// element), restored (3.03), GELU backward (5.03).  An exponential and a
// reciprocal per element take 70 % of the forward's time on their unit.
// ---------------------------------------------------------------------------

// i / d for i < 2^31 and the divisor the host made `magic` and `shift` from.
struct Divisor {
    uint32_t d, magic;
    int shift;
};
__device__ __forceinline__ uint32_t divide(uint32_t i, const Divisor &d) { return d.d == 1 ? i : __umulhi(i, d.magic) >> d.shift; }

// 32 bytes by one access where the rows allow it (every row 32-byte aligned): a
// whole sector, where two of 16 bytes would touch each sector twice.
__device__ __forceinline__ void load_words(const void *p, uint32_t (&w)[8])
{
    asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]) : "l"(p) : "memory");
}
__device__ __forceinline__ void store_words(void *p, const uint32_t (&w)[8])
{
    asm volatile("st.global.v8.b32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};"
                 :: "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]), "l"(p) : "memory");
}

struct Halves {
    Divisor per_row;     // halves of a row: an even number
    uint32_t first_row;  // rows in front of this launch
    uint32_t n;          // halves of this launch
    int wide;            // rows are 32-byte aligned
};

template <typename G> struct Sixteen {
    static constexpr int kWords = G::kBytes * 4;
    static constexpr int kEach = 16 / G::kBytes;         // values in 16 bytes
    // 16 values of a row from column c on; columns past the end read as 0.
    static __device__ __forceinline__ void load(const void *row, int64_t c, int64_t cols, int wide, uint32_t (&w)[kWords])
    {
        const char *p = static_cast<const char *>(row) + c * G::kBytes;
        const int left = static_cast<int>(min(cols - c, int64_t{16}));
        if (wide && left == 16) {
#pragma unroll
            for (int q = 0; q < kWords / 8; ++q) {
                uint32_t v[8];
                load_words(p + 32 * q, v);
#pragma unroll
                for (int e = 0; e < 8; ++e) w[8 * q + e] = v[e];
            }
            return;
        }
#pragma unroll
        for (int q = 0; q < kWords / 4; ++q) {
            if ((q + 1) * kEach <= left) {
                const uint4 v = reinterpret_cast<const uint4 *>(p)[q];
                w[4 * q] = v.x; w[4 * q + 1] = v.y; w[4 * q + 2] = v.z; w[4 * q + 3] = v.w;
            } else {
                w[4 * q] = w[4 * q + 1] = w[4 * q + 2] = w[4 * q + 3] = 0;
#pragma unroll
                for (int e = q * kEach; e < (q + 1) * kEach; ++e) {
                    if (e < left) {
                        if constexpr (G::kBytes == 2)
                            w[e / 2] |= static_cast<uint32_t>(reinterpret_cast<const unsigned short *>(p)[e]) << (e % 2 * 16);
                        else
                            w[e] = reinterpret_cast<const uint32_t *>(p)[e];
                    }
                }
            }
        }
    }
    static __device__ __forceinline__ void widen(const uint32_t (&w)[kWords], float (&f)[16])
    {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            if constexpr (G::kBytes == 2)
                f[e] = __uint_as_float(e % 2 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16);
            else
                f[e] = __uint_as_float(w[e]);
        }
    }
    // Bits of the largest magnitude as a binary32 (NaN above infinity above the rest).
    static __device__ __forceinline__ uint32_t largest(const uint32_t (&w)[kWords])
    {
        uint32_t m = 0;
        if constexpr (G::kBytes == 2) {
#pragma unroll
            for (int q = 0; q < kWords; ++q) m = __vmaxu2(m, w[q] & 0x7fff7fffu);
            return max(m << 16, m & 0xffff0000u);
        } else {
#pragma unroll
            for (int q = 0; q < kWords; ++q) m = max(m, w[q] & 0x7fffffffu);
            return m;
        }
    }
    static __device__ __forceinline__ void store(void *row, int64_t c, int64_t cols, int wide, const float (&f)[16])
    {
        char *p = static_cast<char *>(row) + c * G::kBytes;
        uint32_t w[kWords];
#pragma unroll
        for (int q = 0; q < kWords; ++q) {
            if constexpr (G::kBytes == 2)
                w[q] = pack_bf16(f[2 * q], f[2 * q + 1]);
            else
                w[q] = __float_as_uint(f[q]);
        }
        const int left = static_cast<int>(min(cols - c, int64_t{16}));
        if (wide && left == 16) {
#pragma unroll
            for (int q = 0; q < kWords / 8; ++q) {
                uint32_t v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = w[8 * q + e];
                store_words(p + 32 * q, v);
            }
            return;
        }
#pragma unroll
        for (int q = 0; q < kWords / 4; ++q) {
            if ((q + 1) * kEach <= left) {
                reinterpret_cast<uint4 *>(p)[q] = make_uint4(w[4 * q], w[4 * q + 1], w[4 * q + 2], w[4 * q + 3]);
            } else {
#pragma unroll
                for (int e = q * kEach; e < (q + 1) * kEach; ++e) {
                    if (e < left) {
                        if constexpr (G::kBytes == 2)
                            reinterpret_cast<unsigned short *>(p)[e] = static_cast<unsigned short>(w[e / 2] >> (e % 2 * 16));
                        else
                            reinterpret_cast<uint32_t *>(p)[e] = w[e];
                    }
                }
            }
        }
    }
};

template <typename G, int ACT>
__global__ void __launch_bounds__(kKeepThreads) star_checkpoint_pack_kernel(const __grid_constant__ PackArgs a, const __grid_constant__ Halves h)
{
    wait_for_primary();
    // Whole warps go round the loop: neighbours exchange their magnitudes.
    for (uint32_t base = blockIdx.x * kKeepThreads; base < h.n; base += gridDim.x * kKeepThreads) {
        const uint32_t i = base + threadIdx.x;
        const uint32_t row = divide(i, h.per_row), half = i - row * h.per_row.d;
        const int64_t t = static_cast<int64_t>(h.first_row) + row, c = static_cast<int64_t>(half) * 16;
        const bool in = i < h.n && c < a.kept.cols;
        uint32_t w[Sixteen<G>::kWords];
        uint32_t largest = 0;
        if (in) {
            Sixteen<G>::load(static_cast<const char *>(a.x) + t * a.ld * G::kBytes, c, a.kept.cols, h.wide, w);
            largest = Sixteen<G>::largest(w);
        }
        largest = max(largest, __shfl_xor_sync(0xffffffffu, largest, 1));
        if (!in) continue;
        const int s = scale_byte(largest);
        const float inverse = scale_inverse(s);
        float f[16];
        Sixteen<G>::widen(w, f);
        uint32_t codes[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const uint32_t lo = __byte_perm(code_bits(f[4 * q], inverse), code_bits(f[4 * q + 1], inverse), 0x0040);
            const uint32_t hi = __byte_perm(code_bits(f[4 * q + 2], inverse), code_bits(f[4 * q + 3], inverse), 0x0040);
            codes[q] = s == 255 ? 0u : __byte_perm(lo, hi, 0x5410);
        }
        *reinterpret_cast<uint4 *>(a.kept.codes + t * a.kept.pitch + c) = make_uint4(codes[0], codes[1], codes[2], codes[3]);
        if (half % 2 == 0) a.kept.scales[scale_at(a.kept, t, half / 2)] = static_cast<uint8_t>(s);
        if (a.act_out) {
#pragma unroll
            for (int e = 0; e < 16; e += 2) split_pair(activation<ACT, G::kBytes == 4>(make_pair(f[e], f[e + 1])), &f[e], &f[e + 1]);
            Sixteen<G>::store(static_cast<char *>(a.act_out) + t * a.ld_act * G::kBytes, c, a.kept.cols, h.wide, f);
        }
    }
}

// Values of 16 codes; see weight_grad.cuh for the arithmetic.
__device__ __forceinline__ void widen_sixteen(const uint4 &codes, float scale, float (&f)[16])
{
    const uint32_t w[4] = {codes.x, codes.y, codes.z, codes.w};
    const Pair s = pair_of(scale), off = pair_of(__fmul_rn(scale, -8388736.0f));
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const uint32_t u = w[q] ^ 0x80808080u;
        const Pair lo = make_pair(__uint_as_float(__byte_perm(u, 0x4b000000u, 0x7650)), __uint_as_float(__byte_perm(u, 0x4b000000u, 0x7651)));
        const Pair hi = make_pair(__uint_as_float(__byte_perm(u, 0x4b000000u, 0x7652)), __uint_as_float(__byte_perm(u, 0x4b000000u, 0x7653)));
        split_pair(pair_fma(lo, s, off), &f[4 * q], &f[4 * q + 1]);
        split_pair(pair_fma(hi, s, off), &f[4 * q + 2], &f[4 * q + 3]);
    }
}

// out = act(value), or dy * act'(value).
template <typename G, int ACT, bool BACKWARD>
__global__ void __launch_bounds__(kKeepThreads) star_checkpoint_read_kernel(const __grid_constant__ ReadArgs a, const __grid_constant__ Halves h)
{
    wait_for_primary();
    for (uint32_t i = blockIdx.x * kKeepThreads + threadIdx.x; i < h.n; i += gridDim.x * kKeepThreads) {
        const uint32_t row = divide(i, h.per_row), half = i - row * h.per_row.d;
        const int64_t t = static_cast<int64_t>(h.first_row) + row, c = static_cast<int64_t>(half) * 16;
        if (c >= a.kept.cols) continue;
        const uint4 codes = *reinterpret_cast<const uint4 *>(a.kept.codes + t * a.kept.pitch + c);
        const float scale = scale_value(a.kept.scales[scale_at(a.kept, t, half / 2)]);
        uint32_t w[Sixteen<G>::kWords];
        if constexpr (BACKWARD) Sixteen<G>::load(static_cast<const char *>(a.dy) + t * a.ld_dy * G::kBytes, c, a.kept.cols, h.wide, w);
        float f[16];
        widen_sixteen(codes, scale, f);
        if constexpr (BACKWARD) {
            float dy[16];
            Sixteen<G>::widen(w, dy);
#pragma unroll
            for (int e = 0; e < 16; e += 2)
                split_pair(pair_mul(make_pair(dy[e], dy[e + 1]), activation_slope<ACT, G::kBytes == 4>(make_pair(f[e], f[e + 1]))), &f[e], &f[e + 1]);
        } else {
#pragma unroll
            for (int e = 0; e < 16; e += 2) split_pair(activation<ACT, G::kBytes == 4>(make_pair(f[e], f[e + 1])), &f[e], &f[e + 1]);
        }
        Sixteen<G>::store(static_cast<char *>(a.out) + t * a.ld * G::kBytes, c, a.kept.cols, h.wide, f);
    }
}

// ---------------------------------------------------------------------------
// Any alignment: one lane per element, a warp on kLoose neighbouring blocks of a
// row at a time.  Bound by instructions, two to three times slower.
// ---------------------------------------------------------------------------
constexpr int kLoose = 8;

struct Groups {
    Divisor per_row;     // groups of kLoose blocks in a row
    uint32_t first_row;
    uint32_t n;          // groups of this launch
};

template <typename G, int ACT>
__global__ void __launch_bounds__(kKeepThreads) star_checkpoint_pack_loose_kernel(const __grid_constant__ PackArgs a, const __grid_constant__ Groups h)
{
    wait_for_primary();
    const int lane = threadIdx.x % 32;
    for (uint32_t i = blockIdx.x * (kKeepThreads / 32) + threadIdx.x / 32; i < h.n; i += gridDim.x * (kKeepThreads / 32)) {
        const uint32_t row = divide(i, h.per_row), group = i - row * h.per_row.d;
        const int64_t t = static_cast<int64_t>(h.first_row) + row, c0 = static_cast<int64_t>(group) * (kLoose * 32) + lane;
        const char *src = static_cast<const char *>(a.x) + (t * a.ld + c0) * G::kBytes;
        const int left = static_cast<int>(min(a.kept.cols - c0, static_cast<int64_t>(kLoose * 32)));       // this lane's elements lie below
        const int left_code = static_cast<int>(min(a.kept.pitch - c0, static_cast<int64_t>(kLoose * 32)));
        const int blocks = static_cast<int>(min((a.kept.cols - (c0 - lane) + 31) / 32, static_cast<int64_t>(kLoose)));
        float x[kLoose];
#pragma unroll
        for (int q = 0; q < kLoose; ++q) x[q] = 32 * q < left ? load_value<G>(src, 32 * q) : 0.0f;
        int8_t *codes = a.kept.codes + t * a.kept.pitch + c0;
        uint8_t *scales = a.kept.scales + scale_at(a.kept, t, static_cast<int64_t>(group) * kLoose);
        char *out = static_cast<char *>(a.act_out) + (t * a.ld_act + c0) * G::kBytes;
#pragma unroll
        for (int q = 0; q < kLoose; ++q) {
            if (q >= blocks) break;
            const uint32_t largest = __reduce_max_sync(0xffffffffu, __float_as_uint(x[q]) & 0x7fffffffu);
            const int s = scale_byte(largest);
            if (32 * q < left_code) codes[32 * q] = s == 255 ? 0 : static_cast<int8_t>(code_bits(x[q], scale_inverse(s)) & 0xffu);
            if (lane == 0) scales[q / 4 * 4 * a.kept.tall + q % 4] = static_cast<uint8_t>(s);
            if (a.act_out && 32 * q < left) store_value<G>(out, 32 * q, activation<ACT, G::kBytes == 4>(x[q]));
        }
    }
}

template <typename G, int ACT, bool BACKWARD>
__global__ void __launch_bounds__(kKeepThreads) star_checkpoint_read_loose_kernel(const __grid_constant__ ReadArgs a, const __grid_constant__ Groups h)
{
    wait_for_primary();
    const int lane = threadIdx.x % 32;
    for (uint32_t i = blockIdx.x * (kKeepThreads / 32) + threadIdx.x / 32; i < h.n; i += gridDim.x * (kKeepThreads / 32)) {
        const uint32_t row = divide(i, h.per_row), group = i - row * h.per_row.d;
        const int64_t t = static_cast<int64_t>(h.first_row) + row, c0 = static_cast<int64_t>(group) * (kLoose * 32) + lane;
        const int left = static_cast<int>(min(a.kept.cols - c0, static_cast<int64_t>(kLoose * 32)));
        const int8_t *codes = a.kept.codes + t * a.kept.pitch + c0;
        const uint8_t *scales = a.kept.scales + scale_at(a.kept, t, static_cast<int64_t>(group) * kLoose);
        const char *src = static_cast<const char *>(a.dy) + (t * a.ld_dy + c0) * G::kBytes;
        char *out = static_cast<char *>(a.out) + (t * a.ld + c0) * G::kBytes;
        int code[kLoose];
        float scale[kLoose], dy[kLoose];
#pragma unroll
        for (int q = 0; q < kLoose; ++q) {
            const bool in = 32 * q < left;
            code[q] = in ? codes[32 * q] : 0;
            scale[q] = in ? scale_value(scales[q / 4 * 4 * a.kept.tall + q % 4]) : 0.0f;
            dy[q] = BACKWARD && in ? load_value<G>(src, 32 * q) : 0.0f;
        }
#pragma unroll
        for (int q = 0; q < kLoose; ++q) {
            const float x = __fmul_rn(static_cast<float>(code[q]), scale[q]);
            if (32 * q < left) store_value<G>(out, 32 * q, BACKWARD ? __fmul_rn(dy[q], activation_slope<ACT, G::kBytes == 4>(x)) : activation<ACT, G::kBytes == 4>(x));
        }
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

}  // namespace star
