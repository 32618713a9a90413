// What the operators on rows of logits share: running softmax statistics, and
// walking a row in pieces of 16 bytes (sm_100a).
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "device.cuh"

namespace star {

// The arguments of one pass over the rows of a logits matrix.
struct RowArgs {
    const void *logits;
    int64_t ld;
    int64_t rows;
    int64_t vocab;
    const int64_t *labels;
    const float *weights;        // may be null
    float inv_temperature;
};

constexpr float kLn2 = 0.69314718055994531f;

// Exponents.  With k = log2(e) / temperature and a largest logit m, the power
// exp(z - z_max) is 2^((x - m) k).  The difference comes first: it is exact for
// logits near m, exactly 0 for m itself, and cannot overflow where every logit is
// the type's lowest value (one fma of x k - m k would save an instruction and
// lose all three).
// The reference point: the largest logit, 0 where there is none.
__device__ __forceinline__ float pivot(float m) { return m == -INFINITY ? 0.0f : m; }
__device__ __forceinline__ float exponent(float x, float m, float k) { return __fmul_rn(__fsub_rn(x, pivot(m)), k); }

// Largest logit m of a part of a row and the sum of its 2^exponent(x, m).  The
// sum is 0 for a part with nothing but -inf, NaN if it holds a NaN.  The order in
// which parts join is fixed by the caller, so the result is too.
struct MaxSum {
    float m;
    float s;
};

// What a part's sum is multiplied by when the reference goes from its own m to `to`.
__device__ __forceinline__ float rebase(float m, float to, float k)
{
    return exp2_fast(exponent(m, to, k));
}
__device__ __forceinline__ MaxSum join(MaxSum a, MaxSum b, float k)
{
    const float m = fmaxf(a.m, b.m);
    return MaxSum{m, __fadd_rn(__fmul_rn(a.s, rebase(a.m, m, k)), __fmul_rn(b.s, rebase(b.m, m, k)))};
}

// log p of a logit x, with log s split into its exponent's and its mantissa's
// part so that the large terms cancel: the error stays near the result's own ulp
// instead of that of the log-sum-exp (ten times larger at a vocabulary of 50
// thousand).
__device__ __forceinline__ float log_prob(float x, MaxSum row, float k, float inv_temperature)
{
    const int bits = __float_as_int(row.s);
    const int e = (bits >> 23) - 127;                    // s is near 1 or more (the largest logit's own term), or NaN
    const float f = __int_as_float((bits & 0x007fffff) | 0x3f800000);
    const float d = exponent(x, row.m, k);               // log2 of p s
    if (!(row.s < INFINITY)) return __fadd_rn(d, row.s); // NaN
    const float whole = __fsub_rn(d, static_cast<float>(e));
    // A label masked by the type's lowest value: its exponent does not fit, its log p does.
    const float far = __fmul_rn(__fsub_rn(x, pivot(row.m)), inv_temperature);
    return __fsub_rn(d == -INFINITY ? far : __fmul_rn(whole, kLn2), logf(f));
}

__device__ __forceinline__ float log_sum_exp(MaxSum row, float inv_temperature)
{
    return __fmaf_rn(row.m, inv_temperature, logf(row.s));
}

// Whether the label and the weight leave row t active; *label, *weight.
__device__ __forceinline__ bool row_wanted(const RowArgs &a, int64_t t, int64_t *label, float *weight)
{
    *label = a.labels[t];
    *weight = a.weights ? a.weights[t] : 1.0f;
    return *label >= 0 && *label < a.vocab && *weight != 0.0f;
}

// ---------------------------------------------------------------------------
// Walking rows.  A row is taken in 16-byte pieces ("granules") on the 16-byte
// grid of global memory, so that loads and stores are whole whatever the row's
// phase; the up to 15 bytes before and after them are single elements.
//
// What an element costs beside memory: two exponentials at 16 a cycle and SM are
// 72 % of the time that its four bytes take from HBM and back (bf16), and 12
// instructions about as much again.  Differences, products and sums therefore go
// in packed pairs of binary32, maxima in packed pairs of bf16.
// ---------------------------------------------------------------------------
// The largest over the warp, NaNs passed over.
__device__ __forceinline__ float warp_max(float x)
{
    float r;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float warp_sum(float x)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x = __fadd_rn(x, __shfl_xor_sync(0xffffffffu, x, o));
    return x;
}
// Joins the lanes' parts; every lane receives the result.
__device__ __forceinline__ MaxSum warp_join(MaxSum x, float k)
{
    const float m = warp_max(x.m);
    return MaxSum{m, warp_sum(__fmul_rn(x.s, rebase(x.m, m, k)))};
}

template <typename G> struct Granule {
    static constexpr int kCount = 16 / G::kBytes;                // elements
    static constexpr int kPairs = kCount / 2;
    static __device__ __forceinline__ void widen(const uint4 &v, Pair (&f)[kPairs])
    {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
        if constexpr (G::kBytes == 2) {
#pragma unroll
            for (int e = 0; e < 4; ++e) f[e] = make_pair(__uint_as_float(w[e] << 16), __uint_as_float(w[e] & 0xffff0000u));
        } else {
#pragma unroll
            for (int e = 0; e < 2; ++e) f[e] = make_pair(__uint_as_float(w[2 * e]), __uint_as_float(w[2 * e + 1]));
        }
    }
    static __device__ __forceinline__ uint4 narrow(const Pair (&f)[kPairs])
    {
        float x[kCount];
#pragma unroll
        for (int e = 0; e < kPairs; ++e) split_pair(f[e], &x[2 * e], &x[2 * e + 1]);
        if constexpr (G::kBytes == 2)
            return make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
        else
            return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
    }
};

// The largest of granules, kept packed; NaNs are passed over (the sum shows them).
template <typename G> struct RunningMax;
template <> struct RunningMax<GradBF16> {
    uint32_t m[2] = {0xff80ff80u, 0xff80ff80u};                  // -inf
    static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b)
    {
        uint32_t r;
        asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        return r;
    }
    __device__ __forceinline__ void take(const uint4 &v)
    {
        m[0] = larger(m[0], larger(v.x, v.y));
        m[1] = larger(m[1], larger(v.z, v.w));
    }
    __device__ __forceinline__ float value() const
    {
        const uint32_t r = larger(m[0], m[1]);
        return fmaxf(__uint_as_float(r << 16), __uint_as_float(r & 0xffff0000u));
    }
};
template <> struct RunningMax<GradF32> {
    float m[2] = {-INFINITY, -INFINITY};
    __device__ __forceinline__ void take(const uint4 &v)
    {
        m[0] = fmaxf(m[0], fmaxf(__uint_as_float(v.x), __uint_as_float(v.y)));
        m[1] = fmaxf(m[1], fmaxf(__uint_as_float(v.z), __uint_as_float(v.w)));
    }
    __device__ __forceinline__ float value() const { return fmaxf(m[0], m[1]); }
};

// 2^exponent of every element of a granule.
struct Power {
    Pair minus_m, k;
    __device__ __forceinline__ Power(float m, float kf) : minus_m(make_pair(-pivot(m), -pivot(m))), k(make_pair(kf, kf)) {}
    template <int N> __device__ __forceinline__ void apply(Pair (&f)[N]) const
    {
#pragma unroll
        for (int e = 0; e < N; ++e) {
            float lo, hi;
            split_pair(pair_mul(pair_add(f[e], minus_m), k), &lo, &hi);
            f[e] = make_pair(exp2_fast(lo), exp2_fast(hi));
        }
    }
};

// How a row's elements fall on the 16-byte grid.
struct RowSplit {
    int head;        // elements before the first granule
    int granules;
    int tail;        // elements after the last
};
template <typename G> __device__ __forceinline__ RowSplit split_row(const void *row, int vocab)
{
    constexpr unsigned E = Granule<G>::kCount;
    const unsigned to_grid = (-static_cast<unsigned>(reinterpret_cast<uintptr_t>(row)) & 15u) / G::kBytes;
    const unsigned head = min(to_grid, static_cast<unsigned>(vocab)), rest = static_cast<unsigned>(vocab) - head;
    return RowSplit{static_cast<int>(head), static_cast<int>(rest / E), static_cast<int>(rest % E)};
}

// The granules [begin, begin + count) of a row that a block of a cluster takes.
struct RowShare {
    int begin, count;
};
__device__ __forceinline__ RowShare row_share(int granules, uint32_t rank, int log_blocks)
{
    const int each = (granules + (1 << log_blocks) - 1) >> log_blocks, begin = min(each * static_cast<int>(rank), granules);
    return RowShare{begin, min(each, granules - begin)};
}

constexpr int kBatch = 4;            // granules that a thread loads at once
// Blocks of an SM that the kernels are compiled for: the statistics alone in 1280
// threads of 48 registers, with the gradient 1024 of 64.
__host__ __device__ constexpr int row_blocks(int threads) { return 1280 / threads > 32 ? 32 : 1280 / threads; }
__host__ __device__ constexpr int policy_blocks(int threads) { return 1024 / threads; }

// Takes up to N granules, THREADS apart, into a thread's running maximum and
// sum: the maximum first, on packed pairs, then one rescaling and the powers.
// FULL: all N are there.
template <typename G, int N, int THREADS, bool FULL>
__device__ __forceinline__ void take_batch(MaxSum *x, const uint4 *from, int left, float k)
{
    constexpr int P = Granule<G>::kPairs;
    uint4 v[N];
#pragma unroll
    for (int q = 0; q < N; ++q)
        if (FULL || q * THREADS < left) v[q] = from[q * THREADS];
    RunningMax<G> most;
#pragma unroll
    for (int q = 0; q < N; ++q)
        if (FULL || q * THREADS < left) most.take(v[q]);
    const float m = most.value();
    if (m > x->m) {
        x->s = __fmul_rn(x->s, exp2_fast(exponent(x->m, m, k)));
        x->m = m;
    }
    const Power power(x->m, k);
    Pair total = make_pair(0.0f, 0.0f);
#pragma unroll
    for (int q = 0; q < N; ++q) {
        if (FULL || q * THREADS < left) {
            Pair f[P];
            Granule<G>::widen(v[q], f);
            power.apply(f);
#pragma unroll
            for (int o = P / 2; o > 0; o >>= 1)
#pragma unroll
                for (int e = 0; e < o; ++e) f[e] = pair_add(f[e], f[e + o]);
            total = pair_add(total, f[0]);
        }
    }
    float lo, hi;
    split_pair(total, &lo, &hi);
    x->s = __fadd_rn(x->s, __fadd_rn(lo, hi));
}

// The gradient of up to N granules.
template <typename G, int N, int THREADS, bool FULL>
__device__ __forceinline__ void store_batch(uint4 *to, const uint4 *from, int left, const Power &power, float scale)
{
    constexpr int P = Granule<G>::kPairs;
    const Pair scales = make_pair(scale, scale);
    uint4 v[N];
#pragma unroll
    for (int q = 0; q < N; ++q)
        if (FULL || q * THREADS < left) v[q] = from[q * THREADS];
#pragma unroll
    for (int q = 0; q < N; ++q) {
        if (FULL || q * THREADS < left) {
            Pair g[P];
            Granule<G>::widen(v[q], g);
            power.apply(g);
#pragma unroll
            for (int e = 0; e < P; ++e) g[e] = pair_mul(g[e], scales);
            to[q * THREADS] = Granule<G>::narrow(g);
        }
    }
}

// Joins the warps' parts; meaningful in warp 0.  `sync` waits for the warps.
template <int WARPS, typename Sync> __device__ __forceinline__ MaxSum block_join(MaxSum x, MaxSum *part, float k, Sync sync)
{
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    x = warp_join(x, k);
    if constexpr (WARPS > 1) {
        if (lane == 0) part[warp] = x;
        sync();
        if (warp == 0) x = warp_join(lane < WARPS ? part[lane] : MaxSum{-INFINITY, 0.0f}, k);
    }
    return x;
}

// Joins the blocks' parts; meaningful in warp 0 of every block.
__device__ __forceinline__ MaxSum cluster_join(MaxSum x, MaxSum (&part)[8], uint32_t blocks, uint32_t rank, float k)
{
    const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    if (warp == 0 && lane < blocks) {
        const uint32_t at = peer_address(smem_address(&part[rank]), lane);
        asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" :: "r"(at), "f"(x.m), "f"(x.s) : "memory");
    }
    cluster_sync();
    if (warp == 0) x = warp_join(lane < blocks ? part[lane] : MaxSum{-INFINITY, 0.0f}, k);
    return x;
}

// The element beside the granules that thread i takes, or -1.
__device__ __forceinline__ int edge_element(const RowSplit &s, int i, int vocab)
{
    if (i >= s.head + s.tail) return -1;
    return i < s.head ? i : vocab - s.tail + (i - s.head);
}

// Sums n values per thread slot in a fixed order, in binary64.
__device__ __forceinline__ double block_sum(double x, double *shared)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    __syncthreads();
    if (threadIdx.x % 32 == 0) shared[threadIdx.x / 32] = x;
    __syncthreads();
    x = shared[0];
    for (int w = 1; w < static_cast<int>(blockDim.x) / 32; ++w) x += shared[w];
    return x;
}

}  // namespace star
