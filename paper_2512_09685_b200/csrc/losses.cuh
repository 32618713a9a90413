// Device code of the losses over the vocabulary (sm_100a).
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

// What the preference loss keeps of a row between its steps.
struct RowKept {
    float m;         // largest logit
    float inv_s;     // 1 / sum of exp(z - z_max); 0 for an inactive row
    float logp;
    float coef;
};

// What is made of the rows.  POLICY: the loss and its sums.  Otherwise the
// log-probability alone.
struct RowWork {
    RowArgs row;
    float *logp;                 // may be null where kept is given
    float *lse;                  // may be null
    RowKept *kept;               // may be null
    // POLICY only
    const float *advantages;
    const float *old_logp;       // may be null
    const float *ref_logp;       // may be null
    float clip_low, clip_high, kl_coef;
    float *token_loss;
    float4 *partial;             // the four sums of each block's (cluster's) rows
    void *dlogits;               // may be null
    int64_t ld_dlogits;
    int tries;                   // of a wait
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

// What one active row contributes, and the factor of its gradient:
// dlogits[j] = coef * ((j == label) - p[j]).
struct PolicyRow {
    float loss, gain, kl, clipped, coef;
};

__device__ __forceinline__ PolicyRow policy_row(float lp, float advantage, bool has_old, float old_lp, bool has_ref,
                                                float ref_lp, float clip_low, float clip_high, float kl_coef,
                                                float weight, float inv_temperature)
{
    const float r = has_old ? expf(__fsub_rn(lp, old_lp)) : lp != lp ? lp : 1.0f;    // a NaN row shows in the totals
    // A factor of exactly 0 takes its term out, also where the other one is beyond binary32.
    const bool out_of_it = advantage == 0.0f && r == INFINITY;
    const float u = out_of_it ? 0.0f : __fmul_rn(r, advantage);
    const float c = out_of_it ? 0.0f : __fmul_rn(fminf(fmaxf(r, __fsub_rn(1.0f, clip_low)), __fadd_rn(1.0f, clip_high)), advantage);
    PolicyRow out;
    out.clipped = u > c ? 1.0f : 0.0f;
    const float gain = u > c ? c : u;                    // a NaN in u stays
    float slope = u > c ? 0.0f : -u;
    out.kl = 0.0f;
    float loss = -gain;
    if (has_ref) {
        const float d = __fsub_rn(ref_lp, lp);
        // exp(d) - d - 1 without the cancellation at small d.
        const float em1 = expm1f(d);
        out.kl = __fsub_rn(em1, d);
        if (kl_coef != 0.0f) {
            loss = __fmaf_rn(kl_coef, out.kl, loss);
            slope = __fmaf_rn(kl_coef, -em1, slope);
        }
    }
    out.loss = loss;
    out.gain = gain;
    out.coef = __fmul_rn(__fmul_rn(weight, slope), inv_temperature);
    return out;
}

// Whether the label and the weight leave row t active; *label, *weight.
__device__ __forceinline__ bool row_wanted(const RowArgs &a, int64_t t, int64_t *label, float *weight)
{
    *label = a.labels[t];
    *weight = a.weights ? a.weights[t] : 1.0f;
    return *label >= 0 && *label < a.vocab && *weight != 0.0f;
}

// The scalars of a row, by one thread: its results, and what the gradient needs.
struct alignas(16) RowFactors {
    float m;         // largest logit
    float scale;     // -coef / sum: dlogits[j] = scale * 2^exponent(x, m), + coef at the label
    float coef;
    float label_power;           // 2^exponent(label's logit, m)
    int active;
    int late;                    // a wait for the row ran out: nothing of it holds
};

// What belongs to a row beside its logits, for the thread that finishes it.
struct RowIn {
    float label_logit, advantage, old_lp, ref_lp;
};

struct RowSums {
    double loss, gain, kl, clipped;
};

// The part that others wait for.
template <bool POLICY>
__device__ __forceinline__ RowFactors make_factors(const RowWork &a, bool wanted, MaxSum row, float weight, const RowIn &in, float *lp, PolicyRow *r)
{
    const float inv_t = a.row.inv_temperature, k = __fmul_rn(inv_t, kLog2e);
    RowFactors f{row.m, 0.0f, 0.0f, 0.0f, wanted && !(row.s == 0.0f) ? 1 : 0, 0};
    *lp = 0.0f;
    *r = PolicyRow{0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
    if (f.active) {
        *lp = log_prob(in.label_logit, row, k, inv_t);
        if constexpr (POLICY) {
            *r = policy_row(*lp, in.advantage, a.old_logp != nullptr, in.old_lp, a.ref_logp != nullptr, in.ref_lp, a.clip_low,
                            a.clip_high, a.kl_coef, weight, inv_t);
            f.coef = r->coef;
            f.scale = __fdiv_rn(-r->coef, row.s);
            f.label_power = exp2_fast(exponent(in.label_logit, row.m, k));
        }
    }
    return f;
}
// The rest: results and sums.
template <bool POLICY, bool KEEPS>
__device__ __forceinline__ void finish_row(const RowWork &a, int64_t t, const RowFactors &f, MaxSum row, float weight, float lp,
                                           const PolicyRow &r, RowSums *sums)
{
    if (a.logp) a.logp[t] = lp;
    if constexpr (POLICY) {
        if (f.active) {
            sums->loss += static_cast<double>(weight) * r.loss;
            sums->gain -= static_cast<double>(weight) * r.gain;
            sums->kl += static_cast<double>(weight) * r.kl;
            sums->clipped += static_cast<double>(weight) * r.clipped;
        }
        a.token_loss[t] = r.loss;
    } else {
        if (a.lse) a.lse[t] = f.active ? log_sum_exp(row, a.row.inv_temperature) : 0.0f;
    }
    if (KEEPS && a.kept) a.kept[t] = RowKept{row.m, f.active ? __fdiv_rn(1.0f, row.s) : 0.0f, lp, r.coef};
}

// A block's sums, rounded to binary32 once; they are added in binary64 again.
template <bool POLICY> __device__ __forceinline__ void store_partial(const RowWork &a, int64_t at, const RowSums &sums)
{
    if constexpr (POLICY)
        a.partial[at] = make_float4(static_cast<float>(sums.loss), static_cast<float>(sums.gain), static_cast<float>(sums.kl),
                                    static_cast<float>(sums.clipped));
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

// ---------------------------------------------------------------------------
// The rows' statistics.  A block, or a cluster of 2 to 8 blocks where there are
// few rows, owns a row; every thread keeps a running maximum and sum, which join
// through warps, block and cluster, and one thread makes the row's results.
// Nothing is shared between a row's elements until the join, so many small
// blocks hide one another's loads: 4096 x 50257 bf16 in 68 us (6.0 TB/s; blocks
// of 512 and 1024 threads took 92), 16384 x 16000 in 86 (6.1 TB/s).
// ---------------------------------------------------------------------------
template <typename G, bool POLICY, int THREADS>
__global__ void __launch_bounds__(THREADS, row_blocks(THREADS)) star_row_kernel(const __grid_constant__ RowWork a)
{
    constexpr int kWarps = THREADS / 32, kStep = kBatch * THREADS;
    __shared__ MaxSum warp_part[2][kWarps];
    __shared__ alignas(8) MaxSum block_part[2][8];
    __shared__ float row_in[4];                                  // a RowIn
    __shared__ RowSums sums;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const uint32_t blocks = cluster_size(), rank = cluster_rank();
    const int log_blocks = 31 - __clz(static_cast<int>(blocks));
    const int64_t first = blockIdx.x >> log_blocks, step = gridDim.x >> log_blocks;
    const float k = __fmul_rn(a.row.inv_temperature, kLog2e);
    const int vocab = static_cast<int>(a.row.vocab);
    launch_dependents();
    if (threadIdx.x == 0) sums = RowSums{0.0, 0.0, 0.0, 0.0};
    if (blocks > 1) cluster_sync();                              // the others have started
    wait_for_primary();

    int parity = 0;
    for (int64_t t = first; t < a.row.rows; t += step, parity ^= 1) {
        int64_t label;
        float weight;
        const bool wanted = row_wanted(a.row, t, &label, &weight);
        MaxSum x{-INFINITY, 0.0f};
        if (wanted) {
            const char *base = static_cast<const char *>(a.row.logits) + t * a.row.ld * G::kBytes;
            const RowSplit s = split_row<G>(base, vocab);
            const RowShare own = row_share(s.granules, rank, log_blocks);
            const int edge_at = rank == 0 ? edge_element(s, threadIdx.x, vocab) : -1;
            float edge = 0.0f;
            if (edge_at >= 0) edge = load_value<G>(base, edge_at);
            if (rank == 0 && threadIdx.x < (POLICY ? 4 : 1)) {
                float in = 0.0f;
                if (threadIdx.x == 0) in = load_value<G>(base, label);
                if constexpr (POLICY) {
                    if (threadIdx.x == 1) in = a.advantages[t];
                    if (threadIdx.x == 2 && a.old_logp) in = a.old_logp[t];
                    if (threadIdx.x == 3 && a.ref_logp) in = a.ref_logp[t];
                }
                row_in[threadIdx.x] = in;
            }
            int left = own.count - static_cast<int>(threadIdx.x);
            const uint4 *from = reinterpret_cast<const uint4 *>(base + s.head * G::kBytes) + own.begin + threadIdx.x;
            for (; left > kStep - THREADS; left -= kStep, from += kStep) take_batch<G, kBatch, THREADS, true>(&x, from, left, k);
            if (left > 0) take_batch<G, kBatch, THREADS, false>(&x, from, left, k);
            if (edge_at >= 0) x = join(x, MaxSum{edge, exp2_fast(exponent(edge, edge, k))}, k);
        }
        x = block_join<kWarps>(x, warp_part[parity], k, [] { __syncthreads(); });
        if (blocks > 1) x = cluster_join(x, block_part[parity], blocks, rank, k);
        if (warp == 0 && rank == 0) {
            __syncwarp();                                        // row_in is written
            if (lane == 0) {
                float lp;
                PolicyRow r;
                const RowFactors f = make_factors<POLICY>(a, wanted, x, weight, RowIn{row_in[0], row_in[1], row_in[2], row_in[3]}, &lp, &r);
                finish_row<POLICY, true>(a, t, f, x, weight, lp, r, &sums);
            }
            __syncwarp();                                        // and read, before the next row's
        }
    }
    if (threadIdx.x == 0 && rank == 0) store_partial<POLICY>(a, first, sums);
    if (blocks > 1) cluster_sync();                              // nobody leaves while a peer reads its memory
}

// ---------------------------------------------------------------------------
// The policy loss with its gradient in one reading: a row comes by one bulk copy
// and stays in shared memory from its statistics to its gradient.  Blocks of
// THREADS, as many on an SM as make 1024 threads, so that one block's copy, joins
// and waits run under another's arithmetic.  Longer rows lie in the shared memory
// of a cluster's blocks, which join their parts and each make all factors.  The
// thread that finishes a row makes its factors first and lets the others go before
// it writes results and sums.
//
// A wait that runs out ends all blocks of the row's cluster after that row's joins,
// without results from this row on and with sums of NaN.
//
// 4096 x 50257 bf16, no row masked: 161 us, 5.1 TB/s of reading and writing;
// 4096 x 131072 480 us, 4.5 TB/s.  Other arrangements of the same arithmetic, at
// 50257: two rows in shared memory and one block of 1024 threads 190 us (its warps
// all join at once); four blocks an SM, two to a row, 170; no shared memory and a
// second reading from L1 and L2 186; the copy in 2 or 4 parts, the next row's
// following the second walk part by part, 166 to 212.
// ---------------------------------------------------------------------------
constexpr int kKeepBytesPerThread = 224;     // shared memory for the row: 224 KB an SM

template <typename G, int THREADS, bool CLUSTER>
__global__ void __launch_bounds__(THREADS, policy_blocks(THREADS)) star_policy_kernel(const __grid_constant__ RowWork a)
{
    constexpr int E = Granule<G>::kCount, kWarps = THREADS / 32, kStep = kBatch * THREADS;
    extern __shared__ uint4 kept_row[];
    __shared__ MaxSum warp_part[2][kWarps];
    __shared__ alignas(8) MaxSum block_part[2][8];
    __shared__ RowFactors factors;
    __shared__ RowSums sums;
    __shared__ RowIn row_in;                                     // and the row's weight and label: thread 0's alone
    __shared__ float row_weight;
    __shared__ int row_label;
    // A wait for the row ran out, in any block of the cluster.  One for every other row: a block
    // may tell of the next row while another has yet to read this row's.
    __shared__ int late[2];
    __shared__ alignas(8) uint64_t landed;                       // the row's copy is in place
    const float k = __fmul_rn(a.row.inv_temperature, kLog2e);
    const int vocab = static_cast<int>(a.row.vocab);
    const bool writes = a.dlogits != nullptr;
    const uint32_t blocks = CLUSTER ? cluster_size() : 1, rank = CLUSTER ? cluster_rank() : 0;
    const int log_blocks = CLUSTER ? 31 - __clz(static_cast<int>(blocks)) : 0;
    const int64_t first = blockIdx.x >> log_blocks, step = gridDim.x >> log_blocks;
    launch_dependents();
    if (threadIdx.x == 0) {
        sums = RowSums{0.0, 0.0, 0.0, 0.0};
        late[0] = late[1] = factors.late = 0;
        barrier_init(smem_address(&landed), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    if (blocks > 1) cluster_sync();                              // the others have started
    wait_for_primary();

    const auto row_base = [&](int64_t t) { return static_cast<const char *>(a.row.logits) + t * a.row.ld * G::kBytes; };
    // Thread 0: fetches the block's share of row t.
    const auto fetch = [&](int64_t t) {
        const char *base = row_base(t);
        const RowSplit s = split_row<G>(base, vocab);
        const RowShare own = row_share(s.granules, rank, log_blocks);
        if (own.count == 0) return;
        const uint32_t bytes = static_cast<uint32_t>(own.count) * 16, bar = smem_address(&landed);
        barrier_expect(bar, bytes);
        bulk_load(smem_address(kept_row), base + s.head * G::kBytes + static_cast<int64_t>(own.begin) * 16, bytes, bar);
    };

    uint32_t phase = 0;
    int parity = 0;
    bool wanted;
    {
        int64_t label;
        float weight;
        wanted = row_wanted(a.row, first, &label, &weight);
        if (wanted && threadIdx.x == 0) {
            fetch(first);
            row_label = static_cast<int>(label);
            row_weight = weight;
        }
    }
    for (int64_t t = first; t < a.row.rows && !factors.late; t += step, parity ^= 1) {
        const RowSplit s = split_row<G>(row_base(t), vocab);
        const RowShare own = row_share(s.granules, rank, log_blocks);
        // The next row's label and weight are on their way.
        int64_t next_label = -1;
        float next_weight = 0.0f;
        if (t + step < a.row.rows) {
            next_label = a.row.labels[t + step];
            next_weight = a.row.weights ? a.row.weights[t + step] : 1.0f;
        }
        const int edge_at = rank == 0 ? edge_element(s, threadIdx.x, vocab) : -1;
        float edge = 0.0f;
        MaxSum x{-INFINITY, 0.0f};
        if (wanted) {
            if (edge_at >= 0) edge = load_value<G>(row_base(t), edge_at);
            if (threadIdx.x == 0) {
                row_in.label_logit = load_value<G>(row_base(t), row_label);
                row_in.advantage = a.advantages[t];
                row_in.old_lp = a.old_logp ? a.old_logp[t] : 0.0f;
                row_in.ref_lp = a.ref_logp ? a.ref_logp[t] : 0.0f;
            }
            if (own.count > 0) {
                if (!barrier_wait(smem_address(&landed), phase, a.tries)) {
                    late[parity] = 1;                            // what the walk below finds is not used
                    for (uint32_t q = 0; CLUSTER && q < blocks; ++q)
                        asm volatile("st.shared::cluster.s32 [%0], 1;" :: "r"(peer_address(smem_address(&late[parity]), q)) : "memory");
                }
                phase ^= 1;
            }
            const uint4 *from = kept_row + threadIdx.x;
            int left = own.count - static_cast<int>(threadIdx.x);
            for (; left > kStep - THREADS; left -= kStep, from += kStep) take_batch<G, kBatch, THREADS, true>(&x, from, left, k);
            if (left > 0) take_batch<G, kBatch, THREADS, false>(&x, from, left, k);
            if (edge_at >= 0) x = join(x, MaxSum{edge, exp2_fast(exponent(edge, edge, k))}, k);
        }
        x = block_join<kWarps>(x, warp_part[parity], k, [] { __syncthreads(); });
        if (blocks > 1) x = cluster_join(x, block_part[parity], blocks, rank, k);
        float lp;
        PolicyRow r;
        if (kWarps == 1) __syncwarp();                           // `late` is written, the last row's factors are read
        if (threadIdx.x == 0) {
            factors = make_factors<true>(a, wanted, x, row_weight, row_in, &lp, &r);
            factors.late = late[parity];
        }
        __syncthreads();                                         // the factors; and the first walk is over
        const bool ended = factors.late != 0;
        const bool next_wanted = next_label >= 0 && next_label < vocab && next_weight != 0.0f && !ended;
        if (threadIdx.x == 0 && rank == 0 && !ended) finish_row<true, false>(a, t, factors, x, row_weight, lp, r, &sums);
        if (writes && !ended) {
            const RowFactors f = factors;
            char *out = static_cast<char *>(a.dlogits) + t * a.ld_dlogits * G::kBytes;
            const bool same_phase = (reinterpret_cast<uintptr_t>(out) - reinterpret_cast<uintptr_t>(row_base(t))) % 16 == 0;
            if (same_phase) {
                uint4 *to = reinterpret_cast<uint4 *>(out + s.head * G::kBytes) + own.begin + threadIdx.x;
                int left = own.count - static_cast<int>(threadIdx.x);
                if (f.active) {
                    const Power power(f.m, k);
                    const uint4 *from = kept_row + threadIdx.x;
                    for (; left > kStep - THREADS; left -= kStep, from += kStep, to += kStep)
                        store_batch<G, kBatch, THREADS, true>(to, from, left, power, f.scale);
                    if (left > 0) store_batch<G, kBatch, THREADS, false>(to, from, left, power, f.scale);
                } else {
                    for (; left > 0; left -= THREADS, to += THREADS) *to = make_uint4(0, 0, 0, 0);
                }
            } else {
                for (int e = threadIdx.x; e < own.count * E; e += THREADS)
                    store_value<G>(out, s.head + own.begin * E + e, f.active ? __fmul_rn(f.scale, exp2_fast(exponent(load_value<G>(kept_row, e), f.m, k))) : 0.0f);
            }
            if (edge_at >= 0)
                store_value<G>(out, edge_at, f.active ? __fmul_rn(f.scale, exp2_fast(exponent(edge, f.m, k))) : 0.0f);
            __syncthreads();                                     // the row is read and written
            // The label's element again, by the block that has it.
            if (threadIdx.x == 0 && f.active) {
                const int at = row_label - s.head;
                const bool in_granules = at >= 0 && at < s.granules * E;
                const bool has_label = in_granules ? at / E >= own.begin && at / E < own.begin + own.count : rank == 0;
                if (has_label) store_value<G>(out, row_label, __fmaf_rn(f.scale, f.label_power, f.coef));
            }
        }
        if (next_wanted && threadIdx.x == 0) {
            fetch(t + step);
            row_label = static_cast<int>(next_label);
            row_weight = next_weight;
        }
        wanted = next_wanted;
    }
    if (threadIdx.x == 0 && factors.late) {
        barrier_wait(smem_address(&landed), phase ^ 1, kWaitTries);      // the copy in flight, if any
        sums.loss = sums.gain = sums.kl = sums.clipped = NAN;
    }
    if (threadIdx.x == 0 && rank == 0) store_partial<true>(a, blockIdx.x >> log_blocks, sums);
}

constexpr int kSumThreads = 1024;

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

// sums[0 .. 4) from the parts of n blocks or clusters, by one block.
__device__ __forceinline__ void policy_total(const float4 *partial, int64_t n, float *sums, double *shared)
{
    double s[4] = {0.0, 0.0, 0.0, 0.0};
    for (int64_t i = threadIdx.x; i < n; i += blockDim.x) {
        const float4 x = partial[i];
        s[0] += x.x; s[1] += x.y; s[2] += x.z; s[3] += x.w;
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const double total = block_sum(s[q], shared);
        if (threadIdx.x == 0) sums[q] = static_cast<float>(total);
    }
}

__global__ void __launch_bounds__(kSumThreads) star_policy_sums_kernel(const float4 *partial, int64_t n, float *sums)
{
    __shared__ double shared[kSumThreads / 32];
    wait_for_primary();
    policy_total(partial, n, sums, shared);
}

// ---------------------------------------------------------------------------
// The preference loss in three steps: the rows' log-probabilities (above); per
// pair the loss and every row's factor; the gradient.
// ---------------------------------------------------------------------------
struct PreferenceArgs {
    RowArgs row;
    RowKept *kept;
    const int32_t *seq_offsets;
    int64_t pairs;
    const float *ref_seq_logp;   // may be null
    float beta, smoothing, loss_scale;
    int average;
    float *seq_logp, *pair_loss, *margin, *loss;
    void *dlogits;
    int64_t ld_dlogits;
};

// log(1 + exp(-x))
__device__ __forceinline__ float softplus_neg(float x)
{
    return __fadd_rn(log1pf(expf(-fabsf(x))), fmaxf(-x, 0.0f));
}

constexpr int kPairThreads = 256;

// One block per pair.
__global__ void __launch_bounds__(kPairThreads) star_preference_pair_kernel(const __grid_constant__ PreferenceArgs a)
{
    __shared__ double shared[kPairThreads / 32];
    launch_dependents();
    wait_for_primary();
    for (int64_t i = blockIdx.x; i < a.pairs; i += gridDim.x) {
        int64_t first[2], last[2];
        double total[2], count[2];
        for (int q = 0; q < 2; ++q) {
            first[q] = min(max(static_cast<int64_t>(a.seq_offsets[2 * i + q]), int64_t{0}), a.row.rows);
            last[q] = min(max(static_cast<int64_t>(a.seq_offsets[2 * i + q + 1]), int64_t{0}), a.row.rows);
            double s = 0.0, n = 0.0;
            for (int64_t t = first[q] + threadIdx.x; t < last[q]; t += kPairThreads) {
                s += a.kept[t].logp;
                n += a.kept[t].inv_s == 0.0f ? 0.0 : 1.0;
            }
            total[q] = block_sum(s, shared);
            count[q] = a.average ? fmax(block_sum(n, shared), 1.0) : 1.0;
            total[q] /= count[q];
        }
        double h = total[0] - total[1];
        if (a.ref_seq_logp) h -= static_cast<double>(a.ref_seq_logp[2 * i]) - static_cast<double>(a.ref_seq_logp[2 * i + 1]);
        const float bh = static_cast<float>(a.beta * h);
        const float e = a.smoothing;
        if (threadIdx.x == 0) {
            a.seq_logp[2 * i] = static_cast<float>(total[0]);
            a.seq_logp[2 * i + 1] = static_cast<float>(total[1]);
            a.margin[i] = bh;
            // A factor of exactly 0 takes its term out, however large the margin.
            const float yes = e == 1.0f ? 0.0f : __fmul_rn(1.0f - e, softplus_neg(bh));
            const float no = e == 0.0f ? 0.0f : __fmul_rn(e, softplus_neg(-bh));
            a.pair_loss[i] = __fadd_rn(yes, no);
        }
        // sigmoid(-bh) and sigmoid(bh), each from an exponential that cannot overflow.
        const float x = expf(-fabsf(bh)), big = __fdiv_rn(1.0f, __fadd_rn(1.0f, x)), small = __fmul_rn(x, big);
        const float neg = bh >= 0.0f ? small : big, pos = bh >= 0.0f ? big : small;
        const float slope = -__fmul_rn(a.beta, __fsub_rn(__fmul_rn(1.0f - e, neg), __fmul_rn(e, pos)));
        for (int q = 0; q < 2; ++q) {
            const float coef = static_cast<float>((q ? -1.0 : 1.0) * static_cast<double>(slope) * a.loss_scale *
                                                  a.row.inv_temperature / count[q]);
            for (int64_t t = first[q] + threadIdx.x; t < last[q]; t += kPairThreads) a.kept[t].coef = coef;
        }
    }
}

// loss[0], by the first block of whatever runs last.
__device__ __forceinline__ void preference_total(const float *pair_loss, int64_t pairs, float loss_scale, float *loss, double *shared)
{
    double s = 0.0;
    for (int64_t i = threadIdx.x; i < pairs; i += blockDim.x) s += pair_loss[i];
    s = block_sum(s, shared);
    if (threadIdx.x == 0) loss[0] = static_cast<float>(s * loss_scale);
}

__global__ void __launch_bounds__(kPairThreads) star_preference_total_kernel(const __grid_constant__ PreferenceArgs a)
{
    __shared__ double shared[kPairThreads / 32];
    wait_for_primary();
    preference_total(a.pair_loss, a.pairs, a.loss_scale, a.loss, shared);
}

// ---------------------------------------------------------------------------
// The gradient from what was kept of the rows, in a second reading of the logits:
// for the preference loss, because a row's factor needs every row of its pair;
// for the policy loss where rows are few or too long for shared memory.  Rows are
// taken from the last to the first, so that those read last by the first step are
// still in L2.  A warp takes a run of kGradGranules granules of a row at a time:
// nothing is shared between warps, and short rows fill the blocks as long ones do.
// ---------------------------------------------------------------------------
constexpr int kRowThreads = 256;
constexpr int kGradPerThread = 4;
constexpr int kGradGranules = 32 * kGradPerThread;

struct GradArgs {
    RowArgs row;
    const RowKept *kept;
    void *dlogits;
    int64_t ld_dlogits;
    // The sums that the first block makes: of the pairs' losses, or of the policy loss's parts.
    const float *pair_loss;
    int64_t pairs;
    float loss_scale;
    float *loss;
    const float4 *partial;
    int64_t parts;
    float *sums;
};

template <typename G, bool POLICY> __global__ void __launch_bounds__(kRowThreads, 4) star_row_gradient_kernel(const __grid_constant__ GradArgs a)
{
    constexpr int E = Granule<G>::kCount;
    __shared__ double shared[kRowThreads / 32];
    wait_for_primary();
    if (blockIdx.x == 0) {
        if constexpr (POLICY)
            policy_total(a.partial, a.parts, a.sums, shared);
        else
            preference_total(a.pair_loss, a.pairs, a.loss_scale, a.loss, shared);
    }
    const float k = __fmul_rn(a.row.inv_temperature, kLog2e);
    const int64_t per_row = (a.row.vocab / E + kGradGranules) / kGradGranules;           // the last run may be empty
    const int64_t items = a.row.rows * per_row;
    const int lane = threadIdx.x % 32, warps = kRowThreads / 32;
    for (int64_t item = static_cast<int64_t>(blockIdx.x) * warps + threadIdx.x / 32; item < items; item += static_cast<int64_t>(gridDim.x) * warps) {
        // A division in 32 bits, five times cheaper, for all but the largest.
        const int64_t row = items <= 0xffffffff ? static_cast<uint32_t>(item) / static_cast<uint32_t>(per_row) : item / per_row;
        const int64_t t = a.row.rows - 1 - row, run = item - row * per_row;
        const RowKept r = a.kept[t];
        const bool active = r.inv_s != 0.0f && r.coef != 0.0f;
        const char *base = static_cast<const char *>(a.row.logits) + t * a.row.ld * G::kBytes;
        char *out = static_cast<char *>(a.dlogits) + t * a.ld_dlogits * G::kBytes;
        const RowSplit s = split_row<G>(base, static_cast<int>(a.row.vocab));
        const int64_t label = active ? a.row.labels[t] : -1;
        const float scale = __fmul_rn(-r.coef, r.inv_s);
        const auto grad = [&](float x, int64_t at) {
            const float g = __fmul_rn(scale, exp2_fast(exponent(x, r.m, k)));
            return at == label ? __fadd_rn(g, r.coef) : g;
        };
        const bool same_phase = (reinterpret_cast<uintptr_t>(out) - reinterpret_cast<uintptr_t>(base)) % 16 == 0;
        const int begin = static_cast<int>(run) * kGradGranules, end = min(begin + kGradGranules, s.granules);
        if (same_phase) {
            const uint4 *src = reinterpret_cast<const uint4 *>(base + s.head * G::kBytes);
            uint4 *dst = reinterpret_cast<uint4 *>(out + s.head * G::kBytes);
            if (active) {
                const int64_t at_label = label - s.head;
                const bool label_here = at_label >= static_cast<int64_t>(begin) * E && at_label < static_cast<int64_t>(end) * E &&
                                        (at_label / E - begin) % 32 == lane;
                const float label_logit = label_here ? load_value<G>(src, at_label) : 0.0f;      // before an in-place store
                const int at = begin + lane, left = end - at;
                const Power power(r.m, k);
                if (left > (kGradPerThread - 1) * 32)
                    store_batch<G, kGradPerThread, 32, true>(dst + at, src + at, left, power, scale);
                else if (left > 0)
                    store_batch<G, kGradPerThread, 32, false>(dst + at, src + at, left, power, scale);
                if (label_here) store_value<G>(dst, at_label, grad(label_logit, label));         // by the thread that stored its granule
            } else {
                for (int i = begin + lane; i < end; i += 32) dst[i] = make_uint4(0, 0, 0, 0);
            }
        } else {
            const int64_t last = s.head + static_cast<int64_t>(end) * E;
            for (int64_t at = s.head + static_cast<int64_t>(begin) * E + lane; at < last; at += 32)
                store_value<G>(out, at, active ? grad(load_value<G>(base, at), at) : 0.0f);
        }
        if (run == 0 && lane < s.head + s.tail) {
            const int64_t at = lane < s.head ? lane : a.row.vocab - s.tail + (lane - s.head);
            store_value<G>(out, at, active ? grad(load_value<G>(base, at), at) : 0.0f);
        }
    }
}

}  // namespace star
