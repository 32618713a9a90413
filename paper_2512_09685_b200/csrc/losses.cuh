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

// What is made of a row's statistics.  POLICY: loss, sums and, where dlogits is
// given, the gradient.  Otherwise the log-probability alone.
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
    float4 *partial;             // the four sums of each cluster's rows
    void *dlogits;               // may be null
    int64_t ld_dlogits;
    int granules;                // 16-byte pieces of a row that one block holds at most
};

// ln 2 in two terms (Cody and Waite): the first has 12 bits, so its product with
// an exponent of up to 10 bits is exact.
constexpr float kLn2Hi = 0.693115234375f;
constexpr float kLn2Lo = 3.19461849453e-05f;

// (largest logit, sum of exp(z - largest z)) of a part of a row.  The sum is 0
// for a part with nothing but -inf, NaN if it holds a NaN.  The order in which
// parts join is fixed by the caller, so the result is too.
struct MaxSum {
    float m;
    float s;
};

// The reference point exp is taken from: the largest logit, 0 where there is none.
__device__ __forceinline__ float pivot(float m) { return m == -INFINITY ? 0.0f : m; }

// k = log2(e) / temperature: exp(z - z_max) = 2^((x - m) k).
__device__ __forceinline__ MaxSum join(MaxSum a, MaxSum b, float k)
{
    const float m = fmaxf(a.m, b.m), p = pivot(m);
    const float sa = __fmul_rn(a.s, exp2_fast(__fmul_rn(__fsub_rn(a.m, p), k)));
    const float sb = __fmul_rn(b.s, exp2_fast(__fmul_rn(__fsub_rn(b.m, p), k)));
    return MaxSum{m, __fadd_rn(sa, sb)};
}

// log p of a logit x: (x - m) / temperature - log s, with log s split into its
// exponent's and its mantissa's part so that the large terms cancel exactly:
// the error stays near the result's own ulp instead of that of the
// log-sum-exp (ten times larger at a vocabulary of 50 thousand).
__device__ __forceinline__ float log_prob(float x, MaxSum row, float inv_temperature)
{
    const int bits = __float_as_int(row.s);
    const int e = (bits >> 23) - 127;                    // s >= 1 (the largest logit's own term) or NaN
    const float f = __int_as_float((bits & 0x007fffff) | 0x3f800000);
    float d = __fmul_rn(__fsub_rn(x, row.m), inv_temperature);
    if (!(row.s < INFINITY)) return __fadd_rn(d, row.s); // NaN
    d = __fmaf_rn(static_cast<float>(-e), kLn2Hi, d);
    d = __fmaf_rn(static_cast<float>(-e), kLn2Lo, d);
    return __fsub_rn(d, logf(f));
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
    const float u = __fmul_rn(r, advantage);
    const float c = __fmul_rn(fminf(fmaxf(r, __fsub_rn(1.0f, clip_low)), __fadd_rn(1.0f, clip_high)), advantage);
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
        loss = __fmaf_rn(kl_coef, out.kl, loss);
        slope = __fmaf_rn(kl_coef, -em1, slope);
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
    float scale;     // -coef / sum: dlogits[j] = scale * 2^((x - m) k) + (j == label) coef
    float coef;
    int active;
};

// ---------------------------------------------------------------------------
// Rows too long for a cluster's shared memory: one block per row, three walks
// over it in global memory.
// ---------------------------------------------------------------------------
constexpr int kRowThreads = 256;

// Joins the threads' parts; every thread receives the same result.
__device__ __forceinline__ MaxSum block_join(MaxSum x, float k, MaxSum *shared)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const MaxSum y{__shfl_xor_sync(0xffffffffu, x.m, o), __shfl_xor_sync(0xffffffffu, x.s, o)};
        x = join(x, y, k);
    }
    __syncthreads();
    if (threadIdx.x % 32 == 0) shared[threadIdx.x / 32] = x;
    __syncthreads();
    x = shared[0];
    for (int w = 1; w < static_cast<int>(blockDim.x) / 32; ++w) x = join(x, shared[w], k);
    return x;
}

template <typename G> __device__ MaxSum row_stats(const RowArgs &a, int64_t t, MaxSum *shared)
{
    const float k = __fmul_rn(a.inv_temperature, kLog2e);
    const char *row = static_cast<const char *>(a.logits) + t * a.ld * G::kBytes;
    MaxSum x{-INFINITY, 0.0f};
    for (int64_t j = threadIdx.x; j < a.vocab; j += blockDim.x) x.m = fmaxf(x.m, load_value<G>(row, j));
    const float p = pivot(x.m);
    for (int64_t j = threadIdx.x; j < a.vocab; j += blockDim.x)
        x.s = __fadd_rn(x.s, exp2_fast(__fmul_rn(__fsub_rn(load_value<G>(row, j), p), k)));
    return block_join(x, k, shared);
}

template <typename G>
__device__ void row_gradient(const RowArgs &a, int64_t t, const RowFactors &f, int64_t label, void *dlogits, int64_t ld)
{
    const float k = __fmul_rn(a.inv_temperature, kLog2e);
    const char *src = static_cast<const char *>(a.logits) + t * a.ld * G::kBytes;
    char *dst = static_cast<char *>(dlogits) + t * ld * G::kBytes;
    for (int64_t j = threadIdx.x; j < a.vocab; j += blockDim.x) {
        float g = __fmul_rn(f.scale, exp2_fast(__fmul_rn(__fsub_rn(load_value<G>(src, j), f.m), k)));
        if (j == label) g = __fadd_rn(g, f.coef);
        store_value<G>(dst, j, g);
    }
}

template <typename G> __device__ void row_zero(const RowArgs &a, int64_t t, void *dlogits, int64_t ld)
{
    char *dst = static_cast<char *>(dlogits) + t * ld * G::kBytes;
    for (int64_t j = threadIdx.x; j < a.vocab; j += blockDim.x) store_value<G>(dst, j, 0.0f);
}


// The factors that the first block of the cluster left at this place of its memory.
__device__ __forceinline__ RowFactors peer_factors(uint32_t at)
{
    RowFactors f;
    asm volatile("ld.shared::cluster.v4.b32 {%0, %1, %2, %3}, [%4];"
                 : "=f"(f.m), "=f"(f.scale), "=f"(f.coef), "=r"(f.active) : "r"(peer_address(at, 0)) : "memory");
    return f;
}

struct RowSums {
    double loss = 0.0, gain = 0.0, kl = 0.0, clipped = 0.0;
};

template <bool POLICY>
__device__ __forceinline__ RowFactors finish_row(const RowWork &a, int64_t t, bool wanted, MaxSum row, float weight,
                                                 float label_logit, float advantage, float old_lp, float ref_lp, RowSums *sums)
{
    const bool active = wanted && !(row.s == 0.0f);
    const float inv_t = a.row.inv_temperature;
    float lp = 0.0f;
    PolicyRow r{0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
    if (active) lp = log_prob(label_logit, row, inv_t);
    if (a.logp) a.logp[t] = lp;
    if constexpr (POLICY) {
        if (active) {
            r = policy_row(lp, advantage, a.old_logp != nullptr, old_lp, a.ref_logp != nullptr, ref_lp, a.clip_low, a.clip_high,
                           a.kl_coef, weight, inv_t);
            sums->loss += static_cast<double>(weight) * r.loss;
            sums->gain -= static_cast<double>(weight) * r.gain;
            sums->kl += static_cast<double>(weight) * r.kl;
            sums->clipped += static_cast<double>(weight) * r.clipped;
        }
        a.token_loss[t] = r.loss;
    } else {
        if (a.lse) a.lse[t] = active ? log_sum_exp(row, inv_t) : 0.0f;
        if (a.kept) a.kept[t] = RowKept{row.m, active ? __fdiv_rn(1.0f, row.s) : 0.0f, lp, 0.0f};
    }
    return RowFactors{row.m, active ? __fdiv_rn(-r.coef, row.s) : 0.0f, r.coef, active ? 1 : 0};
}

template <bool POLICY> __device__ __forceinline__ void store_partial(const RowWork &a, int64_t at, const RowSums &sums)
{
    if constexpr (POLICY)
        a.partial[at] = make_float4(static_cast<float>(sums.loss), static_cast<float>(sums.gain), static_cast<float>(sums.kl),
                                    static_cast<float>(sums.clipped));
}

template <typename G, bool POLICY> __global__ void __launch_bounds__(kRowThreads) star_long_row_kernel(const __grid_constant__ RowWork a)
{
    __shared__ MaxSum shared[kRowThreads / 32];
    __shared__ RowFactors factors;
    RowSums sums;
    for (int64_t t = blockIdx.x; t < a.row.rows; t += gridDim.x) {
        int64_t label;
        float weight;
        const bool wanted = row_wanted(a.row, t, &label, &weight);
        MaxSum row{0.0f, 0.0f};
        if (wanted) row = row_stats<G>(a.row, t, shared);
        if (threadIdx.x == 0) {
            const float x = wanted ? load_value<G>(static_cast<const char *>(a.row.logits) + t * a.row.ld * G::kBytes, label) : 0.0f;
            factors = finish_row<POLICY>(a, t, wanted, row, weight, x, POLICY && wanted ? a.advantages[t] : 0.0f,
                                         POLICY && a.old_logp ? a.old_logp[t] : 0.0f, POLICY && a.ref_logp ? a.ref_logp[t] : 0.0f, &sums);
        }
        __syncthreads();
        const RowFactors f = factors;
        if (POLICY && a.dlogits) {
            if (f.active)
                row_gradient<G>(a.row, t, f, label, a.dlogits, a.ld_dlogits);
            else
                row_zero<G>(a.row, t, a.dlogits, a.ld_dlogits);
        }
        __syncthreads();
    }
    if (threadIdx.x == 0) store_partial<POLICY>(a, blockIdx.x, sums);
}

// ---------------------------------------------------------------------------
// Rows that stay in shared memory: read once, written once.
//
// A cluster of 1 to 8 blocks holds a row, each block a run of its 16-byte pieces
// ("granules", on the 16-byte grid of global memory, so that copies and stores
// are whole whatever the row's phase; the up to 15 bytes before and after them
// are single elements of the first block).  The block walks rows with a stride,
// STAGES - 1 rows ahead in flight by asynchronous copies: first walk of a row in
// shared memory: running maximum and sum of every thread; they join through
// warps, block and cluster; one thread makes the row's scalars; second walk: the
// gradient, from shared memory to global memory.
// ---------------------------------------------------------------------------
__device__ __forceinline__ void copy_async(uint32_t dst, const void *src)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" :: "r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" :: "n"(N) : "memory"); }

__device__ __forceinline__ float warp_max(float x)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, o));
    return x;
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
    return MaxSum{m, warp_sum(__fmul_rn(x.s, exp2_fast(__fmul_rn(__fsub_rn(x.m, pivot(m)), k))))};
}

template <typename G> struct Granule {
    static constexpr int kCount = 16 / G::kBytes;                // elements
    static __device__ __forceinline__ void widen(const uint4 &v, float (&f)[kCount])
    {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
        if constexpr (G::kBytes == 2) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                f[2 * e] = __uint_as_float(w[e] << 16);
                f[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
            }
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) f[e] = __uint_as_float(w[e]);
        }
    }
    static __device__ __forceinline__ uint4 narrow(const float (&f)[kCount])
    {
        if constexpr (G::kBytes == 2)
            return make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
        else
            return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
    }
};

// Adds values to a thread's running maximum and sum.
template <int N> __device__ __forceinline__ void absorb(MaxSum *x, const float (&f)[N], float k)
{
    float m = f[0];
#pragma unroll
    for (int e = 1; e < N; ++e) m = fmaxf(m, f[e]);
    if (m > x->m) {
        x->s = __fmul_rn(x->s, exp2_fast(__fmul_rn(__fsub_rn(x->m, m), k)));
        x->m = m;
    }
    const float p = pivot(x->m);
    float e2[N];
#pragma unroll
    for (int e = 0; e < N; ++e) e2[e] = exp2_fast(__fmul_rn(__fsub_rn(f[e], p), k));
#pragma unroll
    for (int o = N / 2; o > 0; o >>= 1)
#pragma unroll
        for (int e = 0; e < o; ++e) e2[e] = __fadd_rn(e2[e], e2[e + o]);
    x->s = __fadd_rn(x->s, e2[0]);
}

// How a row's elements fall on the 16-byte grid.
struct RowSplit {
    int head;        // elements before the first granule
    int granules;
    int tail;        // elements after the last
};
template <typename G> __device__ __forceinline__ RowSplit split_row(uintptr_t address, int64_t vocab)
{
    constexpr int E = Granule<G>::kCount;
    const int to_grid = static_cast<int>((16 - address % 16) % 16) / G::kBytes;
    RowSplit r;
    r.head = static_cast<int>(min(static_cast<int64_t>(to_grid), vocab));
    r.granules = static_cast<int>((vocab - r.head) / E);
    r.tail = static_cast<int>((vocab - r.head) % E);
    return r;
}

template <typename G, bool POLICY, int THREADS, int STAGES>
__global__ void __launch_bounds__(THREADS) star_row_kernel(const __grid_constant__ RowWork a)
{
    constexpr int E = Granule<G>::kCount, kWarps = THREADS / 32;
    extern __shared__ uint4 ring[];                              // [STAGES][a.granules]
    __shared__ MaxSum warp_part[2][kWarps];
    __shared__ alignas(8) MaxSum block_part[2][8];
    __shared__ RowFactors shared_factors;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const uint32_t blocks = cluster_size(), rank = cluster_rank();
    const int64_t first = blockIdx.x / blocks, step = gridDim.x / blocks;
    const float k = __fmul_rn(a.row.inv_temperature, kLog2e);
    const int64_t rows = a.row.rows, vocab = a.row.vocab;
    const bool writes = POLICY && a.dlogits != nullptr;
    launch_dependents();

    // What is known of a row before it is worked on.
    struct Row {
        int64_t label = -1;
        float weight = 0.0f;
        bool wanted = false;
        float edge = 0.0f;               // this thread's element outside the granules (first block)
        float label_logit = 0.0f, advantage = 0.0f, old_lp = 0.0f, ref_lp = 0.0f;      // thread 0
    };
    const auto row_base = [&](int64_t t) { return static_cast<const char *>(a.row.logits) + t * a.row.ld * G::kBytes; };
    const auto look_up = [&](int64_t t) {
        Row r;
        if (t < rows) r.wanted = row_wanted(a.row, t, &r.label, &r.weight);
        return r;
    };
    // Granules [begin, end) of a row are this block's.
    const auto share = [&](const RowSplit &s, int *begin, int *end) {
        const int each = (s.granules + static_cast<int>(blocks) - 1) / static_cast<int>(blocks);
        *begin = min(each * static_cast<int>(rank), s.granules);
        *end = min(*begin + each, s.granules);
    };
    // The element of the row that thread `threadIdx.x` of the first block takes beside the granules, or -1.
    const auto edge_at = [&](const RowSplit &s) -> int64_t {
        const int i = threadIdx.x;
        if (rank != 0 || i >= s.head + s.tail) return -1;
        return i < s.head ? i : vocab - s.tail + (i - s.head);
    };
    const auto fetch = [&](int64_t t, int stage, Row *r) {
        if (r->wanted) {
            const char *base = row_base(t);
            const RowSplit s = split_row<G>(reinterpret_cast<uintptr_t>(base), vocab);
            int begin, end;
            share(s, &begin, &end);
            const char *src = base + s.head * G::kBytes;
            const uint32_t dst = smem_address(ring) + static_cast<uint32_t>(stage * a.granules) * 16;
            for (int i = begin + threadIdx.x; i < end; i += THREADS) copy_async(dst + (i - begin) * 16, src + static_cast<int64_t>(i) * 16);
            const int64_t at = edge_at(s);
            if (at >= 0) r->edge = load_value<G>(base, at);
            if (threadIdx.x == 0) {
                r->label_logit = load_value<G>(base, r->label);
                if constexpr (POLICY) {
                    r->advantage = a.advantages[t];
                    if (a.old_logp) r->old_lp = a.old_logp[t];
                    if (a.ref_logp) r->ref_lp = a.ref_logp[t];
                }
            }
        }
        copy_commit();
    };

    RowSums sums;
    Row row[STAGES];                     // row[0]: the current one, then those in flight
#pragma unroll
    for (int i = 0; i < STAGES; ++i) row[i] = look_up(first + i * step);
#pragma unroll
    for (int i = 0; i + 1 < STAGES; ++i) fetch(first + i * step, i, &row[i]);
    int stage = 0, parity = 0;
    for (int64_t t = first; t < rows; t += step) {
        copy_wait<STAGES - 2>();
        __syncthreads();                                         // this row's copies are in place; the stage of the row before is free
        fetch(t + (STAGES - 1) * step, stage == 0 ? STAGES - 1 : stage - 1, &row[STAGES - 1]);
        const Row next = look_up(t + STAGES * step);
        const Row cur = row[0];

        const char *base = row_base(t);
        const RowSplit s = split_row<G>(reinterpret_cast<uintptr_t>(base), vocab);
        int begin, end;
        share(s, &begin, &end);
        const uint4 *mine = ring + stage * a.granules;
        const int count = end - begin;
        MaxSum x{-INFINITY, 0.0f};
        if (cur.wanted) {
#pragma unroll 2
            for (int i = threadIdx.x; i < count; i += THREADS) {
                float f[E];
                Granule<G>::widen(mine[i], f);
                absorb<E>(&x, f, k);
            }
            if (edge_at(s) >= 0) {
                const float f[1] = {cur.edge};
                absorb<1>(&x, f, k);
            }
            x = warp_join(x, k);
            if (lane == 0) warp_part[parity][warp] = x;
        }
        __syncthreads();
        if (warp == 0 && cur.wanted) {
            x = lane < kWarps ? warp_part[parity][lane] : MaxSum{-INFINITY, 0.0f};
            x = warp_join(x, k);
        }
        if (blocks > 1) {
            if (warp == 0 && lane < static_cast<int>(blocks)) {
                const uint32_t at = peer_address(smem_address(&block_part[parity][rank]), lane);
                asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" :: "r"(at), "f"(x.m), "f"(x.s) : "memory");
            }
            cluster_sync();
            if (warp == 0) {
                x = lane < static_cast<int>(blocks) ? block_part[parity][lane] : MaxSum{-INFINITY, 0.0f};
                x = warp_join(x, k);
            }
        }
        if (threadIdx.x == 0) {
            if (rank == 0) {
                const RowFactors f = finish_row<POLICY>(a, t, cur.wanted, x, cur.weight, cur.label_logit, cur.advantage, cur.old_lp,
                                                        cur.ref_lp, &sums);
                shared_factors = f;
            }
        }
        if (writes) {
            __syncthreads();
            if (blocks > 1) {
                // The first block's thread made the factors; its peers read them.
                cluster_sync();
            }
            const RowFactors f = blocks > 1 ? peer_factors(smem_address(&shared_factors)) : shared_factors;
            char *out = static_cast<char *>(a.dlogits) + t * a.ld_dlogits * G::kBytes;
            const bool same_phase = (reinterpret_cast<uintptr_t>(out) - reinterpret_cast<uintptr_t>(base)) % 16 == 0;
            const int64_t start = s.head + static_cast<int64_t>(begin) * E;          // this block's first element in the granules
            const int64_t at_label = f.active ? cur.label - start : -1;              // relative to it
            if (same_phase) {
                uint4 *dst = reinterpret_cast<uint4 *>(out + start * G::kBytes);
                if (f.active) {
#pragma unroll 2
                    for (int i = threadIdx.x; i < count; i += THREADS) {
                        float g[E];
                        Granule<G>::widen(mine[i], g);
#pragma unroll
                        for (int e = 0; e < E; ++e) g[e] = __fmul_rn(f.scale, exp2_fast(__fmul_rn(__fsub_rn(g[e], f.m), k)));
                        dst[i] = Granule<G>::narrow(g);
                    }
                    // The label's element again, by the thread that stored its granule.
                    if (at_label >= 0 && at_label < static_cast<int64_t>(count) * E && static_cast<int>(at_label) / E % THREADS == static_cast<int>(threadIdx.x)) {
                        const float y = exp2_fast(__fmul_rn(__fsub_rn(load_value<G>(mine, at_label), f.m), k));
                        store_value<G>(dst, at_label, __fadd_rn(__fmul_rn(f.scale, y), f.coef));
                    }
                } else {
                    for (int i = threadIdx.x; i < count; i += THREADS) dst[i] = make_uint4(0, 0, 0, 0);
                }
            } else {
                const int64_t n = static_cast<int64_t>(count) * E;
                for (int64_t i = threadIdx.x; i < n; i += THREADS) {
                    float g = 0.0f;
                    if (f.active) {
                        g = __fmul_rn(f.scale, exp2_fast(__fmul_rn(__fsub_rn(load_value<G>(mine, i), f.m), k)));
                        if (i == at_label) g = __fadd_rn(g, f.coef);
                    }
                    store_value<G>(out, start + i, g);
                }
            }
            const int64_t at = edge_at(s);
            if (at >= 0) {
                float g = 0.0f;
                if (f.active) {
                    g = __fmul_rn(f.scale, exp2_fast(__fmul_rn(__fsub_rn(cur.edge, f.m), k)));
                    if (at == cur.label) g = __fadd_rn(g, f.coef);
                }
                store_value<G>(out, at, g);
            }
        }
#pragma unroll
        for (int i = 0; i + 1 < STAGES; ++i) row[i] = row[i + 1];
        row[STAGES - 1] = next;
        stage = stage + 1 == STAGES ? 0 : stage + 1;
        parity ^= 1;
    }
    copy_wait<0>();
    if (threadIdx.x == 0 && rank == 0) store_partial<POLICY>(a, first, sums);
    if (blocks > 1) cluster_sync();                              // nobody leaves while a peer reads its memory
}

constexpr int kSumThreads = 256;

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

// sums[0 .. 4) from the clusters' parts, one block.
__global__ void __launch_bounds__(kSumThreads) star_policy_sums_kernel(const float4 *terms, int64_t n, float *sums)
{
    __shared__ double shared[kSumThreads / 32];
    wait_for_primary();
    double s[4] = {0.0, 0.0, 0.0, 0.0};
    for (int64_t i = threadIdx.x; i < n; i += kSumThreads) {
        const float4 x = terms[i];
        s[0] += x.x; s[1] += x.y; s[2] += x.z; s[3] += x.w;
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const double total = block_sum(s[q], shared);
        if (threadIdx.x == 0) sums[q] = static_cast<float>(total);
    }
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
__device__ __forceinline__ void preference_total(const PreferenceArgs &a, double *shared)
{
    double s = 0.0;
    for (int64_t i = threadIdx.x; i < a.pairs; i += blockDim.x) s += a.pair_loss[i];
    s = block_sum(s, shared);
    if (threadIdx.x == 0) a.loss[0] = static_cast<float>(s * a.loss_scale);
}

__global__ void __launch_bounds__(kPairThreads) star_preference_total_kernel(const __grid_constant__ PreferenceArgs a)
{
    __shared__ double shared[kPairThreads / 32];
    wait_for_primary();
    preference_total(a, shared);
}

// The gradient, straight from global memory: a second reading of the logits,
// because a row's factor needs every row of its pair.  Rows are taken from the
// last to the first, so that those read last by the first step are still in L2.
// An item is a run of kGradGranules granules of a row.
constexpr int kGradPerThread = 4;
constexpr int kGradGranules = kRowThreads * kGradPerThread;

template <typename G> __global__ void __launch_bounds__(kRowThreads, 4) star_preference_grad_kernel(const __grid_constant__ PreferenceArgs a)
{
    constexpr int E = Granule<G>::kCount;
    __shared__ double shared[kRowThreads / 32];
    wait_for_primary();
    if (blockIdx.x == 0) preference_total(a, shared);
    const float k = __fmul_rn(a.row.inv_temperature, kLog2e);
    const int64_t per_row = (a.row.vocab / E + kGradGranules) / kGradGranules;           // the last run may be empty
    const int64_t items = a.row.rows * per_row;
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const int64_t t = a.row.rows - 1 - item / per_row, run = item % per_row;
        const RowKept r = a.kept[t];
        const bool active = r.inv_s != 0.0f && r.coef != 0.0f;
        const char *base = static_cast<const char *>(a.row.logits) + t * a.row.ld * G::kBytes;
        char *out = static_cast<char *>(a.dlogits) + t * a.ld_dlogits * G::kBytes;
        const RowSplit s = split_row<G>(reinterpret_cast<uintptr_t>(base), a.row.vocab);
        const int64_t label = active ? a.row.labels[t] : -1;
        const float scale = __fmul_rn(-r.coef, r.inv_s);
        const auto grad = [&](float x, int64_t at) {
            const float g = __fmul_rn(scale, exp2_fast(__fmul_rn(__fsub_rn(x, r.m), k)));
            return at == label ? __fadd_rn(g, r.coef) : g;
        };
        const bool same_phase = (reinterpret_cast<uintptr_t>(out) - reinterpret_cast<uintptr_t>(base)) % 16 == 0;
        const int begin = static_cast<int>(run) * kGradGranules, end = min(begin + kGradGranules, s.granules);
        if (same_phase) {
            const uint4 *src = reinterpret_cast<const uint4 *>(base + s.head * G::kBytes);
            uint4 *dst = reinterpret_cast<uint4 *>(out + s.head * G::kBytes);
            if (active) {
                uint4 v[kGradPerThread];
#pragma unroll
                for (int q = 0; q < kGradPerThread; ++q) {
                    const int i = begin + q * kRowThreads + static_cast<int>(threadIdx.x);
                    if (i < end) v[q] = src[i];
                }
                const int64_t at_label = label - s.head;
                const bool label_here = at_label >= static_cast<int64_t>(begin) * E && at_label < static_cast<int64_t>(end) * E &&
                                        (at_label / E - begin) % kRowThreads == threadIdx.x;
                const float label_logit = label_here ? load_value<G>(src, at_label) : 0.0f;      // before an in-place store
#pragma unroll
                for (int q = 0; q < kGradPerThread; ++q) {
                    const int i = begin + q * kRowThreads + static_cast<int>(threadIdx.x);
                    if (i < end) {
                        float g[E];
                        Granule<G>::widen(v[q], g);
#pragma unroll
                        for (int e = 0; e < E; ++e) g[e] = __fmul_rn(scale, exp2_fast(__fmul_rn(__fsub_rn(g[e], r.m), k)));
                        dst[i] = Granule<G>::narrow(g);
                    }
                }
                if (label_here) store_value<G>(dst, at_label, grad(label_logit, label));         // by the thread that stored its granule
            } else {
                for (int i = begin + threadIdx.x; i < end; i += kRowThreads) dst[i] = make_uint4(0, 0, 0, 0);
            }
        } else {
            const int64_t last = s.head + static_cast<int64_t>(end) * E;
            for (int64_t at = s.head + static_cast<int64_t>(begin) * E + threadIdx.x; at < last; at += kRowThreads)
                store_value<G>(out, at, active ? grad(load_value<G>(base, at), at) : 0.0f);
        }
        if (run == 0 && static_cast<int>(threadIdx.x) < s.head + s.tail) {
            const int i = threadIdx.x;
            const int64_t at = i < s.head ? i : a.row.vocab - s.tail + (i - s.head);
            store_value<G>(out, at, active ? grad(load_value<G>(base, at), at) : 0.0f);
        }
    }
}

}  // namespace star
