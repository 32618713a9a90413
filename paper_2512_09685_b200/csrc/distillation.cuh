// Device code of the distillation loss (sm_100a).
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "rows.cuh"

namespace star {

constexpr int kMostListed = 128;             // STAR_MAX_ALTERNATIVES

struct DistillArgs {
    RowArgs row;                 // labels may be null
    const int32_t *ids;          // of the teacher's list
    const float *values;
    int64_t ld_ids, ld_values;
    int k;
    int rest;
    float inv_teacher_temperature;
    float soft, hard;
    float *token_loss;
    float4 *partial;             // the four sums of each block's (cluster's) rows
    void *dlogits;               // may be null
    int64_t ld_dlogits;
    int tries;                   // of a wait
};

// Statistics of the elements that the teacher does not list: the largest, the sum of
// 2^exponent at the loss's temperature, and at temperature 1 where that is another.
struct RestSums {
    float m, s, s1;
};

// What a row's results and gradient are made of.
struct alignas(16) DistillFactors {
    float m_rest;        // the largest element that is not listed
    float rest, rest1;   // dlogits[j] = rest 2^exponent(x, m_rest) + rest1 2^exponent1(x, m_rest)
    float m, s, s1;      // of the whole row
    float shift, log_sum;        // of the teacher's list
    float mass;          // what the teacher's probabilities that count add up to
    float soft, hard;    // weight and coefficients in front of the gradient's parts
    int active;
    int late;            // a wait for the row ran out: nothing of it holds
};

struct DistillSums {
    double loss, kl, ce, weight;
};

// q log(q / p) - q + p, which is never negative; d = log(p / q).  Without the
// cancellation where the two are near.
__device__ __forceinline__ float divergence(float q, float p, float d)
{
    if (q == 0.0f) return p;
    if (fabsf(d) < 1.0f) return __fmul_rn(q, __fsub_rn(expm1f(d), d));
    return __fsub_rn(__fsub_rn(p, q), __fmul_rn(q, d));
}

// A teacher's list of one row, in shared memory.
struct Listed {
    int id[kMostListed];         // -1: absent
    float value[kMostListed];
    float x[kMostListed];        // the student's logit
    int first[kMostListed];      // no entry in front has this id
};

// The same sum in every thread of a warp; NaNs stay.
__device__ __forceinline__ double warp_sum_wide(double x)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

// What makes log-probabilities of the teacher's values v: (v - shift) / temperature -
// log_sum, the difference first, as for the student's.  By a warp.  log_sum = -inf:
// nothing is listed.
struct Normalizer {
    float shift, log_sum;
};
__device__ __forceinline__ Normalizer list_normalizer(const DistillArgs &a, const Listed &list)
{
    if (a.rest) return Normalizer{0.0f, 0.0f};                   // log-probabilities already
    const int lane = threadIdx.x % 32;
    float v[kMostListed / 32], most = -INFINITY;
    bool bad = false;
#pragma unroll
    for (int q = 0; q < kMostListed / 32; ++q) {
        const int i = q * 32 + lane;
        v[q] = i < a.k && list.id[i] >= 0 ? list.value[i] : -INFINITY;
        bad |= v[q] != v[q];
        most = fmaxf(most, v[q]);
    }
    most = warp_max(most);
    if (__any_sync(0xffffffffu, bad) || most == INFINITY) return Normalizer{0.0f, NAN};
    if (most == -INFINITY) return Normalizer{0.0f, -INFINITY};
    float s = 0.0f;
#pragma unroll
    for (int q = 0; q < kMostListed / 32; ++q) s = __fadd_rn(s, expf(__fmul_rn(__fsub_rn(v[q], most), a.inv_teacher_temperature)));
    return Normalizer{most, logf(warp_sum(s))};
}
__device__ __forceinline__ float listed_log(const DistillArgs &a, float v, float shift, float log_sum)
{
    return log_sum == -INFINITY ? -INFINITY : __fsub_rn(__fmul_rn(__fsub_rn(v, shift), a.inv_teacher_temperature), log_sum);
}

// A row's factors and results from its statistics and its list, by a warp.
__device__ __forceinline__ DistillFactors distill_row(const DistillArgs &a, const Listed &list, RestSums rest, bool wanted, float weight,
                                                      float label_logit, Normalizer teacher, float *kl_out, float *ce_out)
{
    const int lane = threadIdx.x % 32;
    const float inv_t = a.row.inv_temperature, k = __fmul_rn(inv_t, kLog2e);
    const bool two = a.hard != 0.0f && inv_t != 1.0f;
    DistillFactors f{};
    f.shift = teacher.shift;
    f.log_sum = teacher.log_sum;
    f.m_rest = rest.m;
    // The listed elements join the rest: an element once, however often it is listed.
    float x[kMostListed / 32], most = rest.m;
    bool present[kMostListed / 32], first[kMostListed / 32];
#pragma unroll
    for (int q = 0; q < kMostListed / 32; ++q) {
        const int i = q * 32 + lane;
        present[q] = i < a.k && list.id[i] >= 0;
        first[q] = present[q] && list.first[i];
        x[q] = present[q] ? list.x[i] : -INFINITY;
        most = fmaxf(most, x[q]);
    }
    f.m = warp_max(most);
    float s = 0.0f, s1 = 0.0f;
#pragma unroll
    for (int q = 0; q < kMostListed / 32; ++q) {
        if (first[q]) {
            s = __fadd_rn(s, exp2_fast(exponent(x[q], f.m, k)));
            if (two) s1 = __fadd_rn(s1, exp2_fast(exponent(x[q], f.m, kLog2e)));
        }
    }
    const float down = rest.s == 0.0f ? 0.0f : rebase(rest.m, f.m, k);
    const float rest_s = __fmul_rn(rest.s, down);                // what is not listed, at the row's reference
    f.s = __fadd_rn(warp_sum(s), rest_s);
    float down1 = 0.0f;
    if (two) {
        down1 = rest.s == 0.0f ? 0.0f : rebase(rest.m, f.m, kLog2e);
        f.s1 = __fadd_rn(warp_sum(s1), __fmul_rn(rest.s1, down1));
    }
    f.active = wanted && !(f.s == 0.0f) ? 1 : 0;
    *kl_out = *ce_out = 0.0f;
    if (!f.active) return f;
    const MaxSum row{f.m, f.s};
    // sum q log(q / p) as a sum of terms of one sign.  They add up to it if both
    // distributions add up to 1; what they do not is put right at the end.
    float terms = 0.0f, again = 0.0f;
    double mass = 0.0;
#pragma unroll
    for (int q = 0; q < kMostListed / 32; ++q) {
        if (present[q]) {
            const float log_q = listed_log(a, list.value[q * 32 + lane], f.shift, f.log_sum), prob = expf(log_q);
            const float log_p = log_prob(x[q], row, k, inv_t), p = expf(log_p);
            mass += prob;
            terms = __fadd_rn(terms, divergence(prob, p, __fsub_rn(log_p, log_q)));
            if (!first[q]) again = __fadd_rn(again, p);
        }
    }
    terms = warp_sum(terms);
    again = warp_sum(again);
    mass = warp_sum_wide(mass);
    const float p0 = __fdiv_rn(rest_s, f.s);
    float q0 = 0.0f, off;                                        // off: by how much the teacher's probabilities miss 1
    if (a.rest) {
        const double left = 1.0 - mass;
        q0 = left > 0.0 && rest.s > 0.0f ? static_cast<float>(left) : 0.0f;
        off = q0 > 0.0f ? 0.0f : static_cast<float>(-left);
        f.mass = q0 > 0.0f ? 1.0f : static_cast<float>(mass);
        if (mass != mass) f.mass = off = NAN;
    } else {
        f.mass = f.log_sum == -INFINITY ? 0.0f : f.log_sum != f.log_sum ? f.log_sum : 1.0f;
        off = __fsub_rn(f.mass, 1.0f);
    }
    // log p0 by its parts: it exists where p0 itself is below binary32.
    const float log_p0 = __fadd_rn(log_prob(rest.m, row, k, inv_t), logf(rest.s));
    terms = __fadd_rn(terms, divergence(q0, p0, q0 > 0.0f ? __fsub_rn(log_p0, logf(q0)) : 0.0f));
    const float kl = __fadd_rn(__fsub_rn(terms, again), off);
    *kl_out = kl;
    if (a.hard != 0.0f) *ce_out = -(two ? log_prob(label_logit, MaxSum{f.m, f.s1}, kLog2e, 1.0f) : log_prob(label_logit, row, k, inv_t));
    // The gradient's factors.
    f.soft = __fmul_rn(__fmul_rn(weight, a.soft), inv_t);
    f.hard = __fmul_rn(weight, a.hard);
    float scale = 0.0f;
    if (a.soft != 0.0f) {
        scale = __fdiv_rn(__fmul_rn(f.mass, down), f.s);
        if (q0 > 0.0f) scale = __fdiv_rn(__fsub_rn(__fmul_rn(f.mass, p0), q0), rest.s);
        scale = __fmul_rn(f.soft, scale);
    }
    if (a.hard != 0.0f) {
        if (two)
            f.rest1 = __fmul_rn(f.hard, __fdiv_rn(down1, f.s1));
        else
            scale = __fmaf_rn(f.hard, __fdiv_rn(down, f.s), scale);
    }
    f.rest = scale;
    return f;
}

// As take_batch, with the sum at temperature 1 where TWO.
template <typename G, int N, int THREADS, bool FULL, bool TWO>
__device__ __forceinline__ void take_rest(RestSums *x, const uint4 *from, int left, float k)
{
    if constexpr (!TWO) {
        MaxSum y{x->m, x->s};
        take_batch<G, N, THREADS, FULL>(&y, from, left, k);
        x->m = y.m;
        x->s = y.s;
    } else {
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
            x->s1 = __fmul_rn(x->s1, exp2_fast(exponent(x->m, m, kLog2e)));
            x->m = m;
        }
        const Pair minus_m = pair_of(-pivot(x->m)), kk = pair_of(k), k1 = pair_of(kLog2e);
        Pair s = pair_of(0.0f), s1 = pair_of(0.0f);
#pragma unroll
        for (int q = 0; q < N; ++q) {
            if (FULL || q * THREADS < left) {
                Pair f[P];
                Granule<G>::widen(v[q], f);
#pragma unroll
                for (int e = 0; e < P; ++e) {
                    const Pair d = pair_add(f[e], minus_m);
                    s = pair_add(s, pair_exp2(pair_mul(d, kk)));
                    s1 = pair_add(s1, pair_exp2(pair_mul(d, k1)));
                }
            }
        }
        float lo, hi;
        split_pair(s, &lo, &hi);
        x->s = __fadd_rn(x->s, __fadd_rn(lo, hi));
        split_pair(s1, &lo, &hi);
        x->s1 = __fadd_rn(x->s1, __fadd_rn(lo, hi));
    }
}
__device__ __forceinline__ RestSums rest_move(RestSums x, float m, float k)
{
    return RestSums{m, __fmul_rn(x.s, rebase(x.m, m, k)), __fmul_rn(x.s1, rebase(x.m, m, kLog2e))};
}
__device__ __forceinline__ RestSums warp_join(RestSums x, float k)
{
    x = rest_move(x, warp_max(x.m), k);
    return RestSums{x.m, warp_sum(x.s), warp_sum(x.s1)};
}
__device__ __forceinline__ RestSums take_one(RestSums x, float v, float k)
{
    const float m = fmaxf(x.m, v);
    x = rest_move(x, m, k);
    return RestSums{m, __fadd_rn(x.s, exp2_fast(exponent(v, m, k))), __fadd_rn(x.s1, exp2_fast(exponent(v, m, kLog2e)))};
}

// The gradient of an element that is not listed.
template <bool TWO> __device__ __forceinline__ float rest_gradient(float x, const DistillFactors &f, float k)
{
    const float g = __fmul_rn(f.rest, exp2_fast(exponent(x, f.m_rest, k)));
    return TWO ? __fmaf_rn(f.rest1, exp2_fast(exponent(x, f.m_rest, kLog2e)), g) : g;
}
template <typename G, int N, int THREADS, bool FULL>
__device__ __forceinline__ void store_two(uint4 *to, const uint4 *from, int left, const DistillFactors &f, float k)
{
    constexpr int P = Granule<G>::kPairs;
    const Pair minus_m = pair_of(-pivot(f.m_rest)), kk = pair_of(k), k1 = pair_of(kLog2e), a = pair_of(f.rest), b = pair_of(f.rest1);
#pragma unroll
    for (int q = 0; q < N; ++q) {
        if (FULL || q * THREADS < left) {
            Pair g[P];
            Granule<G>::widen(from[q * THREADS], g);
#pragma unroll
            for (int e = 0; e < P; ++e) {
                const Pair d = pair_add(g[e], minus_m);
                g[e] = pair_fma(b, pair_exp2(pair_mul(d, k1)), pair_mul(a, pair_exp2(pair_mul(d, kk))));
            }
            to[q * THREADS] = Granule<G>::narrow(g);
        }
    }
}

// ---------------------------------------------------------------------------
// The loss with its gradient in one reading, arranged as the policy loss is: a row
// comes by one bulk copy and stays in shared memory from its statistics to its
// gradient; longer rows, and few, lie in the shared memory of a cluster's blocks.
//
// The probability of what is not listed has to be summed over just that: as 1 - the
// listed ones it would lose all digits where the student is sure of a listed token.
// So the listed elements' logits are read on their own, and -inf is written over
// them in shared memory: the statistics, and the gradient's walk, then see the rest
// alone.  The listed elements' gradients, and the label's, are stored after it.
// ---------------------------------------------------------------------------
constexpr int kDistillBytesPerThread = 208;  // shared memory for the row: 208 KB an SM

template <typename G, int THREADS, bool TWO>
__global__ void __launch_bounds__(THREADS, policy_blocks(THREADS)) star_distillation_kernel(const __grid_constant__ DistillArgs a)
{
    constexpr int E = Granule<G>::kCount, kWarps = THREADS / 32, kStep = kBatch * THREADS;
    static_assert(THREADS >= kMostListed, "a thread to a listed element");
    extern __shared__ uint4 kept_row[];
    __shared__ RestSums warp_part[kWarps];
    __shared__ RestSums block_part[2][8];
    __shared__ DistillFactors factors;
    __shared__ DistillSums sums;
    __shared__ Listed list;
    __shared__ Normalizer teacher;
    __shared__ float row_label_logit;
    __shared__ int edge_listed[32];
    __shared__ int late[2];                                      // of every other row, as in the policy loss
    __shared__ alignas(8) uint64_t landed;                       // the row's copy is in place
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const float k = __fmul_rn(a.row.inv_temperature, kLog2e);
    const int vocab = static_cast<int>(a.row.vocab);
    const uint32_t blocks = cluster_size(), rank = cluster_rank();
    const int log_blocks = 31 - __clz(static_cast<int>(blocks));
    const int64_t first_row = blockIdx.x >> log_blocks, step = gridDim.x >> log_blocks;
    launch_dependents();
    if (threadIdx.x == 0) {
        sums = DistillSums{0.0, 0.0, 0.0, 0.0};
        late[0] = late[1] = factors.late = 0;
        barrier_init(smem_address(&landed), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    if (blocks > 1) cluster_sync();                              // the others have started
    wait_for_primary();

    const auto row_base = [&](int64_t t) { return static_cast<const char *>(a.row.logits) + t * a.row.ld * G::kBytes; };
    // Whether a row takes part, as far as its label and weight say.
    const auto row_in = [&](int64_t t, int64_t *label, float *weight) {
        *label = a.row.labels ? a.row.labels[t] : 0;
        *weight = a.row.weights ? a.row.weights[t] : 1.0f;
        return *label >= 0 && *label < vocab && *weight != 0.0f;
    };
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
    // A thread's entry of row t's list.
    const auto entry = [&](int64_t t, int *id, float *value) {
        *id = -1;
        *value = 0.0f;
        if (static_cast<int>(threadIdx.x) < a.k) {
            const int given = a.ids[t * a.ld_ids + threadIdx.x];
            if (given >= 0 && given < vocab) *id = given;
            *value = a.values[t * a.ld_values + threadIdx.x];
        }
    };

    uint32_t phase = 0;
    int parity = 0;
    for (int64_t t = first_row; t < a.row.rows; t += step, parity ^= 1) {
        const char *base = row_base(t);
        const RowSplit s = split_row<G>(base, vocab);
        const RowShare own = row_share(s.granules, rank, log_blocks);
        int64_t label;
        float weight;
        const bool wanted = row_in(t, &label, &weight);
        if (wanted && threadIdx.x == 0) fetch(t);
        const int edge_at = rank == 0 ? edge_element(s, threadIdx.x, vocab) : -1;
        float edge = 0.0f, x_own = 0.0f, value_own = 0.0f;
        int id_own = -1;
        bool first_own = false;
        RestSums x{-INFINITY, 0.0f, 0.0f};
        if (wanted) {
            entry(t, &id_own, &value_own);
            if (id_own >= 0) x_own = load_value<G>(base, id_own);
            if (threadIdx.x < kMostListed) {
                list.id[threadIdx.x] = id_own;
                list.value[threadIdx.x] = value_own;
                list.x[threadIdx.x] = x_own;
            }
            if (edge_at >= 0) edge = load_value<G>(base, edge_at);
            if (threadIdx.x < 32) edge_listed[threadIdx.x] = 0;
            if (threadIdx.x == 0) row_label_logit = a.row.labels ? load_value<G>(base, label) : 0.0f;
        }
        __syncthreads();                                         // the list
        const int in_own = id_own - s.head - own.begin * E;      // where an id lies in this block's share
        const bool in_share = id_own >= s.head && in_own >= 0 && in_own < own.count * E;
        if (wanted) {
            if (id_own >= 0) {
                first_own = true;
                for (int i = 0; i < static_cast<int>(threadIdx.x); ++i) first_own &= list.id[i] != id_own;
                if (id_own < s.head) edge_listed[id_own] = 1;
                if (id_own >= vocab - s.tail) edge_listed[s.head + id_own - (vocab - s.tail)] = 1;
            }
            if (threadIdx.x < kMostListed) list.first[threadIdx.x] = first_own;
            if (warp == kWarps - 1) {
                const Normalizer n = list_normalizer(a, list);
                if (lane == 0) teacher = n;
            }
            if (own.count > 0) {
                if (!barrier_wait(smem_address(&landed), phase, a.tries)) {
                    late[parity] = 1;                            // what the walk below finds is not used
                    for (uint32_t q = 0; q < blocks; ++q)
                        if (blocks > 1) asm volatile("st.shared::cluster.s32 [%0], 1;" :: "r"(peer_address(smem_address(&late[parity]), q)) : "memory");
                }
                phase ^= 1;
            }
            if (in_share) store_value<G>(kept_row, in_own, -INFINITY);
        }
        __syncthreads();                                         // the listed elements are out of the row
        if (wanted) {
            const uint4 *from = kept_row + threadIdx.x;
            int left = own.count - static_cast<int>(threadIdx.x);
            for (; left > kStep - THREADS; left -= kStep, from += kStep) take_rest<G, kBatch, THREADS, true, TWO>(&x, from, left, k);
            if (left > 0) take_rest<G, kBatch, THREADS, false, TWO>(&x, from, left, k);
            if (edge_at >= 0 && !edge_listed[threadIdx.x]) x = take_one(x, edge, k);
        }
        x = warp_join(x, k);
        if (lane == 0) warp_part[warp] = x;
        __syncthreads();
        if (warp == 0) x = warp_join(lane < kWarps ? warp_part[lane] : RestSums{-INFINITY, 0.0f, 0.0f}, k);
        if (blocks > 1) {
            if (warp == 0 && lane < static_cast<int>(blocks)) {
                const uint32_t at = peer_address(smem_address(&block_part[parity][rank]), lane);
                asm volatile("st.shared::cluster.f32 [%0], %1;\n\tst.shared::cluster.f32 [%0 + 4], %2;\n\tst.shared::cluster.f32 [%0 + 8], %3;"
                             :: "r"(at), "f"(x.m), "f"(x.s), "f"(x.s1) : "memory");
            }
            cluster_sync();
            if (warp == 0) x = warp_join(lane < static_cast<int>(blocks) ? block_part[parity][lane] : RestSums{-INFINITY, 0.0f, 0.0f}, k);
        }
        if (warp == 0) {
            float kl = 0.0f, ce = 0.0f;
            DistillFactors f = distill_row(a, list, x, wanted, weight, wanted ? row_label_logit : 0.0f, wanted ? teacher : Normalizer{0.0f, 0.0f}, &kl, &ce);
            f.late = late[parity];
            if (lane == 0) {
                factors = f;
                if (rank == 0 && !f.late) {
                    // A coefficient of exactly 0 takes its term out.
                    const float soft = a.soft == 0.0f ? 0.0f : __fmul_rn(a.soft, kl), hard = a.hard == 0.0f ? 0.0f : __fmul_rn(a.hard, ce);
                    const float loss = __fadd_rn(soft, hard);
                    a.token_loss[t] = loss;
                    if (f.active) {
                        const double w = weight;
                        sums.loss += w * loss;
                        sums.kl += w * kl;
                        sums.ce += w * ce;
                        sums.weight += w;
                    }
                }
            }
        }
        __syncthreads();                                         // the factors
        const DistillFactors f = factors;
        if (f.late) break;
        if (a.dlogits) {
            char *out = static_cast<char *>(a.dlogits) + t * a.ld_dlogits * G::kBytes;
            const bool same_phase = (reinterpret_cast<uintptr_t>(out) - reinterpret_cast<uintptr_t>(base)) % 16 == 0;
            if (same_phase) {
                uint4 *to = reinterpret_cast<uint4 *>(out + s.head * G::kBytes) + own.begin + threadIdx.x;
                int left = own.count - static_cast<int>(threadIdx.x);
                if (f.active) {
                    const uint4 *from = kept_row + threadIdx.x;
                    if constexpr (TWO) {
                        for (; left > kStep - THREADS; left -= kStep, from += kStep, to += kStep) store_two<G, kBatch, THREADS, true>(to, from, left, f, k);
                        if (left > 0) store_two<G, kBatch, THREADS, false>(to, from, left, f, k);
                    } else {
                        const Power power(f.m_rest, k);
                        for (; left > kStep - THREADS; left -= kStep, from += kStep, to += kStep)
                            store_batch<G, kBatch, THREADS, true>(to, from, left, power, f.rest);
                        if (left > 0) store_batch<G, kBatch, THREADS, false>(to, from, left, power, f.rest);
                    }
                } else {
                    for (; left > 0; left -= THREADS, to += THREADS) *to = make_uint4(0, 0, 0, 0);
                }
            } else {
                for (int e = threadIdx.x; e < own.count * E; e += THREADS)
                    store_value<G>(out, s.head + own.begin * E + e, f.active ? rest_gradient<TWO>(load_value<G>(kept_row, e), f, k) : 0.0f);
            }
            if (edge_at >= 0) store_value<G>(out, edge_at, f.active ? rest_gradient<TWO>(edge, f, k) : 0.0f);
            __syncthreads();                                     // the row is read and written
            if (f.active) {
                // Who stores an element again: the block that has it.
                const auto has = [&](int id) {
                    const int at = id - s.head - own.begin * E;
                    return id < s.head || id >= vocab - s.tail ? rank == 0 : at >= 0 && at < own.count * E;
                };
                const bool labelled = a.row.labels && f.hard != 0.0f;
                if (first_own && has(id_own)) {
                    float q = 0.0f;                              // of all entries with this id
                    for (int i = threadIdx.x; i < a.k; ++i)
                        if (list.id[i] == id_own) q = __fadd_rn(q, expf(listed_log(a, list.value[i], f.shift, f.log_sum)));
                    const float p = expf(log_prob(x_own, MaxSum{f.m, f.s}, k, a.row.inv_temperature));
                    float g = f.soft == 0.0f ? 0.0f : __fmul_rn(f.soft, __fmaf_rn(f.mass, p, -q));
                    if (f.hard != 0.0f) {
                        const float p1 = TWO ? expf(log_prob(x_own, MaxSum{f.m, f.s1}, kLog2e, 1.0f)) : p;
                        g = __fmaf_rn(f.hard, __fsub_rn(p1, labelled && id_own == label ? 1.0f : 0.0f), g);
                    }
                    store_value<G>(out, id_own, g);
                }
                // The label, where it is not listed.
                if (labelled && warp == kWarps - 1 && has(static_cast<int>(label))) {
                    bool listed = false;
                    for (int i = lane; i < a.k; i += 32) listed |= list.id[i] == label;
                    if (!__any_sync(0xffffffffu, listed) && lane == 0)
                        store_value<G>(out, label, __fsub_rn(rest_gradient<TWO>(row_label_logit, f, k), f.hard));
                }
            }
        }
        // The row's memory and list are free: what was written over the row comes before the next copy.
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncthreads();
    }
    if (threadIdx.x == 0 && factors.late) {
        barrier_wait(smem_address(&landed), phase ^ 1, kWaitTries);      // the copy in flight, if any
        sums.loss = sums.kl = sums.ce = sums.weight = NAN;
    }
    if (threadIdx.x == 0 && rank == 0)
        a.partial[first_row] = make_float4(static_cast<float>(sums.loss), static_cast<float>(sums.kl), static_cast<float>(sums.ce), static_cast<float>(sums.weight));
    if (blocks > 1) cluster_sync();                              // nobody leaves while a peer writes to its memory
}

constexpr int kDistillSumThreads = 1024;

__global__ void __launch_bounds__(kDistillSumThreads) star_distillation_sums_kernel(const float4 *partial, int64_t n, float *sums)
{
    __shared__ double shared[kDistillSumThreads / 32];
    wait_for_primary();
    double s[4] = {0.0, 0.0, 0.0, 0.0};
    for (int64_t i = threadIdx.x; i < n; i += kDistillSumThreads) {
        const float4 x = partial[i];
        s[0] += x.x; s[1] += x.y; s[2] += x.z; s[3] += x.w;
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const double total = block_sum(s[q], shared);
        if (threadIdx.x == 0) sums[q] = static_cast<float>(total);
    }
}

}  // namespace star
