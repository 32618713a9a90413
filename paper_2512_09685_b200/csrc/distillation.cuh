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
    int32_t *order;              // may be null: the rows that take part in front, the others behind them, then the number of the first
    void *dlogits;               // may be null
    int64_t ld_dlogits;
    int tries;                   // of a wait
};

// Whether a row takes part, as far as its label and weight say.
__device__ __forceinline__ bool takes_part(const RowArgs &a, int64_t label, float weight)
{
    return (!a.labels || (label >= 0 && label < a.vocab)) && weight != 0.0f;
}

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
    float inv_s;
    float rest_s;        // of what is not listed, at m_rest
    float p_listed;      // the student's probability of the listed
    float p0, q0;        // the probabilities of what is not listed, the student's and the teacher's; q0 of 0: no such term
    float mass;          // what the teacher's probabilities that count add up to
    float soft, hard;    // weight and coefficients in front of the gradient's parts
    int active;
    int late;            // a wait for the row ran out: nothing of it holds
};

// How the sum at temperature 1 is had: kOne, not at all (no label term, or temperature 1
// itself); kTwo, by a power of its own; kSquare and kFourth, for temperatures of 2 and 4,
// as the second and fourth power of the other one.
enum Mode { kOne, kTwo, kSquare, kFourth };

struct DistillSums {
    double loss, kl, ce, weight;
};

// q log(q / p) - q + p, which is never negative; d = log(p / q).  Where the two are near,
// p - q leaves no digits beside q d, and exp(d) - 1 - d is good to 2^-24 / |d| of itself, as
// d^2 / 2 is by what d is off (a series of exp(d) - 1 - d gives the same errors of the loss).
__device__ __forceinline__ float divergence(float q, float p, float d)
{
    if (q == 0.0f) return p;
    if (fabsf(d) < 1.0f) return __fmul_rn(q, __fsub_rn(expm1f(d), d));
    return __fsub_rn(__fsub_rn(p, q), __fmul_rn(q, d));
}

// The same sum in every thread of a warp; NaNs stay.
__device__ __forceinline__ double warp_sum_wide(double x)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

// What a teacher's list says by itself.  (v - shift) / temperature - log_sum is the
// log-probability of a value v, the difference first, as for the student's; log_sum =
// -inf: nothing is listed.
struct Teacher {
    double log_sum;
    float shift;
    float mass;          // of the listed
    float missing;       // 1 - mass where the rest counts, else 0
};
// log s of a normal number, to half a step of its mantissa's part: the exponent's part is exact in binary64.
__device__ __forceinline__ double log_wide(float s)
{
    if (!(s < INFINITY)) return s;                               // NaN
    const int bits = __float_as_int(s);
    return static_cast<double>((bits >> 23) - 127) * 0.693147180559945309417 + static_cast<double>(logf(__int_as_float((bits & 0x007fffff) | 0x3f800000)));
}
// In binary64: a loss near 0 is made of small differences of such logarithms.
__device__ __forceinline__ double listed_log(const DistillArgs &a, float v, const Teacher &t)
{
    if (t.log_sum == -INFINITY) return -INFINITY;
    return (static_cast<double>(v) - static_cast<double>(t.shift)) * static_cast<double>(a.inv_teacher_temperature) - t.log_sum;
}

// A row's list, with a thread for each entry, and what else there is to know of a row
// before its logits are there.
constexpr int kListWarps = kMostListed / 32;
struct Listed {
    int4 id4[kMostListed / 4];   // -1 or less: absent
    float value[kMostListed];    // the teacher's
    int64_t asked_label;         // as given
    float weight;
    int label;                   // -1: none
    float label_logit;
    int wanted;                  // the label and the weight let the row take part
    int row;
    RestSums part[kListWarps];   // the student's statistics of the first entries of each id
    float most[kListWarps];      // of the teacher's values: the largest, -inf, or NaN
    double sum[kListWarps];      // of exp((value - most) / temperature)
    float terms[kListWarps];     // of the loss
    Teacher teacher;
    int edge[32];                // who lists the elements beside the whole pieces; -1: nobody
    int twice, has_label;        // an id is listed twice; the label is listed
    __device__ __forceinline__ const int *ids() const { return reinterpret_cast<const int *>(id4); }
};
template <typename G> __device__ __forceinline__ void mark(void *row, int at, int n)
{
    if constexpr (G::kBytes == 2)
        static_cast<unsigned short *>(row)[at] = static_cast<unsigned short>(n);
    else
        static_cast<int *>(row)[at] = n;
}
template <typename G> __device__ __forceinline__ bool marked(const void *row, int at, int n)
{
    if constexpr (G::kBytes == 2)
        return static_cast<const volatile unsigned short *>(row)[at] == n;
    else
        return static_cast<const volatile int *>(row)[at] == n;
}
// 4 or 8 bytes, asynchronously.
template <int SIZE> __device__ __forceinline__ void copy_word(void *to, const void *from)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" :: "r"(smem_address(to)), "l"(from), "n"(SIZE) : "memory");
}
__device__ __forceinline__ void list_sync() { asm volatile("bar.sync 1, %0;" :: "n"(kMostListed) : "memory"); }

// From the warps' parts.
__device__ __forceinline__ Teacher make_teacher(const DistillArgs &a, const Listed &list)
{
    const int warps = (a.k + 31) / 32;
    float shift = -INFINITY;
    bool bad = false;
    for (int w = 0; w < warps; ++w) {
        bad |= list.most[w] != list.most[w];
        shift = fmaxf(shift, list.most[w]);
    }
    if (bad || shift == INFINITY) return Teacher{NAN, 0.0f, NAN, NAN};
    if (shift == -INFINITY) return a.rest ? Teacher{0.0, 0.0f, 0.0f, 1.0f} : Teacher{-INFINITY, 0.0f, 0.0f, 0.0f};
    double sum = 0.0;
    for (int w = 0; w < warps; ++w)
        if (list.most[w] > -INFINITY) sum += list.sum[w] * static_cast<double>(a.rest ? 1.0f : expf(__fmul_rn(__fsub_rn(list.most[w], shift), a.inv_teacher_temperature)));
    if (a.rest) return Teacher{0.0, 0.0f, static_cast<float>(sum), static_cast<float>(1.0 - sum)};      // log-probabilities already
    return Teacher{log_wide(static_cast<float>(sum)), shift, 1.0f, 0.0f};
}

// A row's factors from its statistics without and of the listed elements, by a warp: what
// the gradient waits for.
template <int MODE>
__device__ __forceinline__ DistillFactors make_factors(const DistillArgs &a, const Teacher &teacher, RestSums rest, RestSums listed, float weight)
{
    const float inv_t = a.row.inv_temperature, k = __fmul_rn(inv_t, kLog2e);
    DistillFactors f{};
    f.m_rest = rest.m;
    f.rest_s = rest.s;
    f.m = fmaxf(rest.m, listed.m);
    const float down = rest.s == 0.0f ? 0.0f : rebase(rest.m, f.m, k);
    const float rest_s = __fmul_rn(rest.s, down);                // what is not listed, at the row's reference
    const float listed_s = __fmul_rn(listed.s, rebase(listed.m, f.m, k));
    f.s = __fadd_rn(listed_s, rest_s);
    f.active = !(f.s == 0.0f);
    f.inv_s = reciprocal_fast(f.s);                              // sums are near 1 or more
    f.p0 = __fmul_rn(rest_s, f.inv_s);
    f.p_listed = __fmul_rn(listed_s, f.inv_s);
    f.q0 = teacher.missing > 0.0f && rest.s > 0.0f ? teacher.missing : 0.0f;
    f.mass = f.q0 > 0.0f ? 1.0f : teacher.mass;
    f.soft = __fmul_rn(__fmul_rn(weight, a.soft), inv_t);
    f.hard = __fmul_rn(weight, a.hard);
    f.s1 = f.s;
    if (a.soft != 0.0f)
        f.rest = __fmul_rn(f.soft, f.q0 > 0.0f ? __fmul_rn(__fsub_rn(f.p0, f.q0), reciprocal_fast(rest.s)) : __fmul_rn(__fmul_rn(f.mass, down), f.inv_s));
    if constexpr (MODE != kOne) {
        const float down1 = rest.s == 0.0f ? 0.0f : rebase(rest.m, f.m, kLog2e);
        f.s1 = __fadd_rn(__fmul_rn(listed.s1, rebase(listed.m, f.m, kLog2e)), __fmul_rn(rest.s1, down1));
        f.rest1 = __fmul_rn(f.hard, __fmul_rn(down1, reciprocal_fast(f.s1)));
    } else {
        f.rest = __fmaf_rn(f.hard, __fmul_rn(down, f.inv_s), f.rest);
    }
    return f;
}

// The two parts of an active row's loss, given the sum of the listed entries' terms.
//
// sum q log(q / p) is made of terms of one sign (divergence above).  They add up to it
// if both distributions add up to 1; what they do not is put right at the end.
__device__ __forceinline__ void row_loss(const DistillArgs &a, const Teacher &teacher, const DistillFactors &f, float terms, float label_logit, float *kl_out,
                                         float *ce_out)
{
    const float inv_t = a.row.inv_temperature, k = __fmul_rn(inv_t, kLog2e);
    const MaxSum row{f.m, f.s};
    float d = 0.0f;
    if (f.q0 > 0.0f) {
        // log p0 and log q0 keep their digits near 0 by way of what is listed, and p0's exists where p0 itself is
        // below binary32 by its parts.
        const float log_p0 = f.p_listed < 0.5f ? log1pf(-f.p_listed) : f.p0 > 1e-30f ? logf(f.p0) : __fadd_rn(log_prob(f.m_rest, row, k, inv_t), logf(f.rest_s));
        d = __fsub_rn(log_p0, teacher.mass < 0.5f ? log1pf(-teacher.mass) : logf(f.q0));
    }
    const float off = f.q0 > 0.0f ? 0.0f : a.rest ? -teacher.missing : __fsub_rn(f.mass, 1.0f);      // the teacher's sum - 1
    *kl_out = __fadd_rn(__fadd_rn(terms, divergence(f.q0, f.p0, d)), off);
    *ce_out = 0.0f;
    if (a.hard != 0.0f) {
        const bool one = inv_t == 1.0f;
        *ce_out = -log_prob(label_logit, MaxSum{f.m, one ? f.s : f.s1}, one ? k : kLog2e, 1.0f);
    }
}

// The powers at both temperatures.
template <int MODE> __device__ __forceinline__ void two_powers(Pair d, Pair k, Pair k1, Pair *p, Pair *p1)
{
    *p = pair_exp2(pair_mul(d, k));
    if constexpr (MODE == kTwo) {
        *p1 = pair_exp2(pair_mul(d, k1));
    } else {
        *p1 = pair_mul(*p, *p);
        if constexpr (MODE == kFourth) *p1 = pair_mul(*p1, *p1);
    }
}

// As take_batch, with the sum at temperature 1 where it is another.
template <typename G, int N, int THREADS, bool FULL, int MODE>
__device__ __forceinline__ void take_rest(RestSums *x, const uint4 *from, int left, float k)
{
    if constexpr (MODE == kOne) {
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
                    Pair p, p1;
                    two_powers<MODE>(pair_add(f[e], minus_m), kk, k1, &p, &p1);
                    s = pair_add(s, p);
                    s1 = pair_add(s1, p1);
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
template <int MODE> __device__ __forceinline__ RestSums warp_join(RestSums x, float k)
{
    const float m = warp_max(x.m);
    return RestSums{m, warp_sum(__fmul_rn(x.s, rebase(x.m, m, k))), MODE == kOne ? 0.0f : warp_sum(__fmul_rn(x.s1, rebase(x.m, m, kLog2e)))};
}
__device__ __forceinline__ RestSums take_one(RestSums x, float v, float k)
{
    const float m = fmaxf(x.m, v);
    x = rest_move(x, m, k);
    return RestSums{m, __fadd_rn(x.s, exp2_fast(exponent(v, m, k))), __fadd_rn(x.s1, exp2_fast(exponent(v, m, kLog2e)))};
}

// The gradient of an element that is not listed, from the factors that it takes.
struct RestFactors {
    float m, rest, rest1;
};
template <int MODE> __device__ __forceinline__ float rest_gradient(float x, const RestFactors &f, float k)
{
    const float g = __fmul_rn(f.rest, exp2_fast(exponent(x, f.m, k)));
    return MODE != kOne ? __fmaf_rn(f.rest1, exp2_fast(exponent(x, f.m, kLog2e)), g) : g;
}
template <typename G, int N, int THREADS, bool FULL, int MODE>
__device__ __forceinline__ void store_rest(uint4 *to, const uint4 *from, int left, const RestFactors &f, float k)
{
    if constexpr (MODE == kOne) {
        store_batch<G, N, THREADS, FULL>(to, from, left, Power(f.m, k), f.rest);
    } else {
        constexpr int P = Granule<G>::kPairs;
        const Pair minus_m = pair_of(-pivot(f.m)), kk = pair_of(k), k1 = pair_of(kLog2e), a = pair_of(f.rest), b = pair_of(f.rest1);
#pragma unroll
        for (int q = 0; q < N; ++q) {
            if (FULL || q * THREADS < left) {
                Pair g[P];
                Granule<G>::widen(from[q * THREADS], g);
#pragma unroll
                for (int e = 0; e < P; ++e) {
                    Pair p, p1;
                    two_powers<MODE>(pair_add(g[e], minus_m), kk, k1, &p, &p1);
                    g[e] = pair_fma(b, p1, pair_mul(a, p));
                }
                to[q * THREADS] = Granule<G>::narrow(g);
            }
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
//
// 4096 x 50257 bf16, k = 64: 179 us, 4.6 TB/s of reading and writing (8192 rows, 35 %
// masked, 277).  Bound by the waits of a row's four barriers and the exponentials (55 % of
// their unit's time).  What a warp does alone between barriers takes eight times as long as
// its instructions, with another row's walk on the SM; so the list is read a row ahead into
// shared memory, its normalizer is found while others wait for the factors, and nothing of
// it lies in registers across the walks (223 us with the spills of that).
// ---------------------------------------------------------------------------
constexpr int kDistillBytesPerThread = 208;  // shared memory for the row: 208 KB an SM

template <typename G, int THREADS, int MODE>
__global__ void __launch_bounds__(THREADS, policy_blocks(THREADS)) star_distillation_kernel(const __grid_constant__ DistillArgs a)
{
    constexpr int E = Granule<G>::kCount, kWarps = THREADS / 32, kStep = kBatch * THREADS;
    // The list's threads: not the first warp's, where there are others.
    constexpr int kListFirst = THREADS > kMostListed ? 128 : 0;
    static_assert(THREADS >= kMostListed, "a thread to a listed element");
    extern __shared__ uint4 kept_row[];
    __shared__ RestSums warp_part[kWarps];
    __shared__ RestSums block_part[2][8];
    __shared__ DistillFactors factors;
    __shared__ DistillSums sums;
    __shared__ Listed lists[2];                                  // of every other row
    __shared__ int ahead[2];                                     // of every other item: its row, where rows are taken in a given order
    __shared__ int late[2];                                      // of every other row, as in the policy loss
    __shared__ alignas(8) uint64_t landed;                       // the row's copy is in place
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int at_list = static_cast<int>(threadIdx.x) - kListFirst, list_warp = at_list / 32;
    const bool lists_it = at_list >= 0 && at_list < kMostListed;
    const bool works = lists_it && list_warp * 32 < a.k;         // this warp has entries
    const float k = __fmul_rn(a.row.inv_temperature, kLog2e);
    const int vocab = static_cast<int>(a.row.vocab);
    const uint32_t blocks = cluster_size(), rank = cluster_rank();
    const int log_blocks = 31 - __clz(static_cast<int>(blocks));
    const int first_item = static_cast<int>(blockIdx.x) >> log_blocks, step = static_cast<int>(gridDim.x) >> log_blocks, rows = static_cast<int>(a.row.rows);
    launch_dependents();
    if (threadIdx.x == 0) {
        sums = DistillSums{0.0, 0.0, 0.0, 0.0};
        late[0] = late[1] = 0;
        barrier_init(smem_address(&landed), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (lists_it) {
        for (Listed &list : lists) {                             // what no record brings
            reinterpret_cast<int *>(list.id4)[at_list] = -1;
            list.value[at_list] = -INFINITY;
        }
        if (at_list == 0) {
            for (Listed &list : lists) {
                list.asked_label = -1;
                list.weight = 1.0f;
                list.label_logit = 0.0f;
            }
        }
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
    const int items = a.order ? a.order[rows] : rows;
    // An item's row, list, label and weight, into shared memory by the list's threads: under way ...
    const auto ask = [&](int item, int parity) {
        Listed &list = lists[parity];
        if (!lists_it || item >= items) return;
        const int64_t t = a.order ? ahead[parity] : item;
        if (at_list < a.k) {
            copy_word<4>(reinterpret_cast<int *>(list.id4) + at_list, a.ids + t * a.ld_ids + at_list);
            copy_word<4>(list.value + at_list, a.values + t * a.ld_values + at_list);
        }
        if (at_list == 0) {
            list.row = static_cast<int>(t);
            if (a.row.labels) copy_word<8>(&list.asked_label, a.row.labels + t);
            if (a.row.weights) copy_word<4>(&list.weight, a.row.weights + t);
            if (a.order && item + step < items) copy_word<4>(&ahead[parity ^ 1], a.order + item + step);
        }
    };
    // No entry in front has its id.
    const auto is_first = [&](const Listed &list, int id) {
        bool first = true;
        for (int i = 0; i < at_list; i += 4) {
            const int4 other = list.id4[i / 4];
            first &= other.x != id && (other.y != id || i + 1 >= at_list) && (other.z != id || i + 2 >= at_list) && (other.w != id || i + 3 >= at_list);
        }
        return first;
    };
    // ... and there: what the teacher's list says by itself.  Where other blocks share the row, a thread's entry's
    // logit, and the label's, are then on their way; a block on its own finds them in its row.
    const auto take_list = [&](int item, Listed &list, float *x, float *label_logit) {
        if (item >= items) {
            if (lists_it && at_list == 0) list.wanted = 0;
            return;
        }
        if (!lists_it) return;
        asm volatile("cp.async.wait_all;" ::: "memory");
        int id = list.ids()[at_list];
        if (id >= vocab) {
            id = -1;
            reinterpret_cast<int *>(list.id4)[at_list] = -1;
        }
        if (at_list < 32) list.edge[at_list] = -1;
        if (at_list == 0) {
            const int64_t asked = list.asked_label;
            const int label = asked >= 0 && asked < vocab ? static_cast<int>(asked) : -1;
            list.label = label;
            list.wanted = takes_part(a.row, asked, list.weight);
            list.twice = list.has_label = 0;
        }
        if (works) {
            const float v = id >= 0 ? list.value[at_list] : -INFINITY, most = warp_max(v);
            const bool bad = __any_sync(0xffffffffu, v != v);
            const float p = v > -INFINITY ? expf(__fmul_rn(a.rest ? v : __fsub_rn(v, most), a.inv_teacher_temperature)) : 0.0f;
            const double sum = a.rest ? warp_sum_wide(p) : warp_sum(p);          // 1 - the sum cancels
            if (lane == 0) {
                list.most[list_warp] = bad ? NAN : most;
                list.sum[list_warp] = sum;
            }
        }
        list_sync();
        if (id >= 0 && id == list.label) list.has_label = 1;
        if (list_warp == 0) {
            const Teacher teacher = make_teacher(a, list);
            if (lane == 0) list.teacher = teacher;
        }
        if (blocks > 1 && at_list == 0 && list.label >= 0) *label_logit = load_value<G>(row_base(list.row), list.label);
        if (blocks > 1 && id >= 0) {
            const char *base = row_base(list.row);
            *x = load_value<G>(base, id);
            const RowSplit s = split_row<G>(base, vocab);
            if (id < s.head) list.edge[id] = at_list;
            if (id >= vocab - s.tail) list.edge[s.head + id - (vocab - s.tail)] = at_list;
            if (!is_first(list, id)) list.twice = 1;
        }
    };

    // A row that takes no part.
    const auto clear = [&](int64_t t) {
        if (threadIdx.x == 0 && rank == 0) a.token_loss[t] = 0.0f;
        if (!a.dlogits) return;
        const RowSplit s = split_row<G>(row_base(t), vocab);
        const RowShare own = row_share(s.granules, rank, log_blocks);
        char *out = static_cast<char *>(a.dlogits) + t * a.ld_dlogits * G::kBytes;
        if ((reinterpret_cast<uintptr_t>(out) - reinterpret_cast<uintptr_t>(row_base(t))) % 16 == 0) {
            uint4 *to = reinterpret_cast<uint4 *>(out + s.head * G::kBytes) + own.begin;
            for (int i = threadIdx.x; i < own.count; i += THREADS) to[i] = make_uint4(0, 0, 0, 0);
        } else {
            for (int i = threadIdx.x; i < own.count * E; i += THREADS) store_value<G>(out, s.head + own.begin * E + i, 0.0f);
        }
        const int edge_at = rank == 0 ? edge_element(s, threadIdx.x, vocab) : -1;
        if (edge_at >= 0) store_value<G>(out, edge_at, 0.0f);
    };
    // In a given order, the rows that take no part are cleared between the others; this block's next one's place.
    int idle = a.order ? items + first_item : rows;

    // A cluster's blocks meet once in every row, whether it takes part or not: between a block's reading of what peers
    // wrote for a row, chosen by its parity, and their writing for the row after the next lies the barrier of the row
    // between, and none depends on what the blocks read to leave together.
    uint32_t phase = 0;
    int parity = 0;
    float x_own = 0.0f, label_logit = 0.0f;
    if (threadIdx.x == 0 && first_item < items) {                // the first row's copy does not wait for its list
        const int64_t t = a.order ? a.order[first_item] : first_item;
        if (takes_part(a.row, a.row.labels ? a.row.labels[t] : 0, a.row.weights ? a.row.weights[t] : 1.0f)) fetch(t);
    }
    if (a.order && lists_it && first_item < items) {
        if (at_list == 0) ahead[0] = a.order[first_item];
        list_sync();
    }
    ask(first_item, 0);
    take_list(first_item, lists[0], &x_own, &label_logit);
    __syncthreads();
    int item = first_item;
    for (; item < items; item += step, parity ^= 1) {
        Listed &list = lists[parity], &next = lists[parity ^ 1];
        const int64_t t = list.row;
        const bool writes = a.dlogits != nullptr;
        const auto out_of = [&] { return static_cast<char *>(a.dlogits) + t * a.ld_dlogits * G::kBytes; };
        const auto same_phase = [&] { return (reinterpret_cast<uintptr_t>(out_of()) - reinterpret_cast<uintptr_t>(row_base(t))) % 16 == 0; };
        const RowSplit s = split_row<G>(row_base(t), vocab);
        const RowShare own = row_share(s.granules, rank, log_blocks);
        const int edge_at = rank == 0 ? edge_element(s, threadIdx.x, vocab) : -1;
        bool active = false;
        if (list.wanted) {
            const float edge = edge_at >= 0 ? load_value<G>(row_base(t), edge_at) : 0.0f;
            if (blocks > 1 && lists_it && at_list == 0) list.label_logit = label_logit;
            // This thread's entry, and where it lies in the block's share.
            const int id = lists_it ? list.ids()[at_list] : -1, in_own = id - s.head - own.begin * E;
            const bool in_share = id >= s.head && in_own >= 0 && in_own < own.count * E;
            if (own.count > 0) {
                if (!barrier_wait(smem_address(&landed), phase, a.tries)) {
                    late[parity] = 1;                            // what the walk below finds is not used
                    for (uint32_t q = 0; q < blocks; ++q)
                        if (blocks > 1) asm volatile("st.shared::cluster.s32 [%0], 1;" :: "r"(peer_address(smem_address(&late[parity]), q)) : "memory");
                }
                phase ^= 1;
            }
            if (blocks == 1 && lists_it) {
                const auto logit = [&](int i) {
                    const int at = i - s.head;
                    return i >= s.head && at < own.count * E ? load_value<G>(kept_row, at) : load_value<G>(row_base(t), i);
                };
                if (id >= 0) x_own = logit(id);
                if (at_list == 0 && list.label >= 0) list.label_logit = logit(list.label);
                list_sync();
                // Whether an id is listed twice: each entry leaves its number in its element's place and looks who was last.
                const int edge_of = id < 0 || in_share ? -1 : id < s.head ? id : s.head + id - (vocab - s.tail);
                if (in_share) mark<G>(kept_row, in_own, at_list);
                if (edge_of >= 0) list.edge[edge_of] = at_list;
                list_sync();
                if (in_share ? !marked<G>(kept_row, in_own, at_list) : edge_of >= 0 && list.edge[edge_of] != at_list) list.twice = 1;
            }
            if (in_share) {
                store_value<G>(kept_row, in_own, -INFINITY);
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");     // before the next copy into its place
            }
            __syncthreads();                                     // the listed elements are out of the row
            bool first = id >= 0;
            if (works) {
                if (list.twice && first) first = is_first(list, id);
                const float one = first ? exp2_fast(exponent(x_own, x_own, k)) : 0.0f;           // 0 for -inf, NaN for a NaN
                const RestSums part = warp_join<MODE>(RestSums{first ? x_own : -INFINITY, one, one}, k);
                if (lane == 0) list.part[list_warp] = part;
            }
            ask(item + step, parity ^ 1);                        // while the walk goes on
            RestSums x{-INFINITY, 0.0f, 0.0f};
            {
                const uint4 *from = kept_row + threadIdx.x;
                int left = own.count - static_cast<int>(threadIdx.x);
                for (; left > kStep - THREADS; left -= kStep, from += kStep) take_rest<G, kBatch, THREADS, true, MODE>(&x, from, left, k);
                if (left > 0) take_rest<G, kBatch, THREADS, false, MODE>(&x, from, left, k);
                if (edge_at >= 0 && list.edge[threadIdx.x] < 0) x = take_one(x, edge, k);
            }
            x = warp_join<MODE>(x, k);
            if (lane == 0) warp_part[warp] = x;
            __syncthreads();
            if (warp == 0) x = warp_join<MODE>(lane < kWarps ? warp_part[lane] : RestSums{-INFINITY, 0.0f, 0.0f}, k);
            if (blocks > 1) {
                if (warp == 0 && lane < static_cast<int>(blocks)) {
                    const uint32_t at = peer_address(smem_address(&block_part[parity][rank]), lane);
                    asm volatile("st.shared::cluster.f32 [%0], %1;\n\tst.shared::cluster.f32 [%0 + 4], %2;\n\tst.shared::cluster.f32 [%0 + 8], %3;"
                                 :: "r"(at), "f"(x.m), "f"(x.s), "f"(x.s1) : "memory");
                }
                cluster_sync();
                if (warp == 0) x = warp_join<MODE>(lane < static_cast<int>(blocks) ? block_part[parity][lane] : RestSums{-INFINITY, 0.0f, 0.0f}, k);
            }
            if (warp == 0) {
                const RestSums listed = warp_join<MODE>(lane * 32 < a.k ? list.part[lane] : RestSums{-INFINITY, 0.0f, 0.0f}, k);
                DistillFactors f = make_factors<MODE>(a, list.teacher, x, listed, list.weight);
                f.late = late[parity];
                if (lane == 0) factors = f;
            }
            float x_next = 0.0f;
            take_list(item + step, next, &x_next, &label_logit); // while the others wait for the factors
            __syncthreads();
            const DistillFactors &f = factors;
            if (f.late) break;
            active = f.active;
            const RestFactors g{f.m_rest, f.rest, f.rest1};
            // The listed elements' gradients, and terms of the loss.
            float listed_gradient = 0.0f;
            if (active && works) {
                float term = 0.0f;
                if (id >= 0) {
                    const float p = __fmul_rn(exp2_fast(exponent(x_own, f.m, k)), f.inv_s);
                    const double log_q = listed_log(a, list.value[at_list], list.teacher), log_s = log_wide(f.s);
                    const double log_p = (static_cast<double>(x_own) - static_cast<double>(pivot(f.m))) * static_cast<double>(a.row.inv_temperature) - log_s;
                    float q = expf(static_cast<float>(log_q));
                    term = divergence(q, p, static_cast<float>(log_p - log_q));
                    if (!first) term = __fsub_rn(term, p);       // its probability has been counted
                    for (int i = at_list + 1; list.twice && i < a.k; ++i)        // q of all entries with this id
                        if (list.ids()[i] == id) q = __fadd_rn(q, expf(static_cast<float>(listed_log(a, list.value[i], list.teacher))));
                    if (f.soft != 0.0f) listed_gradient = __fmul_rn(f.soft, __fmaf_rn(f.mass, p, -q));
                    if (f.hard != 0.0f) {
                        const float p1 = MODE != kOne ? __fmul_rn(exp2_fast(exponent(x_own, f.m, kLog2e)), reciprocal_fast(f.s1)) : p;
                        listed_gradient = __fmaf_rn(f.hard, __fsub_rn(p1, id == list.label ? 1.0f : 0.0f), listed_gradient);
                    }
                }
                term = warp_sum(term);
                if (lane == 0) list.terms[list_warp] = term;
            }
            x_own = x_next;
            if (writes && active) {
                char *out = out_of();
                if (same_phase()) {
                    uint4 *to = reinterpret_cast<uint4 *>(out + s.head * G::kBytes) + own.begin + threadIdx.x;
                    int left = own.count - static_cast<int>(threadIdx.x);
                    const uint4 *from = kept_row + threadIdx.x;
                    for (; left > kStep - THREADS; left -= kStep, from += kStep, to += kStep) store_rest<G, kBatch, THREADS, true, MODE>(to, from, left, g, k);
                    if (left > 0) store_rest<G, kBatch, THREADS, false, MODE>(to, from, left, g, k);
                } else {
                    for (int i = threadIdx.x; i < own.count * E; i += THREADS)
                        store_value<G>(out, s.head + own.begin * E + i, rest_gradient<MODE>(load_value<G>(kept_row, i), g, k));
                }
                if (edge_at >= 0) store_value<G>(out, edge_at, rest_gradient<MODE>(edge, g, k));
            }
            __syncthreads();                                     // the row is read and written
            if (next.wanted && threadIdx.x == 0) fetch(next.row);
            // While that is on its way: the listed elements and the label again, and the row's loss.
            if (writes && active) {
                char *out = out_of();
                // Who stores an element again: the block that has it.
                const auto has = [&](int i) {
                    const int at = i - s.head - own.begin * E;
                    return i < s.head || i >= vocab - s.tail ? rank == 0 : at >= 0 && at < own.count * E;
                };
                if (first && has(id)) store_value<G>(out, id, listed_gradient);
                if (threadIdx.x == THREADS - 1 && list.label >= 0 && f.hard != 0.0f && !list.has_label && has(list.label))
                    store_value<G>(out, list.label, __fsub_rn(rest_gradient<MODE>(list.label_logit, g, k), f.hard));
            }
            if (rank == 0 && threadIdx.x == 32) {
                float kl = 0.0f, ce = 0.0f;
                if (active) {
                    float terms = 0.0f;
                    for (int w = 0; w * 32 < a.k; ++w) terms = __fadd_rn(terms, list.terms[w]);
                    row_loss(a, list.teacher, f, terms, list.label_logit, &kl, &ce);
                }
                // A coefficient of exactly 0 takes its term out.
                const float loss = __fadd_rn(a.soft == 0.0f ? 0.0f : __fmul_rn(a.soft, kl), a.hard == 0.0f ? 0.0f : __fmul_rn(a.hard, ce));
                a.token_loss[t] = loss;
                if (active) {
                    const double w = list.weight;
                    sums.loss += w * loss;
                    sums.kl += w * kl;
                    sums.ce += w * ce;
                    sums.weight += w;
                }
            }
        } else {
            if (blocks > 1) {
                cluster_sync();
                if (late[parity]) break;
            } else {
                __syncthreads();                                 // the last row's list has been read
            }
            ask(item + step, parity ^ 1);
            take_list(item + step, next, &x_own, &label_logit);
            __syncthreads();
            if (next.wanted && threadIdx.x == 0) fetch(next.row);
        }
        // What has no gradient: this row, and as many of the idle ones as keep step with the others.
        int others = idle < rows ? ((rows - idle + step - 1) / step * step + items - item - 1) / (items - item) : 0;
        for (int64_t zero = active ? -1 : t;;) {
            if (zero >= 0) clear(zero);
            if (others-- <= 0 || idle >= rows) break;
            zero = a.order[idle];
            idle += step;
        }
    }
    for (; idle < rows; idle += step) clear(a.order[idle]);      // of a block that had no other row
    __syncthreads();                                             // the sums
    if (threadIdx.x == 0) {
        if (item < items) {                                      // a wait ran out
            barrier_wait(smem_address(&landed), phase ^ 1, kWaitTries);  // the copy in flight, if any
            sums.loss = sums.kl = sums.ce = sums.weight = NAN;
        }
        if (rank == 0)
            a.partial[first_item] = make_float4(static_cast<float>(sums.loss), static_cast<float>(sums.kl), static_cast<float>(sums.ce), static_cast<float>(sums.weight));
    }
    if (blocks > 1) cluster_sync();                              // nobody leaves while a peer writes to its memory
}

// The order of the rows: those that take part in front.  A mask leaves one block more
// rows than another, in the largest of hundreds by a third at 28 rows each; taken from a
// list of those that take part they are dealt out evenly, and the others' zeros are
// written beside them.  One block; a thread has every 1024th row and up to 64 of them.
constexpr int kOrderThreads = 1024;
constexpr int kMostOrdered = 64 * kOrderThreads;

__global__ void __launch_bounds__(kOrderThreads) star_distillation_order_kernel(const __grid_constant__ RowArgs a, int32_t *order)
{
    __shared__ int warp_sums[32];
    launch_dependents();
    wait_for_primary();
    const int rows = static_cast<int>(a.rows), lane = threadIdx.x % 32;
    uint64_t taken = 0;
    int have = 0;                            // rows of this thread
    for (int first = threadIdx.x; first < rows; first += 8 * kOrderThreads) {
        int64_t label[8];
        float weight[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            const int t = first + q * kOrderThreads;
            label[q] = t < rows && a.labels ? a.labels[t] : 0;
            weight[q] = t < rows && a.weights ? a.weights[t] : 1.0f;
        }
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            if (first + q * kOrderThreads < rows) {
                taken |= static_cast<uint64_t>(takes_part(a, label[q], weight[q])) << have;
                ++have;
            }
        }
    }
    const int mine = __popcll(taken);
    int up_to = mine;                        // of the warp's threads up to this one
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
        const int other = __shfl_up_sync(0xffffffffu, up_to, o);
        if (lane >= o) up_to += other;
    }
    if (lane == 31) warp_sums[threadIdx.x / 32] = up_to;
    __syncthreads();
    int total = 0, in_front = 0;
#pragma unroll
    for (int w = 0; w < 32; ++w) {
        if (w == static_cast<int>(threadIdx.x) / 32) in_front = total;
        total += warp_sums[w];
    }
    // The rows in front of this thread's: every thread below has as many as this one or one more.
    const int full = rows / kOrderThreads, rest = rows % kOrderThreads, threads = static_cast<int>(threadIdx.x);
    int at = in_front + up_to - mine, other = total + full * threads + min(threads, rest) - at;
    for (int i = 0; i < have; ++i) {
        const int t = threads + i * kOrderThreads;
        order[taken >> i & 1 ? at++ : other++] = t;
    }
    if (threadIdx.x == 0) order[rows] = total;
}

constexpr int kDistillSumThreads = 1024;     // at most; fewer for few parts

__global__ void __launch_bounds__(kDistillSumThreads) star_distillation_sums_kernel(const float4 *partial, int64_t n, float *sums)
{
    __shared__ double shared[kDistillSumThreads / 32][4];
    wait_for_primary();
    double s[4] = {0.0, 0.0, 0.0, 0.0};
    for (int64_t i = threadIdx.x; i < n; i += blockDim.x) {
        const float4 x = partial[i];
        s[0] += x.x; s[1] += x.y; s[2] += x.z; s[3] += x.w;
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) s[q] = warp_sum_wide(s[q]);
    if (threadIdx.x % 32 == 0) {
#pragma unroll
        for (int q = 0; q < 4; ++q) shared[threadIdx.x / 32][q] = s[q];
    }
    __syncthreads();
    if (threadIdx.x < 4) {
        double total = 0.0;
        for (unsigned w = 0; w < blockDim.x / 32; ++w) total += shared[w][threadIdx.x];
        sums[threadIdx.x] = static_cast<float>(total);
    }
}

}  // namespace star
