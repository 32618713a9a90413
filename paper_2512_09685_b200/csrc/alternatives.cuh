// Device code of log-probabilities with entropy and top alternatives, and of their
// backward pass (sm_100a).
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "rows.cuh"

namespace star {

constexpr int kMostAlternatives = 128;       // STAR_MAX_ALTERNATIVES

struct AlternativesArgs {
    RowArgs row;                 // labels may be null
    int k;
    int32_t *top_ids;
    float *top_logp;
    int64_t ld_top;
    float *logp, *lse, *entropy; // each may be null
};

// Largest logit m, the sum s of 2^exponent(x, m), and t = the sum of
// 2^exponent(x, m) exponent(x, m): the entropy is log s - t log(2) / s, both terms
// of one sign.
struct MaxSums {
    float m, s, t;
};
// A power below the smallest binary32 adds nothing, whatever its exponent.
__device__ __forceinline__ float bounded(float d) { return fmaxf(d, -150.0f); }
__device__ __forceinline__ MaxSums move_to(MaxSums x, float m, float k)
{
    const float d = bounded(exponent(x.m, m, k)), r = exp2_fast(d);
    return MaxSums{m, __fmul_rn(x.s, r), __fmul_rn(r, __fmaf_rn(d, x.s, x.t))};
}
__device__ __forceinline__ MaxSums add(MaxSums a, MaxSums b) { return MaxSums{a.m, __fadd_rn(a.s, b.s), __fadd_rn(a.t, b.t)}; }
__device__ __forceinline__ MaxSums take_one(MaxSums x, float v, float k)
{
    const float m = fmaxf(x.m, v), d = exponent(v, m, k), e = exp2_fast(d);
    return add(move_to(x, m, k), MaxSums{m, e, __fmul_rn(e, bounded(d))});
}
__device__ __forceinline__ MaxSums warp_join(MaxSums x, float k)
{
    x = move_to(x, warp_max(x.m), k);
    return MaxSums{x.m, warp_sum(x.s), warp_sum(x.t)};
}

// As take_batch, with t.  Returns the batch's largest logit.
template <typename G, int N, int THREADS, bool FULL>
__device__ __forceinline__ float take_batch_with_entropy(MaxSums *x, const uint4 *from, int left, float k)
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
    if (m > x->m) *x = move_to(*x, m, k);
    const Pair minus_m = pair_of(-pivot(x->m)), kk = pair_of(k);
    Pair s = pair_of(0.0f), t = pair_of(0.0f);
#pragma unroll
    for (int q = 0; q < N; ++q) {
        if (FULL || q * THREADS < left) {
            Pair f[P];
            Granule<G>::widen(v[q], f);
#pragma unroll
            for (int e = 0; e < P; ++e) {
                float lo, hi;
                split_pair(pair_mul(pair_add(f[e], minus_m), kk), &lo, &hi);
                const Pair p = make_pair(exp2_fast(lo), exp2_fast(hi));
                s = pair_add(s, p);
                t = pair_fma(p, make_pair(bounded(lo), bounded(hi)), t);
            }
        }
    }
    float lo, hi;
    split_pair(s, &lo, &hi);
    x->s = __fadd_rn(x->s, __fadd_rn(lo, hi));
    split_pair(t, &lo, &hi);
    x->t = __fadd_rn(x->t, __fadd_rn(lo, hi));
    return m;
}

// A logit's place in the order: larger for larger logits, one for both zeros.
// -inf has kLowest; a NaN's is beyond +inf or below it.
__device__ __forceinline__ uint32_t order_of(float x)
{
    const uint32_t bits = __float_as_uint(__fadd_rn(x, 0.0f));
    return bits & 0x80000000u ? ~bits : bits | 0x80000000u;
}
constexpr uint32_t kLowest = 0x007fffffu;    // order_of(-inf)
__device__ __forceinline__ float logit_of(uint32_t order) { return __uint_as_float(order & 0x80000000u ? order & 0x7fffffffu : ~order); }

// ---------------------------------------------------------------------------
// Statistics and the k largest logits of a row, in one reading of it from memory, by a
// block, or by a cluster of blocks that share it where there are few rows.
//
// A row falls into groups: what a thread takes (or what up to four neighbours take).
// The k-th largest of the groups' largest logits is at most the k-th largest logit, so
// no logit below it is wanted; and in a row whose large logits lie anywhere little more
// than k are not below it.  (The j-th largest within each warp, joined, needs no warp to
// look at all groups, but leaves a third more: 4096 x 50257, k = 64, 131 us against 117.)
// Every thread has kept the largest logit of each few batches that it took; the whole
// block looks again (in L2) at those that reach the bound, and what it finds are the
// candidates, whose ranks are counted.  Rows that leave too many of them (many equal
// logits, or the large ones side by side) are searched for the k-th largest by counting.
//
// 4096 x 50257 bf16, k = 64: 111 us, of which the walk with its sums 77 (64 without the
// entropy's), the second look 15, ranks 7, the bound 3; issue-bound more than by memory
// (63).
// ---------------------------------------------------------------------------
constexpr int kMostCandidates = 1088;        // of bf16: 128 threads' one granule, and the edges
constexpr int kMostGroups = 512;             // of a cluster; of a block: its threads
constexpr int kSlots = 8;                    // of a thread

struct Candidates {
    uint64_t key[kMostCandidates];           // order in the upper half, 2^31 - 1 - index below
    int count;
};
// `found` is the first block's.
template <bool CLUSTER> __device__ __forceinline__ void put_candidate(Candidates &found, uint32_t order, int index)
{
    const uint64_t key = static_cast<uint64_t>(order) << 32 | static_cast<uint32_t>(0x7fffffff - index);
    if constexpr (CLUSTER) {
        int at;
        asm volatile("atom.relaxed.cluster.shared::cluster.add.u32 %0, [%1], 1;" : "=r"(at) : "r"(peer_address(smem_address(&found.count), 0)) : "memory");
        if (at < kMostCandidates) asm volatile("st.shared::cluster.u64 [%0], %1;" :: "r"(peer_address(smem_address(&found.key[at]), 0)), "l"(key) : "memory");
    } else {
        const int at = atomicAdd(&found.count, 1);
        if (at < kMostCandidates) found.key[at] = key;
    }
}

// By a warp: the largest bound that at least k of n orders reach, or one that few more reach.
template <int EACH> __device__ __forceinline__ uint32_t bound_of(const uint32_t *order, int n, int k)
{
    uint32_t x[EACH], low = 0xffffffffu, high = 0;
#pragma unroll
    for (int q = 0; q < EACH; ++q) {
        const int i = q * 32 + static_cast<int>(threadIdx.x % 32);
        x[q] = i < n ? order[i] : 0;
        if (i < n) low = min(low, x[q]);
        high = max(high, x[q]);
    }
    low = __reduce_min_sync(0xffffffffu, low);
    high = __reduce_max_sync(0xffffffffu, high);
    uint32_t width = high - low;             // the bound lies in [low, low + width]
    while (width > 0) {
        const uint32_t mid = low + (width - width / 2);
        int reach = 0;
#pragma unroll
        for (int q = 0; q < EACH; ++q) reach += x[q] >= mid ? 1 : 0;
        reach = __reduce_add_sync(0xffffffffu, reach);
        if (reach >= k) {
            width -= mid - low;
            low = mid;
            if (reach <= k + k / 8) break;
        } else {
            width = mid - low - 1;
        }
    }
    return low;
}

// A thread's steps along n elements.  They are counted rather than the elements: one beyond
// the last of 2^31 - 1 has no number.
template <int THREADS> __device__ __forceinline__ int row_steps(int n)
{
    return static_cast<int>((static_cast<unsigned>(n) + THREADS - 1 - threadIdx.x) / THREADS);
}

// How many logits of a row reach `bound`, by a block of THREADS; every thread gets it.
template <typename G, int THREADS> __device__ int count_row(const void *base, int vocab, uint32_t bound, int *total)
{
    int n = 0;
    const int steps = row_steps<THREADS>(vocab);
    for (int q = 0; q < steps; ++q) n += order_of(load_value<G>(base, q * THREADS + static_cast<int>(threadIdx.x))) >= bound ? 1 : 0;
    n = __reduce_add_sync(0xffffffffu, n);
    __syncthreads();
    if (threadIdx.x == 0) *total = 0;
    __syncthreads();
    if (threadIdx.x % 32 == 0) atomicAdd(total, n);
    __syncthreads();
    return *total;
}

// The candidates of a row that `low` leaves too many of (but at least k), by one block:
// counting finds a bound that leaves few enough, or the k-th largest logit itself, whose
// equals are then taken by ascending index.  `high`: the largest logit's.  A row of one
// value needs no counting, others up to 32 passes over the row (from L2).
template <typename G, int THREADS>
__device__ __noinline__ void search_row(const void *base, int vocab, int k, uint32_t low, uint32_t high, Candidates &found, int *scratch)
{
    uint32_t width = high - low;
    int reach = kMostCandidates + 1;         // logits at or above low
    while (width > 0 && reach > kMostCandidates) {
        const uint32_t mid = low + (width - width / 2);
        const int n = count_row<G, THREADS>(base, vocab, mid, scratch);
        if (n >= k) {
            width -= mid - low;
            low = mid;
            reach = n;
        } else {
            width = mid - low - 1;
        }
    }
    __syncthreads();
    if (threadIdx.x == 0) found.count = 0;
    __syncthreads();
    const bool ties = reach > kMostCandidates;               // low is the k-th largest, and many equal it
    const int steps = row_steps<THREADS>(vocab);
    for (int q = 0; q < steps; ++q) {
        const int i = q * THREADS + static_cast<int>(threadIdx.x);
        const uint32_t order = order_of(load_value<G>(base, i));
        if (ties ? order > low : order >= low) put_candidate<false>(found, order, i);
    }
    __syncthreads();
    if (!ties) return;
    // One warp, in the order of the indexes.
    if (threadIdx.x < 32) {
        int have = found.count;
        for (int first = 0; first <= (vocab - 1) / 32 && have < k; ++first) {
            const int i = first * 32 + static_cast<int>(threadIdx.x);
            const bool equal = i < vocab && order_of(load_value<G>(base, i)) == low;
            const uint32_t who = __ballot_sync(0xffffffffu, equal);
            const int at = have + __popc(who & ((1u << threadIdx.x) - 1));
            if (equal && at < k) found.key[at] = static_cast<uint64_t>(low) << 32 | static_cast<uint32_t>(0x7fffffff - i);
            have += __popc(who);
        }
        __syncwarp();
        if (threadIdx.x == 0) found.count = min(have, k);
    }
    __syncthreads();
}

// FEW: more registers to a thread, fewer threads to an SM.
template <typename G, int THREADS, bool CLUSTER, bool FEW>
__global__ void __launch_bounds__(THREADS, FEW ? policy_blocks(THREADS) : row_blocks(THREADS)) star_alternatives_kernel(const __grid_constant__ AlternativesArgs a)
{
    constexpr int E = Granule<G>::kCount, kWarps = THREADS / 32, kStep = kBatch * THREADS;
    constexpr int kGroups = CLUSTER ? kMostGroups : THREADS;
    __shared__ alignas(16) float4 parts[CLUSTER ? 8 * kWarps : kWarps];  // of all warps
    __shared__ MaxSums row_sums;
    __shared__ uint32_t row_bound;
    __shared__ uint32_t group_order[kGroups];                    // the first block's
    __shared__ uint32_t slot_order[kSlots][THREADS];
    __shared__ unsigned short hits[kSlots * THREADS];
    __shared__ int n_hits, scratch;
    __shared__ Candidates found;                                 // the first block's
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const uint32_t blocks = CLUSTER ? cluster_size() : 1, rank = CLUSTER ? cluster_rank() : 0;
    const int log_blocks = CLUSTER ? 31 - __clz(static_cast<int>(blocks)) : 0;
    const int warps = kWarps << log_blocks;
    const float k = __fmul_rn(a.row.inv_temperature, kLog2e);
    const int vocab = static_cast<int>(a.row.vocab);
    launch_dependents();
    if constexpr (CLUSTER) cluster_sync();                       // the others have started
    wait_for_primary();

    for (int64_t t = blockIdx.x >> log_blocks; t < a.row.rows; t += gridDim.x >> log_blocks) {
        const char *base = static_cast<const char *>(a.row.logits) + t * a.row.ld * G::kBytes;
        const int64_t label = a.row.labels ? a.row.labels[t] : 0;
        const bool wanted = label >= 0 && label < vocab;         // vocab of 0: none
        MaxSums x{-INFINITY, 0.0f, 0.0f};
        float label_logit = 0.0f;
        if (wanted) {
            const RowSplit s = split_row<G>(base, vocab);
            const RowShare own = row_share(s.granules, rank, log_blocks);
            const uint4 *granules = reinterpret_cast<const uint4 *>(base + s.head * G::kBytes) + own.begin;
            const int edge_at = rank == 0 ? edge_element(s, threadIdx.x, vocab) : -1;
            const float edge = edge_at >= 0 ? load_value<G>(base, edge_at) : -INFINITY;
            if (threadIdx.x == THREADS - 1 && rank == 0 && a.logp) label_logit = load_value<G>(base, label);
            // Batches to a slot: a power of two.
            const int batches = (own.count + kStep - 1) / kStep, log_each = batches > kSlots ? 32 - __clz((batches - 1) / kSlots) : 0;
            int left = own.count - static_cast<int>(threadIdx.x), batch = 0;
            float most = -INFINITY;
            const uint4 *from = granules + threadIdx.x;
            for (; left > 0; left -= kStep, from += kStep) {
                const float m = left > kStep - THREADS ? take_batch_with_entropy<G, kBatch, THREADS, true>(&x, from, left, k)
                                                       : take_batch_with_entropy<G, kBatch, THREADS, false>(&x, from, left, k);
                most = fmaxf(most, m);
                ++batch;
                if ((batch & ((1 << log_each) - 1)) == 0) {
                    slot_order[(batch >> log_each) - 1][threadIdx.x] = order_of(most);
                    most = -INFINITY;
                }
            }
            if ((batch & ((1 << log_each) - 1)) != 0) slot_order[batch >> log_each][threadIdx.x] = order_of(most);
            const int slots = (batch + (1 << log_each) - 1) >> log_each;
            if (edge_at >= 0) x = take_one(x, edge, k);
            if (a.k > 0) {
                uint32_t group = order_of(x.m);
                if constexpr (CLUSTER) {
                    const uint32_t width = blocks / 2;
                    for (uint32_t o = 1; o < width; o *= 2) group = max(group, __shfl_xor_sync(0xffffffffu, group, o));
                    if (threadIdx.x % width == 0)
                        asm volatile("st.shared::cluster.u32 [%0], %1;" :: "r"(peer_address(smem_address(&group_order[(rank * THREADS + threadIdx.x) / width]), 0)), "r"(group) : "memory");
                } else {
                    group_order[threadIdx.x] = group;
                }
            }
            x = warp_join(x, k);
            if constexpr (CLUSTER) {
                if (lane == 0)
                    asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %3};" :: "r"(peer_address(smem_address(&parts[rank * kWarps + warp]), 0)),
                                 "f"(x.m), "f"(x.s), "f"(x.t) : "memory");
            } else if (lane == 0) {
                parts[warp] = make_float4(x.m, x.s, x.t, 0.0f);
            }
            if (threadIdx.x == 0) found.count = n_hits = 0;
            if constexpr (CLUSTER) cluster_sync(); else __syncthreads();
            // One warp joins the sums, another one finds the bound.
            if (warp == 0 && rank == 0) {
                const float4 none = make_float4(-INFINITY, 0.0f, 0.0f, 0.0f);
                const float4 part = lane < warps ? parts[lane] : none;
                x = MaxSums{part.x, part.y, part.z};
                if constexpr (CLUSTER) {
                    const float4 more = lane + 32 < warps ? parts[lane + 32] : none;
                    const float m = fmaxf(part.x, more.x);
                    x = add(move_to(x, m, k), move_to(MaxSums{more.x, more.y, more.z}, m, k));
                }
                x = warp_join(x, k);
                if (lane == 0) row_sums = x;
                if constexpr (CLUSTER) {
                    if (lane > 0 && lane < static_cast<int>(blocks))
                        asm volatile("st.shared::cluster.f32 [%0], %1;" :: "r"(peer_address(smem_address(&row_sums.s), lane)), "f"(x.s) : "memory");
                }
            }
            if (warp == 1 && rank == 0 && a.k > 0) {
                const uint32_t bound = max(bound_of<kGroups / 32>(group_order, CLUSTER ? 2 * THREADS : THREADS, a.k), kLowest + 1);
                if constexpr (CLUSTER) {
                    if (lane < static_cast<int>(blocks))
                        asm volatile("st.shared::cluster.u32 [%0], %1;" :: "r"(peer_address(smem_address(&row_bound), lane)), "r"(bound) : "memory");
                } else if (lane == 0) {
                    row_bound = bound;
                }
            }
            if constexpr (CLUSTER) cluster_sync(); else __syncthreads();
            x = row_sums;                                        // the first block's; another's has the sum alone
            // A second look at what reaches the bound.
            if (a.k > 0 && x.s > 0.0f && x.s < INFINITY) {
                const uint32_t bound = row_bound;
                const float least = logit_of(bound);
                if (edge_at >= 0 && order_of(edge) >= bound) put_candidate<CLUSTER>(found, order_of(edge), edge_at);
                for (int q = 0; q < slots; ++q)
                    if (slot_order[q][threadIdx.x] >= bound) hits[atomicAdd(&n_hits, 1)] = static_cast<unsigned short>(q * THREADS + threadIdx.x);
                __syncthreads();
                const int n = n_hits << (log_each + 2);          // granules
                for (int i = threadIdx.x; i < n; i += THREADS) {
                    const int hit = hits[i >> (log_each + 2)], slot = hit / THREADS;
                    const int g = hit % THREADS + ((slot << (log_each + 2)) + (i & ((4 << log_each) - 1))) * THREADS;
                    if (g >= own.count) continue;
                    const uint4 v = granules[g];
                    RunningMax<G> high;
                    high.take(v);
                    if (!(high.value() >= least)) continue;
                    Pair f[E / 2];
                    Granule<G>::widen(v, f);
                    uint32_t which = 0;
#pragma unroll
                    for (int e = 0; e < E / 2; ++e) {
                        float lo, hi;
                        split_pair(f[e], &lo, &hi);
                        which |= (lo >= least ? 1u : 0u) << (2 * e) | (hi >= least ? 2u : 0u) << (2 * e);
                    }
                    for (; which; which &= which - 1) {          // one, as a rule
                        const int e = __ffs(which) - 1;
                        put_candidate<CLUSTER>(found, order_of(load_value<G>(granules + g, e)), s.head + (own.begin + g) * E + e);
                    }
                }
                if constexpr (CLUSTER) cluster_sync(); else __syncthreads();
                if (rank == 0 && found.count > kMostCandidates) search_row<G, THREADS>(base, vocab, a.k, bound, order_of(x.m), found, &scratch);
            }
        }
        if (rank == 0) {                                         // the rest is the first block's
            const bool active = wanted && !(x.s == 0.0f), whole = active && x.s < INFINITY;
            if (threadIdx.x == THREADS - 1) {
                const float nan = x.s;                           // where the row has no sum
                if (a.logp) a.logp[t] = active ? log_prob(label_logit, MaxSum{x.m, x.s}, k, a.row.inv_temperature) : 0.0f;
                if (a.lse) a.lse[t] = active ? log_sum_exp(MaxSum{x.m, x.s}, a.row.inv_temperature) : -INFINITY;
                if (a.entropy) a.entropy[t] = whole ? __fsub_rn(logf(x.s), __fmul_rn(kLn2, __fdiv_rn(x.t, x.s))) : active ? nan : 0.0f;
            }
            if (a.k > 0) {
                const int n = whole ? found.count : 0, have = min(n, a.k);
                int32_t *ids = a.top_ids + t * a.ld_top;
                float *top = a.top_logp + t * a.ld_top;
                // Four lanes count a candidate's betters.
                for (int i = threadIdx.x / 4; i - static_cast<int>(threadIdx.x / 4) < n; i += THREADS / 4) {
                    const uint64_t key = i < n ? found.key[i] : 0;
                    int rank_of = 0;
                    for (int j = threadIdx.x % 4; j < n; j += 4) rank_of += found.key[j] > key ? 1 : 0;
                    rank_of += __shfl_xor_sync(0xffffffffu, rank_of, 1);
                    rank_of += __shfl_xor_sync(0xffffffffu, rank_of, 2);
                    if (i < n && rank_of < a.k && threadIdx.x % 4 == 0) {
                        const float f = logit_of(static_cast<uint32_t>(key >> 32));
                        ids[rank_of] = 0x7fffffff - static_cast<int32_t>(key & 0xffffffffu);
                        top[rank_of] = log_prob(f, MaxSum{x.m, x.s}, k, a.row.inv_temperature);
                    }
                }
                for (int i = have + threadIdx.x; i < a.k; i += THREADS) {
                    ids[i] = -1;
                    top[i] = active && !whole ? x.s : -INFINITY;
                }
            }
        }
        if (wanted) {                                            // what is shared has been read
            if constexpr (CLUSTER) cluster_sync(); else __syncthreads();
        }
    }
}

// ---------------------------------------------------------------------------
// The backward pass.  With u = z - lse and p = exp(u),
//     dlogits[j] = (sum of the gradients of what names j - p (G + h (u + H))) / temperature,
// G the sum of the gradients of a row's log-probabilities, h that of its entropy H.
// A block takes a row, or a part of one where there are few.  What the label or an
// alternative names is found out once for all of it, a thread to an entry; their
// elements' logits are read before anything is stored (the gradient may replace the
// logits) and their gradients stored after it.
//
// Bound by memory: 4096 x 50257 bf16 135 us with entropy, 6.1 TB/s; 151 with 64
// alternatives (a warp to each 1024 elements, which asked anew what names them, 174 and
// 228).
// ---------------------------------------------------------------------------
struct AlternativesGradArgs {
    RowArgs row;                 // labels may be null
    const float *lse, *entropy, *d_logp, *d_entropy;     // entropy and the gradients may be null
    int k;
    const int32_t *top_ids;
    const float *d_top;
    int64_t ld_top, ld_d_top;
    void *dlogits;
    int64_t ld_dlogits;
};

// What a row's dense part is made with.
struct AlternativesRow {
    float lse, inv_temperature;
    float plain, slope;          // -p (plain + slope u) / temperature
};
__device__ __forceinline__ float dense_gradient(float x, const AlternativesRow &r)
{
    const float u = fmaxf(__fmaf_rn(x, r.inv_temperature, -r.lse), -200.0f);
    return __fmul_rn(exp2_fast(__fmul_rn(u, kLog2e)), __fmaf_rn(r.slope, u, r.plain));
}

// Two elements.  The bound keeps 0 * -inf out.
__device__ __forceinline__ Pair dense_gradient(Pair x, const AlternativesRow &r)
{
    float lo, hi;
    split_pair(pair_fma(x, pair_of(r.inv_temperature), pair_of(-r.lse)), &lo, &hi);
    const Pair u = make_pair(fmaxf(lo, -200.0f), fmaxf(hi, -200.0f));
    return pair_mul(pair_exp2(pair_mul(u, pair_of(kLog2e))), pair_fma(pair_of(r.slope), u, pair_of(r.plain)));
}

template <typename G, int THREADS> __global__ void __launch_bounds__(THREADS, row_blocks(THREADS)) star_alternatives_backward_kernel(const __grid_constant__ AlternativesGradArgs a, int parts)
{
    constexpr int E = Granule<G>::kCount, P = Granule<G>::kPairs, kStep = kBatch * THREADS;
    __shared__ int4 id4[kMostAlternatives / 4];
    __shared__ float grads[kMostAlternatives], warp_sums[kMostAlternatives / 32];
    __shared__ int label_listed;
    const int *ids = reinterpret_cast<const int *>(id4);
    launch_dependents();
    wait_for_primary();
    const int vocab = static_cast<int>(a.row.vocab), lane = threadIdx.x % 32;
    for (int64_t item = blockIdx.x; item < a.row.rows * parts; item += gridDim.x) {
        const int64_t t = parts == 1 ? item : item / parts;
        const int part = static_cast<int>(item - t * parts);
        const char *base = static_cast<const char *>(a.row.logits) + t * a.row.ld * G::kBytes;
        char *out = static_cast<char *>(a.dlogits) + t * a.ld_dlogits * G::kBytes;
        const RowSplit s = split_row<G>(base, vocab);
        const int each = (s.granules + parts - 1) / parts, begin = min(each * part, s.granules), end = min(begin + each, s.granules);
        const int edge_at = part == 0 ? edge_element(s, threadIdx.x, vocab) : -1;
        const float lse = a.lse[t];
        const int64_t label = a.row.labels ? a.row.labels[t] : 0;
        const bool active = lse != -INFINITY && label >= 0 && label < vocab;
        const bool same_phase = (reinterpret_cast<uintptr_t>(out) - reinterpret_cast<uintptr_t>(base)) % 16 == 0;
        const auto here = [&](int id) {
            const int at = id - s.head;
            return id < s.head || id >= vocab - s.tail ? part == 0 : at >= begin * E && at < end * E;
        };
        AlternativesRow r{lse, a.row.inv_temperature, 0.0f, 0.0f};
        const float d_logp = active && a.d_logp ? a.d_logp[t] : 0.0f;
        // This thread's entry: the elements' logit and the gradients of all that names it.  -1: none, or none of its own.
        int named = -1;
        float logit = 0.0f, sum = 0.0f;
        if (active) {
            const float h = a.d_entropy ? a.d_entropy[t] : 0.0f;
            float all = d_logp;
            if (a.k > 0) {
                if (threadIdx.x < kMostAlternatives) {
                    int id = -1;
                    if (static_cast<int>(threadIdx.x) < a.k) {
                        id = a.top_ids[t * a.ld_top + threadIdx.x];
                        if (id < 0 || id >= vocab)
                            id = -1;
                        else
                            sum = a.d_top[t * a.ld_d_top + threadIdx.x];
                    }
                    const float total = warp_sum(sum);
                    if (lane == 0) warp_sums[threadIdx.x / 32] = total;
                    grads[threadIdx.x] = sum;
                    reinterpret_cast<int *>(id4)[threadIdx.x] = id;
                    named = id;
                }
                if (threadIdx.x == 0) label_listed = 0;
                __syncthreads();
                for (int w = 0; w * 32 < a.k; ++w) all = __fadd_rn(all, warp_sums[w]);
                if (named >= 0 && here(named)) {
                    // The first entry with an id takes the gradients of all of them.
                    const int mine = static_cast<int>(threadIdx.x);
                    for (int i = 0; i < a.k; i += 4) {
                        const int4 other = id4[i / 4];
                        if (other.x != named && other.y != named && other.z != named && other.w != named) continue;
                        for (int q = i; q < i + 4; ++q) {
                            if (ids[q] != named || q == mine) continue;
                            if (q < mine) named = -2;
                            sum = __fadd_rn(sum, grads[q]);
                        }
                        if (named < 0) break;
                    }
                    if (named >= 0) {
                        logit = load_value<G>(base, named);
                        if (a.d_logp && named == label) {
                            sum = __fadd_rn(sum, d_logp);
                            label_listed = 1;
                        }
                    }
                } else {
                    named = -1;
                }
            }
            if (threadIdx.x == THREADS - 1 && a.d_logp && here(static_cast<int>(label))) {
                named = static_cast<int>(label);
                logit = load_value<G>(base, named);
                sum = d_logp;
            }
            if (a.k > 0 || a.d_logp) __syncthreads();        // the named elements' logits are read
            float plain = h == 0.0f ? all : __fmaf_rn(h, a.entropy[t], all);
            if (lse != lse) plain = lse;                     // a NaN row's gradient is NaN
            r.plain = -__fmul_rn(plain, r.inv_temperature);
            r.slope = -__fmul_rn(h, r.inv_temperature);
        }
        const float edge = active && edge_at >= 0 ? load_value<G>(base, edge_at) : 0.0f;
        if (same_phase) {
            const uint4 *src = reinterpret_cast<const uint4 *>(base + s.head * G::kBytes) + begin + threadIdx.x;
            uint4 *dst = reinterpret_cast<uint4 *>(out + s.head * G::kBytes) + begin + threadIdx.x;
            for (int left = end - begin - static_cast<int>(threadIdx.x); left > 0; left -= kStep, src += kStep, dst += kStep) {
                if (!active) {
#pragma unroll
                    for (int q = 0; q < kBatch; ++q)
                        if (q * THREADS < left) dst[q * THREADS] = make_uint4(0, 0, 0, 0);
                    continue;
                }
                uint4 v[kBatch];
#pragma unroll
                for (int q = 0; q < kBatch; ++q)
                    if (q * THREADS < left) v[q] = src[q * THREADS];
#pragma unroll
                for (int q = 0; q < kBatch; ++q) {
                    if (q * THREADS < left) {
                        Pair g[P];
                        Granule<G>::widen(v[q], g);
#pragma unroll
                        for (int e = 0; e < P; ++e) g[e] = dense_gradient(g[e], r);
                        dst[q * THREADS] = Granule<G>::narrow(g);
                    }
                }
            }
        } else {
            // Without a sign: one beyond the last of 2^31 - 1 needs the 32nd bit.
            const unsigned last = s.head + end * E;
            for (unsigned at = s.head + begin * E + threadIdx.x; at < last; at += THREADS)
                store_value<G>(out, at, active ? dense_gradient(load_value<G>(base, at), r) : 0.0f);
        }
        if (edge_at >= 0) store_value<G>(out, edge_at, active ? dense_gradient(edge, r) : 0.0f);
        if (active && (a.k > 0 || a.d_logp)) {
            __syncthreads();                                 // the part is stored
            if (threadIdx.x == THREADS - 1 && a.k > 0 && label_listed) named = -1;
            if (named >= 0) store_value<G>(out, named, __fmaf_rn(sum, r.inv_temperature, dense_gradient(logit, r)));
            if (a.k > 0 && gridDim.x < a.row.rows * parts) __syncthreads();              // the list is read
        }
    }
}

}  // namespace star
