// Device code of the losses over the vocabulary (sm_100a).
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "rows.cuh"

namespace star {

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
