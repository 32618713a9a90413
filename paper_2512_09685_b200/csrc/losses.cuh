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

struct PolicyArgs {
    RowArgs row;
    const float *advantages;
    const float *old_logp;       // may be null
    const float *ref_logp;       // may be null
    float clip_low, clip_high, kl_coef;
    float *logp;
    float *token_loss;
    float4 *terms;               // per row: the weighted terms of the four sums
    void *dlogits;               // may be null
    int64_t ld_dlogits;
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

// ---------------------------------------------------------------------------
// One block per row, three walks over it.
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
__device__ void row_gradient(const RowArgs &a, int64_t t, MaxSum row, int64_t label, float coef, void *dlogits, int64_t ld)
{
    const float k = __fmul_rn(a.inv_temperature, kLog2e);
    const char *src = static_cast<const char *>(a.logits) + t * a.ld * G::kBytes;
    char *dst = static_cast<char *>(dlogits) + t * ld * G::kBytes;
    const float scale = __fdiv_rn(-coef, row.s);
    for (int64_t j = threadIdx.x; j < a.vocab; j += blockDim.x) {
        float g = __fmul_rn(scale, exp2_fast(__fmul_rn(__fsub_rn(load_value<G>(src, j), row.m), k)));
        if (j == label) g = __fadd_rn(g, coef);
        store_value<G>(dst, j, g);
    }
}

template <typename G> __device__ void row_zero(const RowArgs &a, int64_t t, void *dlogits, int64_t ld)
{
    char *dst = static_cast<char *>(dlogits) + t * ld * G::kBytes;
    for (int64_t j = threadIdx.x; j < a.vocab; j += blockDim.x) store_value<G>(dst, j, 0.0f);
}

template <typename G> __global__ void __launch_bounds__(kRowThreads) star_policy_kernel(const __grid_constant__ PolicyArgs a)
{
    __shared__ MaxSum shared[kRowThreads / 32];
    for (int64_t t = blockIdx.x; t < a.row.rows; t += gridDim.x) {
        int64_t label;
        float weight;
        bool active = row_wanted(a.row, t, &label, &weight);
        MaxSum row{0.0f, 0.0f};
        if (active) row = row_stats<G>(a.row, t, shared);
        active = active && !(row.s == 0.0f);
        PolicyRow r{0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
        float lp = 0.0f;
        if (active) {
            const float x = load_value<G>(static_cast<const char *>(a.row.logits) + t * a.row.ld * G::kBytes, label);
            lp = log_prob(x, row, a.row.inv_temperature);
            r = policy_row(lp, a.advantages[t], a.old_logp != nullptr, a.old_logp ? a.old_logp[t] : 0.0f,
                           a.ref_logp != nullptr, a.ref_logp ? a.ref_logp[t] : 0.0f, a.clip_low, a.clip_high,
                           a.kl_coef, weight, a.row.inv_temperature);
        }
        __syncthreads();                                 // the label's logit is read: the row may be overwritten
        if (threadIdx.x == 0) {
            a.logp[t] = lp;
            a.token_loss[t] = r.loss;
            a.terms[t] = active ? make_float4(weight * r.loss, -weight * r.gain, weight * r.kl, weight * r.clipped)
                                : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        }
        if (a.dlogits) {
            if (active)
                row_gradient<G>(a.row, t, row, label, r.coef, a.dlogits, a.ld_dlogits);
            else
                row_zero<G>(a.row, t, a.dlogits, a.ld_dlogits);
        }
    }
}

constexpr int kSumThreads = 512;

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

// sums[0 .. 4) from the rows' terms, one block.
__global__ void __launch_bounds__(kSumThreads) star_policy_sums_kernel(const float4 *terms, int64_t n, float *sums)
{
    __shared__ double shared[kSumThreads / 32];
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
// Log-probabilities alone, and the preference loss in three steps: the rows'
// log-probabilities; per pair the loss and every row's factor; the gradient.
// ---------------------------------------------------------------------------

// What the preference loss keeps of a row between its steps.
struct RowKept {
    float m;         // largest logit
    float inv_s;     // 1 / sum of exp(z - z_max); 0 for an inactive row
    float logp;
    float coef;
};

struct LogprobArgs {
    RowArgs row;
    float *logp;                 // may be null
    float *lse;                  // may be null
    RowKept *kept;               // may be null
};

template <typename G> __global__ void __launch_bounds__(kRowThreads) star_logprob_kernel(const __grid_constant__ LogprobArgs a)
{
    __shared__ MaxSum shared[kRowThreads / 32];
    for (int64_t t = blockIdx.x; t < a.row.rows; t += gridDim.x) {
        int64_t label;
        float weight;
        bool active = row_wanted(a.row, t, &label, &weight);
        MaxSum row{0.0f, 0.0f};
        if (active) row = row_stats<G>(a.row, t, shared);
        active = active && !(row.s == 0.0f);
        if (threadIdx.x == 0) {
            float lp = 0.0f, lse = 0.0f;
            if (active) {
                const float x = load_value<G>(static_cast<const char *>(a.row.logits) + t * a.row.ld * G::kBytes, label);
                lp = log_prob(x, row, a.row.inv_temperature);
                lse = log_sum_exp(row, a.row.inv_temperature);
            }
            if (a.logp) a.logp[t] = lp;
            if (a.lse) a.lse[t] = lse;
            if (a.kept) a.kept[t] = RowKept{row.m, active ? __fdiv_rn(1.0f, row.s) : 0.0f, lp, 0.0f};
        }
    }
}

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
    preference_total(a, shared);
}

template <typename G> __global__ void __launch_bounds__(kRowThreads) star_preference_grad_kernel(const __grid_constant__ PreferenceArgs a)
{
    __shared__ double shared[kRowThreads / 32];
    if (blockIdx.x == 0) preference_total(a, shared);
    for (int64_t t = blockIdx.x; t < a.row.rows; t += gridDim.x) {
        const RowKept r = a.kept[t];
        if (r.inv_s != 0.0f && r.coef != 0.0f)
            row_gradient<G>(a.row, t, MaxSum{r.m, __fdiv_rn(1.0f, r.inv_s)}, a.row.labels[t], r.coef, a.dlogits, a.ld_dlogits);
        else
            row_zero<G>(a.row, t, a.dlogits, a.ld_dlogits);
    }
}

}  // namespace star
