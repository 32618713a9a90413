// Entry points of the losses over the vocabulary: argument checks on the host,
// then the launches.
#include <cmath>

#include "internal.h"
#include "losses.cuh"

namespace {

using namespace star;

// Blocks of a grid over `rows` rows (every kernel strides over the rest).
int row_grid(int64_t rows) { return static_cast<int>(rows < 148 * 64 ? rows : 148 * 64); }

// The checks that the three operators share.  read[0] is the logits' extent.
star_status_t check_rows(const void *logits, star_dtype_t dtype, int64_t rows, int64_t vocab, int64_t ld,
                         const int64_t *labels, float temperature, RowArgs *out, Extent *read)
{
    if (!is_dtype(dtype) || vocab < 0) return STAR_ERR_INVALID_ARG;
    if (!(temperature > 0.0f) || !std::isfinite(temperature) || !std::isfinite(1.0f / temperature) ||
        !std::isfinite(1.0f / temperature * kLog2e))
        return STAR_ERR_INVALID_ARG;
    star_status_t st = check_matrix(logits, rows, vocab, ld, dtype_size(dtype), &read[0]);
    if (st == STAR_OK) st = check_vector(labels, rows, 8, false, &read[1]);
    if (st != STAR_OK) return st;
    *out = RowArgs{logits, ld, rows, vocab, labels, nullptr, 1.0f / temperature};
    return STAR_OK;
}

// dlogits: its own memory, or exactly the logits.
star_status_t check_gradient(const void *dlogits, int64_t ld_dlogits, star_dtype_t dtype, const RowArgs &row,
                             const Extent &logits, Extent *out)
{
    *out = Extent{};
    if (!dlogits) return STAR_OK;
    const star_status_t st = check_matrix(dlogits, row.rows, row.vocab, ld_dlogits, dtype_size(dtype), out);
    if (st != STAR_OK) return st;
    const bool in_place = dlogits == row.logits && (ld_dlogits == row.ld || row.rows <= 1);
    return !in_place && overlap(*out, logits) ? STAR_ERR_INVALID_ARG : STAR_OK;
}

// No written buffer may share memory with a read one or another written one.
star_status_t check_disjoint(const Extent *written, int n_written, const Extent *read, int n_read)
{
    for (int i = 0; i < n_written; ++i)
        if (overlaps_any(written[i], read, n_read) || overlaps_any(written[i], written, i)) return STAR_ERR_INVALID_ARG;
    return STAR_OK;
}

star_status_t check_workspace(const void *workspace, size_t have, int64_t rows, int64_t sequences, Extent *out)
{
    size_t need = 0;
    const star_status_t st = star_loss_workspace_bytes(rows, sequences, &need);
    if (st != STAR_OK) return st;
    if (!workspace) return STAR_ERR_NULL_POINTER;
    if (reinterpret_cast<uintptr_t>(workspace) % 16 != 0) return STAR_ERR_INVALID_ARG;
    if (have < need) return STAR_ERR_WORKSPACE_TOO_SMALL;
    *out = extent(workspace, need);
    return STAR_OK;
}

}  // namespace

extern "C" star_status_t star_token_logprobs(const void *logits, star_dtype_t dtype, int64_t rows, int64_t vocab,
                                             int64_t ld, const int64_t *labels, float temperature, float *logp,
                                             float *lse, void *cuda_stream)
{
    LogprobArgs a{};
    Extent read[2], written[2];
    star_status_t st = check_rows(logits, dtype, rows, vocab, ld, labels, temperature, &a.row, read);
    if (st == STAR_OK) st = check_vector(logp, rows, 4, false, &written[0]);
    if (st == STAR_OK) st = check_vector(lse, rows, 4, true, &written[1]);
    if (st == STAR_OK) st = check_disjoint(written, 2, read, 2);
    if (st != STAR_OK || rows == 0) return st;
    a.logp = logp;
    a.lse = lse;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (dtype == STAR_DTYPE_BF16)
        star_logprob_kernel<GradBF16><<<row_grid(rows), kRowThreads, 0, stream>>>(a);
    else
        star_logprob_kernel<GradF32><<<row_grid(rows), kRowThreads, 0, stream>>>(a);
    return launched();
}

extern "C" star_status_t star_loss_workspace_bytes(int64_t rows, int64_t sequences, size_t *bytes_out)
{
    if (!bytes_out) return STAR_ERR_NULL_POINTER;
    if (rows < 0 || sequences < 0 || static_cast<uint64_t>(rows) > kMaxBytes / 16 ||
        static_cast<uint64_t>(sequences) > kMaxBytes / 16)
        return STAR_ERR_INVALID_ARG;
    *bytes_out = static_cast<size_t>(rows) * 16 + 16;
    return STAR_OK;
}

extern "C" star_status_t star_policy_loss(const void *logits, star_dtype_t dtype, int64_t rows, int64_t vocab,
                                          int64_t ld, const int64_t *labels, const float *weights,
                                          const float *advantages, const float *old_logp, const float *ref_logp,
                                          float temperature, float clip_low, float clip_high, float kl_coef,
                                          float *logp, float *token_loss, float *sums, void *dlogits,
                                          int64_t ld_dlogits, void *workspace, size_t workspace_bytes,
                                          void *cuda_stream)
{
    if (!(clip_low >= 0.0f && clip_low <= 1.0f) || !(clip_high >= 0.0f) || !std::isfinite(kl_coef))
        return STAR_ERR_INVALID_ARG;
    PolicyArgs a{};
    Extent read[6], written[5];
    star_status_t st = check_rows(logits, dtype, rows, vocab, ld, labels, temperature, &a.row, read);
    if (st == STAR_OK) st = check_vector(weights, rows, 4, true, &read[2]);
    if (st == STAR_OK) st = check_vector(advantages, rows, 4, false, &read[3]);
    if (st == STAR_OK) st = check_vector(old_logp, rows, 4, true, &read[4]);
    if (st == STAR_OK) st = check_vector(ref_logp, rows, 4, true, &read[5]);
    if (st == STAR_OK) st = check_vector(logp, rows, 4, false, &written[0]);
    if (st == STAR_OK) st = check_vector(token_loss, rows, 4, false, &written[1]);
    if (st == STAR_OK) st = check_vector(sums, 4, 4, false, &written[2]);
    if (st == STAR_OK) st = check_workspace(workspace, workspace_bytes, rows, 0, &written[3]);
    if (st == STAR_OK) st = check_disjoint(written, 4, read, 6);
    if (st == STAR_OK) st = check_gradient(dlogits, ld_dlogits, dtype, a.row, read[0], &written[4]);
    if (st == STAR_OK && (overlaps_any(written[4], read + 1, 5) || overlaps_any(written[4], written, 4)))
        st = STAR_ERR_INVALID_ARG;
    if (st != STAR_OK) return st;
    a.row.weights = weights;
    a.advantages = advantages;
    a.old_logp = old_logp;
    a.ref_logp = ref_logp;
    a.clip_low = clip_low;
    a.clip_high = clip_high;
    a.kl_coef = kl_coef;
    a.logp = logp;
    a.token_loss = token_loss;
    a.terms = static_cast<float4 *>(workspace);
    a.dlogits = dlogits;
    a.ld_dlogits = ld_dlogits;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (rows > 0) {
        if (dtype == STAR_DTYPE_BF16)
            star_policy_kernel<GradBF16><<<row_grid(rows), kRowThreads, 0, stream>>>(a);
        else
            star_policy_kernel<GradF32><<<row_grid(rows), kRowThreads, 0, stream>>>(a);
        st = launched();
        if (st != STAR_OK) return st;
    }
    star_policy_sums_kernel<<<1, kSumThreads, 0, stream>>>(a.terms, rows, sums);
    return launched();
}

extern "C" star_status_t star_preference_loss(const void *logits, star_dtype_t dtype, int64_t rows, int64_t vocab,
                                              int64_t ld, const int64_t *labels, const int32_t *seq_offsets,
                                              int64_t pairs, const float *ref_seq_logp, float temperature, float beta,
                                              float label_smoothing, int average, float loss_scale, float *seq_logp,
                                              float *pair_loss, float *margin, float *loss, void *dlogits,
                                              int64_t ld_dlogits, void *workspace, size_t workspace_bytes,
                                              void *cuda_stream)
{
    if (!std::isfinite(beta) || !std::isfinite(loss_scale) || !(label_smoothing >= 0.0f && label_smoothing <= 1.0f) ||
        pairs < 0 || pairs > (int64_t{1} << 30))
        return STAR_ERR_INVALID_ARG;
    PreferenceArgs a{};
    Extent read[4], written[6];
    star_status_t st = check_rows(logits, dtype, rows, vocab, ld, labels, temperature, &a.row, read);
    if (st == STAR_OK) st = check_vector(seq_offsets, 2 * pairs + 1, 4, false, &read[2]);
    if (st == STAR_OK) st = check_vector(ref_seq_logp, 2 * pairs, 4, true, &read[3]);
    if (st == STAR_OK) st = check_vector(seq_logp, 2 * pairs, 4, false, &written[0]);
    if (st == STAR_OK) st = check_vector(pair_loss, pairs, 4, false, &written[1]);
    if (st == STAR_OK) st = check_vector(margin, pairs, 4, false, &written[2]);
    if (st == STAR_OK) st = check_vector(loss, 1, 4, false, &written[3]);
    if (st == STAR_OK) st = check_workspace(workspace, workspace_bytes, rows, 2 * pairs, &written[4]);
    if (st == STAR_OK) st = check_disjoint(written, 5, read, 4);
    if (st == STAR_OK) st = check_gradient(dlogits, ld_dlogits, dtype, a.row, read[0], &written[5]);
    if (st == STAR_OK && (overlaps_any(written[5], read + 1, 3) || overlaps_any(written[5], written, 5)))
        st = STAR_ERR_INVALID_ARG;
    if (st != STAR_OK) return st;
    a.kept = static_cast<RowKept *>(workspace);
    a.seq_offsets = seq_offsets;
    a.pairs = pairs;
    a.ref_seq_logp = ref_seq_logp;
    a.beta = beta;
    a.smoothing = label_smoothing;
    a.loss_scale = loss_scale;
    a.average = average;
    a.seq_logp = seq_logp;
    a.pair_loss = pair_loss;
    a.margin = margin;
    a.loss = loss;
    a.dlogits = dlogits;
    a.ld_dlogits = ld_dlogits;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    const bool bf16 = dtype == STAR_DTYPE_BF16;
    if (rows > 0) {
        LogprobArgs p{};
        p.row = a.row;
        p.kept = a.kept;
        if (bf16)
            star_logprob_kernel<GradBF16><<<row_grid(rows), kRowThreads, 0, stream>>>(p);
        else
            star_logprob_kernel<GradF32><<<row_grid(rows), kRowThreads, 0, stream>>>(p);
        if ((st = launched()) != STAR_OK) return st;
    }
    if (pairs > 0) {
        star_preference_pair_kernel<<<static_cast<int>(pairs < 65536 ? pairs : 65536), kPairThreads, 0, stream>>>(a);
        if ((st = launched()) != STAR_OK) return st;
    }
    if (dlogits && rows > 0) {
        if (bf16)
            star_preference_grad_kernel<GradBF16><<<row_grid(rows), kRowThreads, 0, stream>>>(a);
        else
            star_preference_grad_kernel<GradF32><<<row_grid(rows), kRowThreads, 0, stream>>>(a);
    } else {
        star_preference_total_kernel<<<1, kPairThreads, 0, stream>>>(a);
    }
    return launched();
}
