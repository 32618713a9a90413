// Entry points of log-probabilities with entropy and top alternatives: argument
// checks on the host, then one launch.
#include <algorithm>

#include "alternatives.cuh"
#include "rows_host.h"

namespace {

using namespace star;

static_assert(kMostAlternatives == STAR_MAX_ALTERNATIVES, "the kernels' and the interface's limit");

// The checks of k and of the matrices of alternatives; ids may not be missing where k > 0.
star_status_t check_top(const void *p, int64_t rows, int k, int64_t ld, Extent *out)
{
    *out = Extent{};
    return k > 0 ? check_matrix(p, rows, k, ld, 4, out) : STAR_OK;
}

}  // namespace

extern "C" star_status_t star_token_alternatives(const void *logits, star_dtype_t dtype, int64_t rows, int64_t vocab, int64_t ld,
                                                 const int64_t *labels, float temperature, int k, int32_t *top_ids,
                                                 float *top_logp, int64_t ld_top, float *logp, float *lse, float *entropy,
                                                 void *cuda_stream)
{
    if (k < 0) return STAR_ERR_INVALID_ARG;
    if (k > kMostAlternatives) return STAR_ERR_UNSUPPORTED;
    AlternativesArgs a{};
    Extent read[2], written[5];
    star_status_t st = check_rows(logits, dtype, rows, vocab, ld, labels, temperature, &a.row, read, true);
    if (st == STAR_OK) st = check_top(top_ids, rows, k, ld_top, &written[0]);
    if (st == STAR_OK) st = check_top(top_logp, rows, k, ld_top, &written[1]);
    if (st == STAR_OK) st = check_vector(logp, rows, 4, true, &written[2]);
    if (st == STAR_OK) st = check_vector(lse, rows, 4, true, &written[3]);
    if (st == STAR_OK) st = check_vector(entropy, rows, 4, true, &written[4]);
    if (st == STAR_OK && logp && !labels && rows > 0) st = STAR_ERR_NULL_POINTER;
    if (st == STAR_OK) st = check_disjoint(written, 5, read, 2);
    if (st != STAR_OK || rows == 0) return st;
    a.k = k;
    a.top_ids = top_ids;
    a.top_logp = top_logp;
    a.ld_top = ld_top;
    a.logp = logp;
    a.lse = lse;
    a.entropy = entropy;
    constexpr int kThreads = 256;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    const dim3 grid(static_cast<unsigned>(std::min<int64_t>(rows, int64_t{1} << 20)));
    return dtype == STAR_DTYPE_BF16 ? launch(star_alternatives_kernel<GradBF16, kThreads>, grid, kThreads, 0, dim3(1), stream, a)
                                    : launch(star_alternatives_kernel<GradF32, kThreads>, grid, kThreads, 0, dim3(1), stream, a);
}

extern "C" star_status_t star_token_alternatives_backward(void *dlogits, int64_t ld_dlogits, const void *logits, star_dtype_t dtype,
                                                          int64_t rows, int64_t vocab, int64_t ld, const int64_t *labels,
                                                          float temperature, const float *lse, const float *entropy,
                                                          const float *d_logp, const float *d_entropy, int k,
                                                          const int32_t *top_ids, int64_t ld_top, const float *d_top_logp,
                                                          int64_t ld_d_top, void *cuda_stream)
{
    if (k < 0) return STAR_ERR_INVALID_ARG;
    if (k > kMostAlternatives) return STAR_ERR_UNSUPPORTED;
    AlternativesGradArgs a{};
    Extent read[8], written;
    star_status_t st = check_rows(logits, dtype, rows, vocab, ld, labels, temperature, &a.row, read, true);
    if (st == STAR_OK) st = check_vector(lse, rows, 4, false, &read[2]);
    if (st == STAR_OK) st = check_vector(entropy, rows, 4, d_entropy == nullptr, &read[3]);
    if (st == STAR_OK) st = check_vector(d_logp, rows, 4, true, &read[4]);
    if (st == STAR_OK) st = check_vector(d_entropy, rows, 4, true, &read[5]);
    if (st == STAR_OK) st = check_top(top_ids, rows, k, ld_top, &read[6]);
    if (st == STAR_OK) st = check_top(d_top_logp, rows, k, ld_d_top, &read[7]);
    if (st == STAR_OK && d_logp && !labels && rows > 0) st = STAR_ERR_NULL_POINTER;
    if (st == STAR_OK && !dlogits && rows > 0 && vocab > 0) st = STAR_ERR_NULL_POINTER;
    if (st == STAR_OK) st = check_gradient(dlogits, ld_dlogits, dtype, a.row, read[0], &written);
    if (st == STAR_OK && overlaps_any(written, read + 1, 7)) st = STAR_ERR_INVALID_ARG;
    if (st != STAR_OK || rows == 0 || vocab == 0) return st;
    a.lse = lse;
    a.entropy = entropy;
    a.d_logp = d_logp;
    a.d_entropy = d_entropy;
    a.k = k;
    a.top_ids = top_ids;
    a.d_top = d_top_logp;
    a.ld_top = ld_top;
    a.ld_d_top = ld_d_top;
    a.dlogits = dlogits;
    a.ld_dlogits = ld_dlogits;
    const int64_t per_row = vocab * dtype_size(dtype) / 16 / kAltGranules + 1;           // of a warp
    const int64_t most = 148 * 64, warps = kAltThreads / 32;
    const dim3 grid(static_cast<unsigned>(rows > most * warps / per_row ? most : (rows * per_row + warps - 1) / warps));
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    return dtype == STAR_DTYPE_BF16 ? launch(star_alternatives_backward_kernel<GradBF16>, grid, kAltThreads, 0, dim3(1), stream, a)
                                    : launch(star_alternatives_backward_kernel<GradF32>, grid, kAltThreads, 0, dim3(1), stream, a);
}
