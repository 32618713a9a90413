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

template <typename G, int THREADS, bool CLUSTER, bool FEW> star_status_t launch_rows(const AlternativesArgs &a, int cluster, cudaStream_t stream)
{
    const int64_t clusters = std::min<int64_t>(a.row.rows, int64_t{1} << 20);
    return launch(star_alternatives_kernel<G, THREADS, CLUSTER, FEW>, dim3(static_cast<unsigned>(clusters * cluster)), THREADS, 0,
                  dim3(static_cast<unsigned>(cluster)), stream, a);
}

// Threads to a row: few for short rows, as for the rows' statistics (walk_rows of the
// losses), but at least two groups of them to an alternative, four in rows where the
// second look costs less than what it finds; more where there are few rows.  us:
//     rows x vocab, k            64 threads    128    256
//     16384 x  4000,  8  bf16          63.8   80.9    132
//     16384 x  4000, 64  bf16                  153    193
//      4096 x 16000, 20  bf16          44.1   42.0   55.1
//      4096 x 50257,  8  bf16                 87.7   97.3
//      4096 x 50257, 64  bf16                  126    116
//      2048 x 50257, 64  fp32                  125   95.4
// Few long rows: clusters of up to eight blocks, half a block to an SM in all, one or two
// of longer rows, beyond which some wait for others to end.  us by blocks to a row, k = 20:
//     rows x vocab        1      2      4      8  taken
//      1 x  20011 bf16   5.3    6.4    5.8    5.8     1
//      9 x  32001 bf16   6.4    7.5    6.5    6.2     8
//     74 x  32001 bf16   8.0    9.1    9.8   13.4     1
//      9 x  50257 bf16   8.6    8.4    7.3    6.6     8
//     37 x  50257 bf16   9.3    9.0    8.4    9.4     4
//    148 x  50257 bf16  10.1   11.2   15.8   22.9     1
//     37 x 128256 bf16  15.2   12.6   11.3   11.0     8
//    148 x 128256 bf16  21.8   18.4   23.5   29.1     2
//    296 x 128256 bf16  24.7   23.6   36.6   50.0     2
//     74 x  32001 fp32   8.2    7.9    8.9   13.0     4
//    148 x  32001 fp32  10.6    9.4   14.8   20.9     2
// And 64 registers to a thread instead of 48 while all blocks fit the GPU at once:
// 400 x 50257, 20 bf16 20.2 -> 16.7 us.
template <typename G> star_status_t run_rows(const AlternativesArgs &a, cudaStream_t stream)
{
    const int64_t granules = a.row.vocab * G::kBytes / 16;
    const int64_t most = granules < 6000 ? 148 / 2 : granules < 8000 ? 148 : 148 * 2;
    int cluster = 1;
    while (granules >= 3600 && cluster < 8 && a.row.rows * cluster * 2 <= (cluster == 1 && granules >= 12000 ? 148 * 4 : most)) cluster *= 2;
    if (cluster > 1) return launch_rows<G, 256, true, true>(a, cluster, stream);
    int threads = granules <= 2048 ? 64 : granules <= 8192 ? 128 : 256;
    while (threads < 256 && (threads < (granules > 2048 ? 4 : 2) * a.k || (threads < granules && a.row.rows * threads < 148 * 800))) threads *= 2;
    switch (threads) {
    case 64: return launch_rows<G, 64, false, false>(a, 1, stream);
    case 128: return launch_rows<G, 128, false, false>(a, 1, stream);
    default: return a.row.rows <= 148 * 4 ? launch_rows<G, 256, false, true>(a, 1, stream) : launch_rows<G, 256, false, false>(a, 1, stream);
    }
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
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    return dtype == STAR_DTYPE_BF16 ? run_rows<GradBF16>(a, stream) : run_rows<GradF32>(a, stream);
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
    // Blocks to a row: until every SM has five, as long as each has a step of its own.  Half a block for short
    // rows, if it has a thread for the label beside the alternatives'.
    const int64_t granules = vocab * dtype_size(dtype) / 16;
    const bool small = granules <= 1024 && k < 128;
    int64_t parts = 1;
    while (parts * 2 * kBatch * 256 <= granules && rows * parts < 148 * 5) parts *= 2;
    const dim3 grid(static_cast<unsigned>(std::min<int64_t>(rows * parts, 0x7fffffff)));
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    const int n = static_cast<int>(parts);
    if (dtype == STAR_DTYPE_BF16)
        return small ? launch(star_alternatives_backward_kernel<GradBF16, 128>, grid, 128, 0, dim3(1), stream, a, n)
                     : launch(star_alternatives_backward_kernel<GradBF16, 256>, grid, 256, 0, dim3(1), stream, a, n);
    return small ? launch(star_alternatives_backward_kernel<GradF32, 128>, grid, 128, 0, dim3(1), stream, a, n)
                 : launch(star_alternatives_backward_kernel<GradF32, 256>, grid, 256, 0, dim3(1), stream, a, n);
}
