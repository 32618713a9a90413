// Entry points of the losses over the vocabulary: argument checks on the host,
// then the launches.
#include <algorithm>
#include <atomic>
#include <cmath>

#include "internal.h"
#include "losses.cuh"
#include "rows_host.h"

namespace star {

static std::atomic<int> g_wait_attempts{kWaitTries};
int wait_attempts() { return g_wait_attempts.load(std::memory_order_relaxed); }

}  // namespace star

namespace {

using namespace star;

// The rows' statistics.
//
// Threads to a row: as few as keep an SM busy, since a row's joins and the wait
// for its first loads cost the same for any number; but 128 or 256 for rows of
// more than 32 or 128 KB, whose last ones would otherwise be waited for.  More
// for fewer rows, until there are about 900 threads to an SM.  bf16, us:
//   rows x vocab      32 threads     64    128    256
//   16384 x  4000           29.8   34.3   39.5   51.5
//    4096 x 16000           26.1   28.9   27.0   30.8
//    4096 x 50257           72.1   74.9   68.2   70.3
//    4096 x 131072         177    184    165    161
//    2048 x  8192           11.2    9.6   10.6   12.2
//     512 x  8192            9.0    6.7    5.7    5.2
// Few long rows: clusters of blocks, up to four blocks of 256 threads to an SM.
// 1, 2, 4 and 8 blocks to a row:
//      64 x 50257            9.7    8.0    6.5    6.7
//     256 x 50257           11.0   10.2   12.6   17.5
//      64 x  8192            3.0    3.6    3.6    3.8   (16 KB: one block)
template <typename G, bool POLICY, int THREADS>
star_status_t launch_rows(const RowWork &a, int cluster, int *parts_out, cudaStream_t stream)
{
    static Held known;
    constexpr auto kernel = star_row_kernel<G, POLICY, THREADS>;
    int held = 0;
    const cudaError_t e = held_clusters(kernel, known, THREADS, cluster, 0, &held);
    if (e != cudaSuccess) return cuda_failed(e);
    // Blocks of a warp: as many as the device holds, each with many rows (16384 x
    // 200: 10.5 us, a block each 18.0).  Larger ones: a block each, which evens out
    // their ends and rows that are skipped (16384 x 50257 with 128 threads: 252 us,
    // as many as it holds 286).
    const int64_t most = THREADS == 32 ? held : int64_t{1} << 20, clusters = std::min(a.row.rows, most);
    *parts_out = static_cast<int>(clusters);
    return launch(kernel, dim3(static_cast<unsigned>(clusters * cluster)), THREADS, 0, dim3(static_cast<unsigned>(cluster)), stream, a);
}

template <typename G, bool POLICY> star_status_t walk_rows(const RowWork &a, int *parts_out, cudaStream_t stream)
{
    const int64_t granules = a.row.vocab * G::kBytes / 16;
    int cluster = 1, threads = granules <= 2048 ? 32 : granules <= 8192 ? 128 : 256;
    while (threads < 256 && threads < granules && a.row.rows * threads < 148 * 800) threads *= 2;
    while (granules > 2048 && cluster < 8 && a.row.rows * cluster * 2 <= 148 * 4 && granules / (cluster * 2) >= 448) cluster *= 2;
    switch (threads) {
    case 32: return launch_rows<G, POLICY, 32>(a, cluster, parts_out, stream);
    case 64: return launch_rows<G, POLICY, 64>(a, cluster, parts_out, stream);
    case 128: return launch_rows<G, POLICY, 128>(a, cluster, parts_out, stream);
    default: return launch_rows<G, POLICY, 256>(a, cluster, parts_out, stream);
    }
}

// The policy loss in one reading of the rows.
template <typename G, int THREADS, bool CLUSTER> star_status_t launch_policy(const RowWork &a, int cluster, int *parts_out, cudaStream_t stream)
{
    static Held known;
    constexpr auto kernel = star_policy_kernel<G, THREADS, CLUSTER>;
    const int64_t granules = a.row.vocab * G::kBytes / 16;
    const int kib = static_cast<int>(((granules + cluster - 1) / cluster * 16 + 1023) / 1024);
    int held = 0;
    const cudaError_t e = held_clusters(kernel, known, THREADS, cluster, kib, &held);
    if (e != cudaSuccess) return cuda_failed(e);
    const int64_t clusters = std::min<int64_t>(a.row.rows, held);
    *parts_out = static_cast<int>(clusters);
    return launch(kernel, dim3(static_cast<unsigned>(clusters * cluster)), THREADS, static_cast<size_t>(kib) * 1024, dim3(static_cast<unsigned>(cluster)), stream, a);
}

// Whether the policy loss is made in one reading, and the smallest block whose
// part of the SM's shared memory holds a row; rows of more than 112 KB are shared
// by a cluster of blocks.  Two readings where the second finds the logits in L2,
// up to 45 MB of them, and rows are too few to hide one another's waits.  The same
// with and without a gradient, so that both give the same bits.  us:
//     rows x vocab         one   two         rows x vocab            one   two
//      148 x 50257 bf16   15.7  14.5           600 x 32000 bf16     26.7  23.3
//      444 x 50257 bf16   30.0  28.6          1024 x 16000 bf16     23.5  22.0
//      600 x 50257 bf16   35.8  36.5          4096 x  1000 fp32     14.0  20.2
//     2048 x 50257 bf16   89.0   116           300 x 131072 bf16    43.6  48.9
//      200 x 50257 fp32   30.9  25.0          1024 x 131072 bf16     130   143
//      444 x 50257 fp32   44.3  52.2          1024 x 200000 fp32     318   385
// Clusters for rows that a block of 1024 threads could hold, 57500 bf16: 1024 rows
// 66.5 us against 71.4, 4096 rows 247 against 250.  And of 2 x 256 threads instead
// of a block of 512, 50257 bf16: 50.1 against 54.1 and 170 against 165: not taken.
bool one_reading(int64_t rows, int64_t vocab, int size, int *threads, int *cluster)
{
    const int64_t bytes = vocab * size;
    if (rows <= 1024 && bytes * rows <= 45'000'000) return false;
    *cluster = 1;
    for (int t : {32, 64, 128, 256, 512}) {
        *threads = t;
        if (bytes <= kKeepBytesPerThread * t) return true;
    }
    for (int t : {256, 512}) {
        *threads = t;
        for (int c : {4, 8}) {
            *cluster = c;
            if (bytes <= int64_t{kKeepBytesPerThread} * t * c) return true;
        }
    }
    return false;
}

template <typename G> star_status_t run_policy(const RowWork &a, int threads, int cluster, int *parts_out, cudaStream_t stream)
{
    if (cluster > 1)
        return threads == 256 ? launch_policy<G, 256, true>(a, cluster, parts_out, stream) : launch_policy<G, 512, true>(a, cluster, parts_out, stream);
    switch (threads) {
    case 32: return launch_policy<G, 32, false>(a, 1, parts_out, stream);
    case 64: return launch_policy<G, 64, false>(a, 1, parts_out, stream);
    case 128: return launch_policy<G, 128, false>(a, 1, parts_out, stream);
    case 256: return launch_policy<G, 256, false>(a, 1, parts_out, stream);
    default: return launch_policy<G, 512, false>(a, 1, parts_out, stream);
    }
}

// The gradient from what was kept of the rows.
template <bool POLICY> star_status_t launch_gradient(const GradArgs &g, star_dtype_t dtype, cudaStream_t stream)
{
    const int64_t per_row = g.row.vocab * dtype_size(dtype) / 16 / kGradGranules + 1;        // of a warp
    const int64_t most = 148 * 64, warps = kRowThreads / 32;
    const dim3 grid(static_cast<unsigned>(g.row.rows > most * warps / per_row ? most : (g.row.rows * per_row + warps - 1) / warps));
    return dtype == STAR_DTYPE_BF16 ? launch(star_row_gradient_kernel<GradBF16, POLICY>, grid, kRowThreads, 0, dim3(1), stream, g)
                                    : launch(star_row_gradient_kernel<GradF32, POLICY>, grid, kRowThreads, 0, dim3(1), stream, g);
}

}  // namespace

extern "C" star_status_t star_token_logprobs(const void *logits, star_dtype_t dtype, int64_t rows, int64_t vocab,
                                             int64_t ld, const int64_t *labels, float temperature, float *logp,
                                             float *lse, void *cuda_stream)
{
    RowWork a{};
    Extent read[2], written[2];
    star_status_t st = check_rows(logits, dtype, rows, vocab, ld, labels, temperature, &a.row, read);
    if (st == STAR_OK) st = check_vector(logp, rows, 4, false, &written[0]);
    if (st == STAR_OK) st = check_vector(lse, rows, 4, true, &written[1]);
    if (st == STAR_OK) st = check_disjoint(written, 2, read, 2);
    if (st != STAR_OK || rows == 0) return st;
    a.logp = logp;
    a.lse = lse;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    int clusters = 0;
    return dtype == STAR_DTYPE_BF16 ? walk_rows<GradBF16, false>(a, &clusters, stream) : walk_rows<GradF32, false>(a, &clusters, stream);
}

extern "C" star_status_t star_loss_workspace_bytes(int64_t rows, int64_t sequences, size_t *bytes_out)
{
    if (!bytes_out) return STAR_ERR_NULL_POINTER;
    if (rows < 0 || sequences < 0 || static_cast<uint64_t>(rows) > kMaxBytes / 16 ||
        static_cast<uint64_t>(sequences) > kMaxBytes / 16)
        return STAR_ERR_INVALID_ARG;
    // What is kept of every row, and the partial sums of up to as many blocks.
    *bytes_out = static_cast<size_t>(rows) * 32 + 16;
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
    RowWork a{};
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
    a.partial = static_cast<float4 *>(workspace);
    a.dlogits = dlogits;
    a.ld_dlogits = ld_dlogits;
    a.tries = wait_attempts();
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    const bool bf16 = dtype == STAR_DTYPE_BF16;
    int parts = 0, threads = 0, cluster = 1;
    const bool once = one_reading(rows, vocab, dtype_size(dtype), &threads, &cluster);
    if (once) {
        st = bf16 ? run_policy<GradBF16>(a, threads, cluster, &parts, stream) : run_policy<GradF32>(a, threads, cluster, &parts, stream);
    } else if (rows > 0) {
        if (dlogits) a.kept = reinterpret_cast<RowKept *>(a.partial + rows);
        st = bf16 ? walk_rows<GradBF16, true>(a, &parts, stream) : walk_rows<GradF32, true>(a, &parts, stream);
    }
    if (st != STAR_OK) return st;
    if (!once && rows > 0 && dlogits) {
        GradArgs g{};
        g.row = a.row;
        g.kept = a.kept;
        g.dlogits = dlogits;
        g.ld_dlogits = ld_dlogits;
        g.partial = a.partial;
        g.parts = parts;
        g.sums = sums;
        return launch_gradient<true>(g, dtype, stream);
    }
    return launch(star_policy_sums_kernel, dim3(1), kSumThreads, 0, dim3(1), stream, static_cast<const float4 *>(a.partial),
                  static_cast<int64_t>(parts), sums);
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
    if (rows > 0) {
        const bool bf16 = dtype == STAR_DTYPE_BF16;
        RowWork p{};
        p.row = a.row;
        p.kept = a.kept;
        int clusters = 0;
        st = bf16 ? walk_rows<GradBF16, false>(p, &clusters, stream) : walk_rows<GradF32, false>(p, &clusters, stream);
        if (st != STAR_OK) return st;
    }
    if (pairs > 0) {
        st = launch(star_preference_pair_kernel, dim3(static_cast<unsigned>(std::min<int64_t>(pairs, 65536))), kPairThreads, 0, dim3(1), stream, a);
        if (st != STAR_OK) return st;
    }
    if (!dlogits || rows == 0) return launch(star_preference_total_kernel, dim3(1), kPairThreads, 0, dim3(1), stream, a);
    GradArgs g{};
    g.row = a.row;
    g.kept = a.kept;
    g.dlogits = dlogits;
    g.ld_dlogits = ld_dlogits;
    g.pair_loss = pair_loss;
    g.pairs = pairs;
    g.loss_scale = loss_scale;
    g.loss = loss;
    return launch_gradient<false>(g, dtype, stream);
}

extern "C" star_status_t star_set_wait_attempts(int attempts)
{
    if (attempts < 0) return STAR_ERR_INVALID_ARG;
    g_wait_attempts.store(std::min(attempts, kWaitTries), std::memory_order_relaxed);
    return STAR_OK;
}

extern "C" star_status_t star_check_waits(void *cuda_stream)
{
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    cudaStreamCaptureStatus capturing = cudaStreamCaptureStatusNone;
    cudaError_t e = cudaStreamIsCapturing(stream, &capturing);
    if (e != cudaSuccess) return cuda_failed(e);
    if (capturing != cudaStreamCaptureStatusNone) return STAR_ERR_UNSUPPORTED;
    int here = 0, there = 0, distillation = 0;
    e = take_expired(stream, &here);
    if (e == cudaSuccess) e = weight_grad_expired(stream, &there);
    if (e == cudaSuccess) e = distillation_expired(stream, &distillation);
    if (e != cudaSuccess) return cuda_failed(e);
    return here || there || distillation ? STAR_ERR_TIMEOUT : STAR_OK;
}
