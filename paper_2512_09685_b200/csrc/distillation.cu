// Entry point of the distillation loss: argument checks on the host, then the
// launches.
#include <algorithm>
#include <cmath>

#include "distillation.cuh"
#include "rows_host.h"

namespace star {

cudaError_t distillation_expired(cudaStream_t stream, int *expired) { return take_expired(stream, expired); }

}  // namespace star

namespace {

using namespace star;

static_assert(kMostListed == STAR_MAX_ALTERNATIVES, "the kernels' and the interface's limit");

template <typename G, int THREADS, int MODE>
star_status_t launch_loss(const DistillArgs &a, int cluster, int *parts_out, cudaStream_t stream)
{
    static Held known;
    constexpr auto kernel = star_distillation_kernel<G, THREADS, MODE>;
    const int64_t granules = a.row.vocab * G::kBytes / 16;
    const int kib = static_cast<int>(((granules + cluster - 1) / cluster * 16 + 1023) / 1024);
    int held = 0;
    const cudaError_t e = held_clusters(kernel, known, THREADS, cluster, kib, &held, kDistillBytesPerThread);
    if (e != cudaSuccess) return cuda_failed(e);
    const int64_t clusters = std::min<int64_t>(a.row.rows, held);
    *parts_out = static_cast<int>(clusters);
    // Rows in order of taking part, where some may not, every block has a few, and there is enough to do to make up
    // for finding it, whether or not any are masked; us as they come -> in order:
    //                             35 % masked        none
    //      4096 x  12000 bf16     51.4 ->  47.2    51.8 ->  57.4     98 MB: not taken
    //      8192 x  12200 bf16     95.7 ->  83.0    99.0 ->   109    200 MB
    //     65536 x   2000 bf16      551 ->   376     454 ->   508
    //      2048 x  50257 bf16     87.3 ->  85.1    94.3 ->  97.8
    //      8192 x  50257 bf16      304 ->   275     340 ->   349
    //      1024 x  50257 fp32     83.1 ->  83.8    93.6 ->  97.2    206 MB, clusters of two
    //      2048 x 131072 bf16      291 ->   244     324 ->   328    clusters of four
    DistillArgs work = a;
    if ((!a.row.labels && !a.row.weights) || a.row.rows < 4 * clusters || a.row.rows > kMostOrdered ||
        a.row.rows * a.row.vocab * G::kBytes < 200'000'000) {
        work.order = nullptr;
    } else {
        const star_status_t st = launch(star_distillation_order_kernel, dim3(1), kOrderThreads, 0, dim3(1), stream, a.row, work.order);
        if (st != STAR_OK) return st;
    }
    return launch(kernel, dim3(static_cast<unsigned>(clusters * cluster)), THREADS, static_cast<size_t>(kib) * 1024, dim3(static_cast<unsigned>(cluster)), stream, work);
}

template <typename G, int MODE> star_status_t run_threads(const DistillArgs &a, int threads, int cluster, int *parts_out, cudaStream_t stream)
{
    switch (threads) {
    case 128: return launch_loss<G, 128, MODE>(a, cluster, parts_out, stream);
    case 256: return launch_loss<G, 256, MODE>(a, cluster, parts_out, stream);
    default: return launch_loss<G, 512, MODE>(a, cluster, parts_out, stream);
    }
}

template <typename G> star_status_t run_mode(const DistillArgs &a, int threads, int cluster, int *parts_out, cudaStream_t stream)
{
    const float inv_t = a.row.inv_temperature;
    if (a.hard == 0.0f || inv_t == 1.0f) return run_threads<G, kOne>(a, threads, cluster, parts_out, stream);
    if (inv_t == 0.5f) return run_threads<G, kSquare>(a, threads, cluster, parts_out, stream);
    if (inv_t == 0.25f) return run_threads<G, kFourth>(a, threads, cluster, parts_out, stream);
    return run_threads<G, kTwo>(a, threads, cluster, parts_out, stream);
}

// The smallest block whose part of the SM's shared memory holds a row, or a cluster
// of them; the cluster's blocks may take an SM's shared memory each.  Where there are few
// rows, more threads to one: 302 x 3071 bf16 with 128, 256 and 512 threads 9.0, 8.4 and 10
// to 13 us (256 taken), 1 x 6661 with 128 and 512 8.2 and 7.5; 590 x 3071 with 128 and 256
// 11.8 and 12.0.  And clusters of more blocks for few long rows; us by blocks to a row:
//     rows x vocab        1      2      4      8  taken
//      9 x  32001 bf16  10.0   11.7   10.9   10.8     1
//      1 x  50257 bf16  10.9   11.2   10.7   10.2     8
//      9 x  50257 bf16  11.1   11.7   11.1   10.6     8
//     18 x  50257 bf16  12.1   13.1   12.3   13.0     4
//     37 x  50257 bf16  12.1   13.0   12.8   17.9     1   (the GPU does not hold as many clusters of 8 at once)
//      9 x 100001 bf16         13.4   11.7   11.1     8
//     18 x 100001 bf16         13.9   12.2   12.3     4
//     37 x 100001 bf16         14.2   13.8   19.1     2
bool shape(int64_t rows, int64_t vocab, int size, int *threads, int *cluster)
{
    const int64_t bytes = vocab * size;
    *cluster = 1;
    *threads = 512;
    for (int t : {512, 256, 128})
        if (bytes <= int64_t{kDistillBytesPerThread} * t) *threads = t;
    while (*cluster < 8 && bytes > int64_t{kDistillBytesPerThread} * *threads * *cluster) *cluster *= 2;
    while (*threads < 512 && rows * *threads < 148 * 512 && bytes > 16 * *threads) *threads *= 2;
    while (*cluster < 8 && rows * *cluster * 2 < 148 / 2 && bytes >= 98304) *cluster *= 2;
    return bytes <= int64_t{kDistillBytesPerThread} * 1024 * *cluster;
}

}  // namespace

extern "C" star_status_t star_distillation_loss(const void *logits, star_dtype_t dtype, int64_t rows, int64_t vocab, int64_t ld,
                                                const int32_t *teacher_ids, int64_t ld_ids, const float *teacher_values,
                                                int64_t ld_values, int k, int rest, float teacher_temperature,
                                                const int64_t *labels, const float *weights, float temperature, float soft_coef,
                                                float label_coef, float *token_loss, float *sums, void *dlogits,
                                                int64_t ld_dlogits, void *workspace, size_t workspace_bytes, void *cuda_stream)
{
    if (k < 0 || !std::isfinite(soft_coef) || !std::isfinite(label_coef) || !(teacher_temperature > 0.0f) ||
        !std::isfinite(teacher_temperature) || !std::isfinite(1.0f / teacher_temperature))
        return STAR_ERR_INVALID_ARG;
    if (k > kMostListed) return STAR_ERR_UNSUPPORTED;
    DistillArgs a{};
    Extent read[5], written[4];
    star_status_t st = check_rows(logits, dtype, rows, vocab, ld, labels, temperature, &a.row, read, label_coef == 0.0f);
    if (st == STAR_OK) st = check_vector(weights, rows, 4, true, &read[2]);
    if (st == STAR_OK && k > 0) st = check_matrix(teacher_ids, rows, k, ld_ids, 4, &read[3]);
    if (st == STAR_OK && k > 0) st = check_matrix(teacher_values, rows, k, ld_values, 4, &read[4]);
    if (st == STAR_OK) st = check_vector(token_loss, rows, 4, false, &written[0]);
    if (st == STAR_OK) st = check_vector(sums, 4, 4, false, &written[1]);
    if (st == STAR_OK) st = check_workspace(workspace, workspace_bytes, rows, 0, &written[2]);
    if (st == STAR_OK) st = check_disjoint(written, 3, read, 5);
    if (st == STAR_OK) st = check_gradient(dlogits, ld_dlogits, dtype, a.row, read[0], &written[3]);
    if (st == STAR_OK && (overlaps_any(written[3], read + 1, 4) || overlaps_any(written[3], written, 3))) st = STAR_ERR_INVALID_ARG;
    if (st != STAR_OK) return st;
    int threads = 0, cluster = 0, parts = 0;
    if (rows > 0x3fffffff || !shape(rows, vocab, dtype_size(dtype), &threads, &cluster)) return STAR_ERR_UNSUPPORTED;
    a.row.weights = weights;
    a.ids = teacher_ids;
    a.values = teacher_values;
    a.ld_ids = ld_ids;
    a.ld_values = ld_values;
    a.k = k;
    a.rest = rest != 0;
    a.inv_teacher_temperature = 1.0f / teacher_temperature;
    a.soft = soft_coef;
    a.hard = label_coef;
    a.token_loss = token_loss;
    a.partial = static_cast<float4 *>(workspace);
    a.order = reinterpret_cast<int32_t *>(a.partial + rows);     // 4 bytes for each row and 4 more: there are 16 and 16
    a.dlogits = dlogits;
    a.ld_dlogits = ld_dlogits;
    a.tries = wait_attempts();
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (rows > 0) {
        st = dtype == STAR_DTYPE_BF16 ? run_mode<GradBF16>(a, threads, cluster, &parts, stream) : run_mode<GradF32>(a, threads, cluster, &parts, stream);
        if (st != STAR_OK) return st;
    }
    int sum_threads = 32;
    while (sum_threads < kDistillSumThreads && sum_threads * 2 <= parts) sum_threads *= 2;
    return launch(star_distillation_sums_kernel, dim3(1), sum_threads, 0, dim3(1), stream, static_cast<const float4 *>(a.partial),
                  static_cast<int64_t>(parts), sums);
}
