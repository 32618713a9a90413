// Entry points of the root-mean-square norm: argument checks on the host, then
// the launches.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "checkpoint_host.h"
#include "norm.cuh"
#include "rows_host.h"

namespace {

using namespace star;

// Rows of sums that a backward pass may write: eight blocks on each of 148 SMs.
constexpr int64_t kMostParts = 148 * 8;

// The gain: a vector in its own type, or none.
star_status_t check_gain(const void *gain, star_dtype_t dtype, int64_t cols, Extent *out)
{
    *out = Extent{};
    if (!gain) return STAR_OK;
    if (!is_dtype(dtype)) return STAR_ERR_INVALID_ARG;
    return check_vector(gain, cols, dtype_size(dtype), false, out);
}

// An optional checkpoint: both buffers or neither.
star_status_t check_optional_kept(const int8_t *codes, const uint8_t *scales, int64_t rows, int64_t cols, Kept *out, Extent *at)
{
    at[0] = at[1] = Extent{};
    if (!codes && !scales) return STAR_OK;
    return check_kept(codes, scales, rows, cols, out, at);
}

// Whether every row of an optional matrix starts on a boundary of `bytes`.
bool on_grid(const void *p, int64_t ld, int size, int bytes)
{
    return !p || (reinterpret_cast<uintptr_t>(p) % static_cast<unsigned>(bytes) == 0 && (ld * size) % bytes == 0);
}

constexpr int kBackEach = 2;

// The threads that share a row, `each` columns to one: the next power of two.
int row_threads(int64_t cols, int each)
{
    int t = 32;
    while (t < 1024 && cols > int64_t{t} * each) t *= 2;
    return t;
}

// f with the number of threads at compile time, of those between LEAST and MOST.
template <int LEAST, int MOST, typename F> star_status_t with_threads(int threads, F f)
{
    if constexpr (LEAST < MOST)
        if (threads > LEAST) return with_threads<LEAST * 2, MOST>(threads, f);
    return f(std::integral_constant<int, LEAST>());
}

// How a row falls to threads: whole pieces of 16 bytes, single columns, or in turns.
enum Way { kPieces, kColumns, kLong };

template <typename G> star_status_t run_norm(const NormArgs &a, Way way, cudaStream_t stream)
{
    const auto blocks = [&](int threads) {
        const int block = norm_block(threads);
        return dim3(static_cast<unsigned>(std::min<int64_t>((a.rows * threads + block - 1) / block, 148 * 32)));
    };
    const int64_t cols = a.cols;
    if (way == kPieces) {
        // Half a block of 32 to a thread, or one: 4096 x 8192 bf16 49.7 and 43.2 us, 8192 x 4096 fp32 79.9 and 84.6.
        if (cols <= 4096)
            return with_threads<32, 256>(row_threads(cols, 16), [&](auto t) {
                return launch(star_rms_norm_kernel<G, decltype(t)::value, 1>, blocks(t), norm_block(t), 0, dim3(1), stream, a);
            });
        return with_threads<256, 512>(row_threads(cols, 32), [&](auto t) {
            return launch(star_rms_norm_kernel<G, decltype(t)::value, 2>, blocks(t), norm_block(t), 0, dim3(1), stream, a);
        });
    }
    if (way == kColumns) {
        if (cols <= 128) return launch(star_rms_norm_columns_kernel<G, 32, 4>, blocks(32), norm_block(32), 0, dim3(1), stream, a);
        if (cols <= 8192)
            return with_threads<32, 1024>(row_threads(cols, 8), [&](auto t) {
                return launch(star_rms_norm_columns_kernel<G, decltype(t)::value, 8>, blocks(t), norm_block(t), 0, dim3(1), stream, a);
            });
        return launch(star_rms_norm_columns_kernel<G, 1024, 16>, blocks(1024), 1024, 0, dim3(1), stream, a);
    }
    return launch(star_rms_norm_long_kernel<G>, dim3(static_cast<unsigned>(std::min<int64_t>(a.rows, 148 * 32))), kNormThreads, 0, dim3(1), stream, a);
}

// Blocks that stay, each with a row of sums: as many as the GPU holds.
template <int THREADS, typename Kernel>
star_status_t launch_backward(Kernel kernel, Held &known, int kib, const NormGradArgs &a, int64_t *parts, cudaStream_t stream)
{
    constexpr int kBlock = norm_block(THREADS);
    int held = 0;
    const cudaError_t e = held_clusters(kernel, known, kBlock, 1, kib, &held);
    if (e != cudaSuccess) return cuda_failed(e);
    *parts = std::min<int64_t>({(a.rows * THREADS + kBlock - 1) / kBlock, held, kMostParts});
    return launch(kernel, dim3(static_cast<unsigned>(*parts)), kBlock, static_cast<size_t>(kib) * 1024, dim3(1), stream, a);
}

template <typename G, bool KEPT> star_status_t run_backward(const NormGradArgs &a, Way way, int64_t *parts, cudaStream_t stream)
{
    const int64_t cols = a.cols;
    if (way == kPieces)
        return with_threads<32, 1024>(row_threads(cols, kBackEach * 16 / G::kBytes), [&](auto t) {
            constexpr int kThreads = decltype(t)::value;
            // Rows on their way: 16384 x 4096 bf16 with 2, 3 and 4 of them 88.4, 89.1, 90.0 us, 8192 x 4096 fp32 88.6, 82.2, 89.2.
            constexpr int kStages = G::kBytes == 4 && kThreads <= 512 ? 3 : 2;
            constexpr int kKib = (NormRing<G, KEPT, kBackEach, kStages>::kThread * norm_block(kThreads) + 1023) / 1024;
            static Held known;
            return launch_backward<kThreads>(star_rms_norm_backward_kernel<G, KEPT, kThreads, kBackEach, kStages>, known, kKib, a, parts, stream);
        });
    // Four columns to a thread, or eight where a block has no more threads: 4096 x 4095 66.4 and 103 us.  (Forward the
    // other way round, 130 and 89.5.)
    if (way == kColumns && cols <= 4096)
        return with_threads<32, 1024>(row_threads(cols, 4), [&](auto t) {
            constexpr int kThreads = decltype(t)::value;
            static Held known;
            return launch_backward<kThreads>(star_rms_norm_backward_columns_kernel<G, KEPT, kThreads, 4>, known, 0, a, parts, stream);
        });
    if (way == kColumns) {
        static Held known;
        return launch_backward<1024>(star_rms_norm_backward_columns_kernel<G, KEPT, 1024, 8>, known, 0, a, parts, stream);
    }
    *parts = std::min(a.rows, kMostParts);
    return launch(star_rms_norm_backward_long_kernel<G>, dim3(static_cast<unsigned>(*parts)), kNormThreads, 0, dim3(1), stream, a);
}

bool same(const void *a, int64_t ld_a, const void *b, int64_t ld_b, int64_t rows) { return a == b && (ld_a == ld_b || rows <= 1); }

}  // namespace

extern "C" star_status_t star_rms_norm(void *y, int64_t ld_y, const void *x, int64_t ld_x, const void *residual, int64_t ld_residual,
                                       void *total, int64_t ld_total, star_dtype_t dtype, int64_t rows, int64_t cols,
                                       const void *gain, star_dtype_t gain_dtype, float eps, float *rstd, int8_t *codes,
                                       uint8_t *scales, void *cuda_stream)
{
    if (!is_dtype(dtype) || !(eps > 0.0f) || !std::isfinite(eps)) return STAR_ERR_INVALID_ARG;
    if (rows > 0x7fffffff || cols > 0x7fffffff - 64) return STAR_ERR_UNSUPPORTED;
    const int size = dtype_size(dtype);
    NormArgs a{};
    Extent read[3], written[5];
    star_status_t st = check_matrix(x, rows, cols, ld_x, size, &read[0]);
    if (st == STAR_OK && residual) st = check_matrix(residual, rows, cols, ld_residual, size, &read[1]);
    if (st == STAR_OK) st = check_gain(gain, gain_dtype, cols, &read[2]);
    if (st == STAR_OK) st = check_matrix(y, rows, cols, ld_y, size, &written[0]);
    if (st == STAR_OK) st = check_vector(rstd, rows, 4, true, &written[1]);
    if (st == STAR_OK) st = check_optional_kept(codes, scales, rows, cols, &a.kept, &written[2]);
    if (st == STAR_OK && total) st = check_matrix(total, rows, cols, ld_total, size, &written[4]);
    if (st != STAR_OK) return st;
    for (int i = 0; i < 4; ++i)
        if (overlaps_any(written[i], read, 3) || overlaps_any(written[i], written, i)) return STAR_ERR_INVALID_ARG;
    // The stream may replace x or the residual.
    if (overlaps_any(written[4], written, 4) || overlap(written[4], read[2]) ||
        (overlap(written[4], read[0]) && !same(total, ld_total, x, ld_x, rows)) ||
        (overlap(written[4], read[1]) && !same(total, ld_total, residual, ld_residual, rows)))
        return STAR_ERR_INVALID_ARG;
    if (rows == 0 || cols == 0) return STAR_OK;
    a.x = x;
    a.residual = residual;
    a.total = total;
    a.y = y;
    a.gain = gain;
    a.rstd = rstd;
    a.ld_x = ld_x;
    a.ld_residual = ld_residual;
    a.ld_total = ld_total;
    a.ld_y = ld_y;
    a.rows = rows;
    a.cols = static_cast<int>(cols);
    a.eps = eps;
    a.inv_cols = 1.0 / static_cast<double>(cols);
    a.gain_wide = gain_dtype == STAR_DTYPE_F32;
    const auto grid = [&](int bytes) {
        return on_grid(x, ld_x, size, bytes) && on_grid(residual, ld_residual, size, bytes) && on_grid(total, ld_total, size, bytes) &&
               on_grid(y, ld_y, size, bytes);
    };
    a.wide = grid(32);
    const Way way = cols > 16384 ? kLong : grid(16) ? kPieces : kColumns;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    return dtype == STAR_DTYPE_BF16 ? run_norm<GradBF16>(a, way, stream) : run_norm<GradF32>(a, way, stream);
}

extern "C" star_status_t star_rms_norm_workspace_bytes(int64_t rows, int64_t cols, size_t *bytes_out)
{
    if (!bytes_out) return STAR_ERR_NULL_POINTER;
    if (rows < 0 || cols < 0 || static_cast<uint64_t>(cols) > kMaxBytes / 16 / kMostParts) return STAR_ERR_INVALID_ARG;
    *bytes_out = static_cast<size_t>(std::min(rows, kMostParts)) * static_cast<size_t>(cols) * 4 + 16;
    return STAR_OK;
}

extern "C" star_status_t star_rms_norm_backward(void *dx, int64_t ld_dx, void *dgain, star_dtype_t dgain_dtype, int accumulate,
                                                const void *dy, int64_t ld_dy, const void *total, int64_t ld_total,
                                                const int8_t *codes, const uint8_t *scales, const void *d_total,
                                                int64_t ld_d_total, star_dtype_t dtype, int64_t rows, int64_t cols,
                                                const void *gain, star_dtype_t gain_dtype, const float *rstd, void *workspace,
                                                size_t workspace_bytes, void *cuda_stream)
{
    if (!is_dtype(dtype) || (total && (codes || scales))) return STAR_ERR_INVALID_ARG;
    if (dgain && !is_dtype(dgain_dtype)) return STAR_ERR_INVALID_ARG;
    if (rows > 0x7fffffff || cols > 0x7fffffff - 64) return STAR_ERR_UNSUPPORTED;
    const int size = dtype_size(dtype);
    NormGradArgs a{};
    Extent read[7], written[3];
    star_status_t st = check_matrix(dy, rows, cols, ld_dy, size, &read[0]);
    if (st == STAR_OK && d_total) st = check_matrix(d_total, rows, cols, ld_d_total, size, &read[1]);
    if (st == STAR_OK && (total || !(codes || scales))) st = check_matrix(total, rows, cols, ld_total, size, &read[2]);
    if (st == STAR_OK) st = check_optional_kept(codes, scales, rows, cols, &a.kept, &read[3]);
    if (st == STAR_OK) st = check_gain(gain, gain_dtype, cols, &read[5]);
    if (st == STAR_OK) st = check_vector(rstd, rows, 4, false, &read[6]);
    if (st == STAR_OK) st = check_matrix(dx, rows, cols, ld_dx, size, &written[0]);
    if (st == STAR_OK && dgain) st = check_vector(dgain, cols, dtype_size(dgain_dtype), false, &written[1]);
    size_t need = 0;
    if (st == STAR_OK) st = star_rms_norm_workspace_bytes(rows, cols, &need);
    if (st != STAR_OK) return st;
    if (dgain) {
        if (!workspace) return STAR_ERR_NULL_POINTER;
        if (reinterpret_cast<uintptr_t>(workspace) % 16 != 0) return STAR_ERR_INVALID_ARG;
        if (workspace_bytes < need) return STAR_ERR_WORKSPACE_TOO_SMALL;
        written[2] = extent(workspace, need);
    }
    for (int i = 1; i < 3; ++i)
        if (overlaps_any(written[i], read, 7) || overlaps_any(written[i], written, i)) return STAR_ERR_INVALID_ARG;
    // dx may replace dy or d_total.
    if (overlaps_any(written[0], read + 2, 5) || (overlap(written[0], read[0]) && !same(dx, ld_dx, dy, ld_dy, rows)) ||
        (overlap(written[0], read[1]) && !same(dx, ld_dx, d_total, ld_d_total, rows)))
        return STAR_ERR_INVALID_ARG;
    if (cols == 0) return STAR_OK;
    a.dx = dx;
    a.dy = dy;
    a.total = total;
    a.gain = gain;
    a.rstd = rstd;
    a.d_total = d_total;
    a.ld_dx = ld_dx;
    a.ld_dy = ld_dy;
    a.ld_total = ld_total;
    a.ld_d_total = ld_d_total;
    a.rows = rows;
    a.cols = static_cast<int>(cols);
    a.inv_cols = 1.0 / static_cast<double>(cols);
    a.gain_wide = gain_dtype == STAR_DTYPE_F32;
    a.partial = dgain ? static_cast<float *>(workspace) : nullptr;
    const auto grid = [&](int bytes) {
        return on_grid(dx, ld_dx, size, bytes) && on_grid(dy, ld_dy, size, bytes) && on_grid(total, ld_total, size, bytes) &&
               on_grid(d_total, ld_d_total, size, bytes);
    };
    a.wide = grid(32);
    const Way way = grid(16) && cols <= 1024 * kBackEach * 16 / size ? kPieces : cols <= 1024 * 8 ? kColumns : kLong;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    int64_t parts = 0;
    if (rows > 0) {
        if (dtype == STAR_DTYPE_BF16)
            st = total ? run_backward<GradBF16, false>(a, way, &parts, stream) : run_backward<GradBF16, true>(a, way, &parts, stream);
        else
            st = total ? run_backward<GradF32, false>(a, way, &parts, stream) : run_backward<GradF32, true>(a, way, &parts, stream);
        if (st != STAR_OK) return st;
    }
    if (!dgain) return STAR_OK;
    const dim3 gain_grid(static_cast<unsigned>(std::min<int64_t>((cols + 31) / 32, 148 * 16)));
    const float *partial = static_cast<const float *>(workspace);
    int gain_threads = 32;                               // four rows of sums to a warp, up to 32 warps
    while (gain_threads < kGainThreads && gain_threads / 8 < parts) gain_threads *= 2;
    return dgain_dtype == STAR_DTYPE_BF16
               ? launch(star_rms_norm_gain_kernel<GradBF16>, gain_grid, gain_threads, 0, dim3(1), stream, partial, parts, a.cols, dgain, accumulate)
               : launch(star_rms_norm_gain_kernel<GradF32>, gain_grid, gain_threads, 0, dim3(1), stream, partial, parts, a.cols, dgain, accumulate);
}
