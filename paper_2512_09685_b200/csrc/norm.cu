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

// The threads that share a row, `each` columns to one: the next power of two.  0: a
// row is too long for a block.
int row_threads(int64_t cols, int each)
{
    for (int t : {32, 64, 128, 256, 512, 1024})
        if (cols <= int64_t{t} * each) return t;
    return 0;
}

template <typename F> star_status_t with_threads(int threads, F f)
{
    switch (threads) {
    case 32: return f(std::integral_constant<int, 32>());
    case 64: return f(std::integral_constant<int, 64>());
    case 128: return f(std::integral_constant<int, 128>());
    case 256: return f(std::integral_constant<int, 256>());
    case 512: return f(std::integral_constant<int, 512>());
    default: return f(std::integral_constant<int, 1024>());
    }
}

template <typename G, int EACH> star_status_t run_norm(const NormArgs &a, int threads, cudaStream_t stream)
{
    if (threads == 0)
        return launch(star_rms_norm_loose_kernel<G>, dim3(static_cast<unsigned>(std::min<int64_t>(a.rows, 148 * 32))), kNormThreads, 0, dim3(1), stream, a);
    return with_threads(threads, [&](auto t) {
        constexpr int kThreads = decltype(t)::value, kBlock = norm_block(kThreads);
        const int64_t blocks = (a.rows * kThreads + kBlock - 1) / kBlock;
        return launch(star_rms_norm_kernel<G, kThreads, EACH>, dim3(static_cast<unsigned>(std::min<int64_t>(blocks, 148 * 32))), kBlock, 0, dim3(1), stream, a);
    });
}

template <typename G, bool KEPT> star_status_t run_backward(const NormGradArgs &a, int threads, int64_t *parts, cudaStream_t stream)
{
    if (threads == 0) {
        *parts = std::min(a.rows, kMostParts);
        return launch(star_rms_norm_backward_loose_kernel<G>, dim3(static_cast<unsigned>(*parts)), kNormThreads, 0, dim3(1), stream, a);
    }
    return with_threads(threads, [&](auto t) {
        constexpr int kThreads = decltype(t)::value, kBlock = norm_block(kThreads);
        constexpr int kStages = G::kBytes == 4 && kThreads <= 512 ? 3 : 2;
        constexpr int kKib = (NormRing<G, KEPT, kBackEach, kStages>::kThread * kBlock + 1023) / 1024;
        static Held known;
        int held = 0;
        constexpr auto kernel = star_rms_norm_backward_kernel<G, KEPT, kThreads, kBackEach, kStages>;
        const cudaError_t e = held_clusters(kernel, known, kBlock, 1, kKib, &held);
        if (e != cudaSuccess) return cuda_failed(e);
        *parts = std::min<int64_t>({(a.rows * kThreads + kBlock - 1) / kBlock, held, kMostParts});
        return launch(kernel, dim3(static_cast<unsigned>(*parts)), kBlock, kKib * 1024, dim3(1), stream, a);
    });
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
    const int each = cols <= 4096 ? 1 : 2, threads = grid(16) ? row_threads(cols, each * 16) : 0;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (each == 1) return dtype == STAR_DTYPE_BF16 ? run_norm<GradBF16, 1>(a, threads, stream) : run_norm<GradF32, 1>(a, threads, stream);
    return dtype == STAR_DTYPE_BF16 ? run_norm<GradBF16, 2>(a, threads, stream) : run_norm<GradF32, 2>(a, threads, stream);
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
    const int threads = grid(16) ? row_threads(cols, kBackEach * 16 / size) : 0;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    int64_t parts = 0;
    if (rows > 0) {
        if (dtype == STAR_DTYPE_BF16)
            st = total ? run_backward<GradBF16, false>(a, threads, &parts, stream) : run_backward<GradBF16, true>(a, threads, &parts, stream);
        else
            st = total ? run_backward<GradF32, false>(a, threads, &parts, stream) : run_backward<GradF32, true>(a, threads, &parts, stream);
        if (st != STAR_OK) return st;
    }
    if (!dgain) return STAR_OK;
    const dim3 gain_grid(static_cast<unsigned>(std::min<int64_t>((cols + 31) / 32, 148 * 16)));
    const float *partial = static_cast<const float *>(workspace);
    return dgain_dtype == STAR_DTYPE_BF16
               ? launch(star_rms_norm_gain_kernel<GradBF16>, gain_grid, kGainThreads, 0, dim3(1), stream, partial, parts, a.cols, dgain, accumulate)
               : launch(star_rms_norm_gain_kernel<GradF32>, gain_grid, kGainThreads, 0, dim3(1), stream, partial, parts, a.cols, dgain, accumulate);
}
