// Entry points of the root-mean-square norm: argument checks on the host, then
// the launches.
#include <algorithm>
#include <cmath>

#include "checkpoint_host.h"
#include "norm.cuh"

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
    a.inv_cols = static_cast<float>(1.0 / static_cast<double>(cols));
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    const dim3 grid(static_cast<unsigned>(std::min<int64_t>(rows, 148 * 32)));
    const bool wide_gain = gain_dtype == STAR_DTYPE_F32;
    if (dtype == STAR_DTYPE_BF16)
        return wide_gain ? launch(star_rms_norm_loose_kernel<GradBF16, GradF32>, grid, kNormThreads, 0, dim3(1), stream, a)
                         : launch(star_rms_norm_loose_kernel<GradBF16, GradBF16>, grid, kNormThreads, 0, dim3(1), stream, a);
    return wide_gain ? launch(star_rms_norm_loose_kernel<GradF32, GradF32>, grid, kNormThreads, 0, dim3(1), stream, a)
                     : launch(star_rms_norm_loose_kernel<GradF32, GradBF16>, grid, kNormThreads, 0, dim3(1), stream, a);
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
    a.inv_cols = static_cast<float>(1.0 / static_cast<double>(cols));
    a.partial = dgain ? static_cast<float *>(workspace) : nullptr;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    const int64_t parts = std::min(rows, kMostParts);
    if (rows > 0) {
        const dim3 grid(static_cast<unsigned>(parts));
        const bool wide_gain = gain_dtype == STAR_DTYPE_F32;
        if (dtype == STAR_DTYPE_BF16)
            st = wide_gain ? launch(star_rms_norm_backward_loose_kernel<GradBF16, GradF32>, grid, kNormThreads, 0, dim3(1), stream, a)
                           : launch(star_rms_norm_backward_loose_kernel<GradBF16, GradBF16>, grid, kNormThreads, 0, dim3(1), stream, a);
        else
            st = wide_gain ? launch(star_rms_norm_backward_loose_kernel<GradF32, GradF32>, grid, kNormThreads, 0, dim3(1), stream, a)
                           : launch(star_rms_norm_backward_loose_kernel<GradF32, GradBF16>, grid, kNormThreads, 0, dim3(1), stream, a);
        if (st != STAR_OK) return st;
    }
    if (!dgain) return STAR_OK;
    const dim3 grid(static_cast<unsigned>(std::min<int64_t>((cols + 31) / 32, 148 * 16)));
    const float *partial = static_cast<const float *>(workspace);
    return dgain_dtype == STAR_DTYPE_BF16
               ? launch(star_rms_norm_gain_kernel<GradBF16>, grid, kGainThreads, 0, dim3(1), stream, partial, parts, a.cols, dgain, accumulate)
               : launch(star_rms_norm_gain_kernel<GradF32>, grid, kGainThreads, 0, dim3(1), stream, partial, parts, a.cols, dgain, accumulate);
}
