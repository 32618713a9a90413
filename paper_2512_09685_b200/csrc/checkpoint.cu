// Entry points of activations kept in 8 bits: argument checks on the host, then
// one kernel launch.
#include <type_traits>

#include "checkpoint.cuh"
#include "checkpoint_host.h"

namespace {

using namespace star;

bool is_act(int act) { return act >= STAR_ACT_NONE && act <= STAR_ACT_SILU; }

int grid_for(int64_t work) { return static_cast<int>(work < 1 ? 1 : work < 148 * 32 ? work : 148 * 32); }

// Calls f with the activation as a compile-time number.
template <typename F> void with_act(int act, F f)
{
    switch (act) {
    case STAR_ACT_GELU_TANH: f(std::integral_constant<int, STAR_ACT_GELU_TANH>()); break;
    case STAR_ACT_GELU_ERF: f(std::integral_constant<int, STAR_ACT_GELU_ERF>()); break;
    case STAR_ACT_SILU: f(std::integral_constant<int, STAR_ACT_SILU>()); break;
    default: f(std::integral_constant<int, STAR_ACT_NONE>()); break;
    }
}

}  // namespace

extern "C" star_status_t star_checkpoint_sizes(int64_t rows, int64_t cols, int64_t *pitch_out, size_t *code_bytes_out,
                                               size_t *scale_bytes_out)
{
    if (!pitch_out || !code_bytes_out || !scale_bytes_out) return STAR_ERR_NULL_POINTER;
    const int64_t most = int64_t{1} << 52;
    if (rows < 0 || cols < 0 || rows > most || cols > most) return STAR_ERR_INVALID_ARG;
    const int64_t pitch = (cols + 15) / 16 * 16, tall = (rows + 63) / 64 * 64, tiles = (cols + 127) / 128;
    if (rows > 0 && pitch > most / rows) return STAR_ERR_INVALID_ARG;
    if (tiles > 0 && tall > most / tiles) return STAR_ERR_INVALID_ARG;
    *pitch_out = pitch;
    *code_bytes_out = static_cast<size_t>(rows) * static_cast<size_t>(pitch);
    *scale_bytes_out = rows == 0 ? 0 : static_cast<size_t>(tiles) * static_cast<size_t>(tall) * 4;
    return STAR_OK;
}

extern "C" star_status_t star_checkpoint_pack(int8_t *codes, uint8_t *scales, const void *x, star_dtype_t dtype,
                                              int64_t rows, int64_t cols, int64_t ld, star_activation_t act,
                                              void *act_out, int64_t ld_act, void *cuda_stream)
{
    if (!is_dtype(dtype) || !is_act(act)) return STAR_ERR_INVALID_ARG;
    PackArgs a{};
    Extent written[2], in, out;
    star_status_t st = check_kept(codes, scales, rows, cols, &a.kept, written);
    if (st == STAR_OK) st = check_matrix(x, rows, cols, ld, dtype_size(dtype), &in);
    if (st == STAR_OK && act_out) st = check_matrix(act_out, rows, cols, ld_act, dtype_size(dtype), &out);
    if (st != STAR_OK || rows == 0 || cols == 0) return st;
    const bool in_place = act_out == x && (ld_act == ld || rows <= 1);
    if (overlaps_any(in, written, 2) || overlaps_any(out, written, 2) || (!in_place && overlap(in, out)))
        return STAR_ERR_INVALID_ARG;
    a.x = x;
    a.ld = ld;
    a.act_out = act_out;
    a.ld_act = ld_act;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    const int grid = grid_for((rows * ((cols + 31) / 32) + 7) / 8);
    with_act(act, [&](auto k) {
        constexpr int ACT = decltype(k)::value;
        if (dtype == STAR_DTYPE_BF16)
            star_checkpoint_pack_kernel<GradBF16, ACT><<<grid, kPackThreads, 0, stream>>>(a);
        else
            star_checkpoint_pack_kernel<GradF32, ACT><<<grid, kPackThreads, 0, stream>>>(a);
    });
    return launched();
}

namespace {

template <bool BACKWARD> star_status_t read_kept(UnpackArgs &a, star_dtype_t dtype, int act, void *cuda_stream)
{
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    const int grid = grid_for((a.kept.rows * a.kept.cols + kPackThreads - 1) / kPackThreads);
    with_act(act, [&](auto k) {
        constexpr int ACT = decltype(k)::value;
        if (dtype == STAR_DTYPE_BF16)
            star_checkpoint_read_kernel<GradBF16, ACT, BACKWARD><<<grid, kPackThreads, 0, stream>>>(a);
        else
            star_checkpoint_read_kernel<GradF32, ACT, BACKWARD><<<grid, kPackThreads, 0, stream>>>(a);
    });
    return launched();
}

}  // namespace

extern "C" star_status_t star_checkpoint_unpack(void *out, star_dtype_t dtype, int64_t ld, const int8_t *codes,
                                                const uint8_t *scales, int64_t rows, int64_t cols,
                                                star_activation_t act, void *cuda_stream)
{
    if (!is_dtype(dtype) || !is_act(act)) return STAR_ERR_INVALID_ARG;
    UnpackArgs a{};
    Extent read[2], written;
    star_status_t st = check_kept(codes, scales, rows, cols, &a.kept, read);
    if (st == STAR_OK) st = check_matrix(out, rows, cols, ld, dtype_size(dtype), &written);
    if (st == STAR_OK && overlaps_any(written, read, 2)) st = STAR_ERR_INVALID_ARG;
    if (st != STAR_OK || rows == 0 || cols == 0) return st;
    a.out = out;
    a.ld = ld;
    return read_kept<false>(a, dtype, act, cuda_stream);
}

extern "C" star_status_t star_checkpoint_act_backward(void *dx, int64_t ld_dx, const void *dy, int64_t ld_dy,
                                                      star_dtype_t dtype, const int8_t *codes, const uint8_t *scales,
                                                      int64_t rows, int64_t cols, star_activation_t act,
                                                      void *cuda_stream)
{
    if (!is_dtype(dtype) || !is_act(act)) return STAR_ERR_INVALID_ARG;
    UnpackArgs a{};
    Extent read[3], written;
    star_status_t st = check_kept(codes, scales, rows, cols, &a.kept, read);
    if (st == STAR_OK) st = check_matrix(dy, rows, cols, ld_dy, dtype_size(dtype), &read[2]);
    if (st == STAR_OK) st = check_matrix(dx, rows, cols, ld_dx, dtype_size(dtype), &written);
    if (st != STAR_OK || rows == 0 || cols == 0) return st;
    const bool in_place = dx == dy && (ld_dx == ld_dy || rows <= 1);
    if (overlaps_any(written, read, 2) || (!in_place && overlap(written, read[2]))) return STAR_ERR_INVALID_ARG;
    a.out = dx;
    a.ld = ld_dx;
    a.dy = dy;
    a.ld_dy = ld_dy;
    return read_kept<true>(a, dtype, act, cuda_stream);
}
