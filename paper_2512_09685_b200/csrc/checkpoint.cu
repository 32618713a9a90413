// Entry points of activations kept in 8 bits: argument checks on the host, then
// one kernel launch.
#include <type_traits>

#include "checkpoint.cuh"
#include "internal.h"

namespace {

using namespace star;

star_status_t launched()
{
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return cuda_failed(e);
    count_launch();
    return STAR_OK;
}

// Checks a checkpoint's buffers; *codes and *scales span them.
star_status_t check_kept(const int8_t *codes, const uint8_t *scales, int64_t rows, int64_t cols, Kept *out, Extent *at)
{
    size_t code_bytes = 0, scale_bytes = 0;
    int64_t pitch = 0;
    const star_status_t st = star_checkpoint_sizes(rows, cols, &pitch, &code_bytes, &scale_bytes);
    if (st != STAR_OK) return st;
    at[0] = at[1] = Extent{};
    *out = Kept{const_cast<int8_t *>(codes), const_cast<uint8_t *>(scales), rows, cols, pitch, (rows + 63) / 64 * 64};
    if (code_bytes == 0) return STAR_OK;
    if (!codes || !scales) return STAR_ERR_NULL_POINTER;
    if (reinterpret_cast<uintptr_t>(codes) % 16 != 0 || reinterpret_cast<uintptr_t>(scales) % 16 != 0)
        return STAR_ERR_INVALID_ARG;
    at[0] = extent(codes, code_bytes);
    at[1] = extent(scales, scale_bytes);
    return overlap(at[0], at[1]) ? STAR_ERR_INVALID_ARG : STAR_OK;
}

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

extern "C" star_status_t star_checkpoint_weight_grad(void *dw, star_dtype_t dw_dtype, int64_t ld_dw, int transposed,
                                                     const void *dy, star_dtype_t dy_dtype, int64_t ld_dy,
                                                     const int8_t *codes, const uint8_t *scales, int64_t rows,
                                                     int64_t cols, int64_t outs, int accumulate, void *cuda_stream)
{
    if (!is_dtype(dw_dtype) || !is_dtype(dy_dtype) || outs < 0) return STAR_ERR_INVALID_ARG;
    WeightGradArgs a{};
    Extent read[3], written;
    star_status_t st = check_kept(codes, scales, rows, cols, &a.kept, read);
    if (st == STAR_OK) st = check_matrix(dy, rows, outs, ld_dy, dtype_size(dy_dtype), &read[2]);
    if (st == STAR_OK)
        st = check_matrix(dw, transposed ? cols : outs, transposed ? outs : cols, ld_dw, dtype_size(dw_dtype), &written);
    if (st == STAR_OK && overlaps_any(written, read, 3)) st = STAR_ERR_INVALID_ARG;
    if (st != STAR_OK || cols == 0 || outs == 0 || (rows == 0 && accumulate)) return st;
    a.dy = dy;
    a.ld_dy = ld_dy;
    a.dw = dw;
    a.stride_o = transposed ? 1 : ld_dw;
    a.stride_c = transposed ? ld_dw : 1;
    a.outs = outs;
    a.accumulate = accumulate;
    const int64_t across = (cols + 31) / 32, down = (outs + 31) / 32;
    if (across > 0x7fffffff) return STAR_ERR_UNSUPPORTED;
    const dim3 grid(static_cast<unsigned>(across), static_cast<unsigned>(down < 65535 ? down : 65535));
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    const bool y16 = dy_dtype == STAR_DTYPE_BF16, w16 = dw_dtype == STAR_DTYPE_BF16;
    if (y16 && w16)
        star_weight_grad_kernel<GradBF16, GradBF16><<<grid, 256, 0, stream>>>(a);
    else if (y16)
        star_weight_grad_kernel<GradBF16, GradF32><<<grid, 256, 0, stream>>>(a);
    else if (w16)
        star_weight_grad_kernel<GradF32, GradBF16><<<grid, 256, 0, stream>>>(a);
    else
        star_weight_grad_kernel<GradF32, GradF32><<<grid, 256, 0, stream>>>(a);
    return launched();
}
