// Entry points of activations kept in 8 bits: argument checks on the host, then
// one kernel launch.
#include <algorithm>
#include <type_traits>

#include "checkpoint.cuh"
#include "checkpoint_host.h"

namespace {

using namespace star;

bool is_act(int act) { return act >= STAR_ACT_NONE && act <= STAR_ACT_SILU; }

int grid_for(int64_t blocks) { return static_cast<int>(blocks < 1 ? 1 : blocks < 148 * 64 ? blocks : 148 * 64); }

// Whether every row of a matrix starts on a boundary of `bytes`.
bool on_grid(const void *p, int64_t ld, int size, int bytes = 16)
{
    return reinterpret_cast<uintptr_t>(p) % static_cast<unsigned>(bytes) == 0 && (ld * size) % bytes == 0;
}

// i / d = (i * magic) >> (32 + shift) for all i < 2^31: magic = floor(2^(32 + shift) / d) + 1
// with 2^shift the power of two at or below d - 1, so that it fits 32 bits.
Divisor make_divisor(uint32_t d)
{
    Divisor r{d, 0, 0};
    while (d > 1 && (uint64_t{1} << (r.shift + 1)) < d) ++r.shift;
    r.magic = static_cast<uint32_t>((uint64_t{1} << (32 + r.shift)) / d + 1);
    return r;
}

// Runs launch_items(items, grid) on the rows in runs of at most 2^30 items, `per_row`
// of them to a row (one run, for all but checkpoints of 16 GB and more).
template <typename Items, typename F> star_status_t by_rows(int64_t rows, int64_t per_row, int items_per_block, F launch_items)
{
    const int64_t most = (int64_t{1} << 30) / per_row;
    for (int64_t first = 0; first < rows; first += most) {
        const int64_t n = std::min(most, rows - first) * per_row;
        Items items{};
        items.per_row = make_divisor(static_cast<uint32_t>(per_row));
        items.first_row = static_cast<uint32_t>(first);
        items.n = static_cast<uint32_t>(n);
        const star_status_t st = launch_items(items, grid_for((n + items_per_block - 1) / items_per_block));
        if (st != STAR_OK) return st;
    }
    return STAR_OK;
}
template <typename F> star_status_t by_halves(int64_t rows, int64_t cols, bool wide, F launch_items)
{
    return by_rows<Halves>(rows, (cols + 31) / 32 * 2, kKeepThreads, [&](Halves h, int grid) {
        h.wide = wide;
        return launch_items(h, grid);
    });
}
template <typename F> star_status_t by_groups(int64_t rows, int64_t cols, F launch_items)
{
    return by_rows<Groups>(rows, ((cols + 31) / 32 + kLoose - 1) / kLoose, kKeepThreads / 32, launch_items);
}

// Rows and the items of a row are numbered in 32 bits.
bool countable(int64_t rows, int64_t cols) { return rows <= 0x7fffffff && cols <= (int64_t{1} << 32); }

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
    if (!countable(rows, cols)) return STAR_ERR_UNSUPPORTED;
    const int size = dtype_size(dtype);
    const bool vector = on_grid(x, ld, size) && (!act_out || on_grid(act_out, ld_act, size));
    const bool wide = on_grid(x, ld, size, 32) && (!act_out || on_grid(act_out, ld_act, size, 32));
    with_act(act, [&](auto k) {
        constexpr int ACT = decltype(k)::value;
        if (vector)
            st = by_halves(rows, cols, wide, [&](const Halves &h, int grid) {
                if (dtype == STAR_DTYPE_BF16)
                    return launch(star_checkpoint_pack_kernel<GradBF16, ACT>, dim3(static_cast<unsigned>(grid)), kKeepThreads, 0, dim3(1), stream, a, h);
                return launch(star_checkpoint_pack_kernel<GradF32, ACT>, dim3(static_cast<unsigned>(grid)), kKeepThreads, 0, dim3(1), stream, a, h);
            });
        else
            st = by_groups(rows, cols, [&](const Groups &h, int grid) {
                if (dtype == STAR_DTYPE_BF16)
                    return launch(star_checkpoint_pack_loose_kernel<GradBF16, ACT>, dim3(static_cast<unsigned>(grid)), kKeepThreads, 0, dim3(1), stream, a, h);
                return launch(star_checkpoint_pack_loose_kernel<GradF32, ACT>, dim3(static_cast<unsigned>(grid)), kKeepThreads, 0, dim3(1), stream, a, h);
            });
    });
    return st;
}

namespace {

template <bool BACKWARD> star_status_t read_kept(const ReadArgs &a, star_dtype_t dtype, int act, void *cuda_stream)
{
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (!countable(a.kept.rows, a.kept.cols)) return STAR_ERR_UNSUPPORTED;
    const int size = dtype_size(dtype);
    const bool vector = on_grid(a.out, a.ld, size) && (!BACKWARD || on_grid(a.dy, a.ld_dy, size));
    const bool wide = on_grid(a.out, a.ld, size, 32) && (!BACKWARD || on_grid(a.dy, a.ld_dy, size, 32));
    star_status_t st = STAR_OK;
    with_act(act, [&](auto k) {
        constexpr int ACT = decltype(k)::value;
        if (vector)
            st = by_halves(a.kept.rows, a.kept.cols, wide, [&](const Halves &h, int grid) {
                if (dtype == STAR_DTYPE_BF16)
                    return launch(star_checkpoint_read_kernel<GradBF16, ACT, BACKWARD>, dim3(static_cast<unsigned>(grid)), kKeepThreads, 0, dim3(1), stream, a, h);
                return launch(star_checkpoint_read_kernel<GradF32, ACT, BACKWARD>, dim3(static_cast<unsigned>(grid)), kKeepThreads, 0, dim3(1), stream, a, h);
            });
        else
            st = by_groups(a.kept.rows, a.kept.cols, [&](const Groups &h, int grid) {
                if (dtype == STAR_DTYPE_BF16)
                    return launch(star_checkpoint_read_loose_kernel<GradBF16, ACT, BACKWARD>, dim3(static_cast<unsigned>(grid)), kKeepThreads, 0, dim3(1), stream, a, h);
                return launch(star_checkpoint_read_loose_kernel<GradF32, ACT, BACKWARD>, dim3(static_cast<unsigned>(grid)), kKeepThreads, 0, dim3(1), stream, a, h);
            });
    });
    return st;
}

}  // namespace

extern "C" star_status_t star_checkpoint_unpack(void *out, star_dtype_t dtype, int64_t ld, const int8_t *codes,
                                                const uint8_t *scales, int64_t rows, int64_t cols,
                                                star_activation_t act, void *cuda_stream)
{
    if (!is_dtype(dtype) || !is_act(act)) return STAR_ERR_INVALID_ARG;
    ReadArgs a{};
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
    ReadArgs a{};
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
