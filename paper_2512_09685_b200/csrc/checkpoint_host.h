// Argument checks shared by the entry points that take a checkpoint.
#pragma once

#include "checkpoint.cuh"
#include "internal.h"

namespace star {

// Checks a checkpoint's buffers; *codes and *scales span them.
inline star_status_t check_kept(const int8_t *codes, const uint8_t *scales, int64_t rows, int64_t cols, Kept *out, Extent *at)
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

}  // namespace star
