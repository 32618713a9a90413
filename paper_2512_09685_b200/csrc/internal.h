// What the library's source files share: error and launch bookkeeping (defined
// in api.cu) and the argument checks of operators on matrices with a row stride.
#pragma once

#include <cstddef>
#include <cstdint>

#include <cuda_runtime.h>

#include "star.h"

namespace star {

// Notes the error for star_last_cuda_error() and returns STAR_ERR_CUDA.
star_status_t cuda_failed(cudaError_t e);
// One more kernel launched (star_launch_count).
void count_launch();

// Attempts of a wait inside a kernel (star_set_wait_attempts).
int wait_attempts();

// Whether a wait of the weight gradient's kernels has run out (and no longer
// after this), once the work on `stream` is done.
cudaError_t weight_grad_expired(cudaStream_t stream, int *expired);

// The status of the launch just made; `e` is what the launching call returned.
inline star_status_t launched(cudaError_t e = cudaSuccess)
{
    const cudaError_t noted = cudaGetLastError();
    if (e == cudaSuccess) e = noted;
    if (e != cudaSuccess) return cuda_failed(e);
    count_launch();
    return STAR_OK;
}

// Launches `kernel` as a programmatic dependent of the kernel in front of it in
// the stream: its blocks may be set up before that one is done, and wait by
// themselves before they touch memory.  Also the cheaper launch for the host, by
// 1 to 2 us.  `cluster` of one block: none.
template <typename... Params, typename... Args>
star_status_t launch(void (*kernel)(Params...), dim3 grid, int threads, size_t smem, dim3 cluster, cudaStream_t stream, const Args &...args)
{
    cudaLaunchConfig_t config{};
    config.gridDim = grid;
    config.blockDim = dim3(static_cast<unsigned>(threads));
    config.dynamicSmemBytes = smem;
    config.stream = stream;
    cudaLaunchAttribute attributes[2] = {};
    attributes[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attributes[0].val.programmaticStreamSerializationAllowed = 1;
    attributes[1].id = cudaLaunchAttributeClusterDimension;
    attributes[1].val.clusterDim.x = cluster.x;
    attributes[1].val.clusterDim.y = cluster.y;
    attributes[1].val.clusterDim.z = cluster.z;
    config.attrs = attributes;
    config.numAttrs = cluster.x * cluster.y * cluster.z > 1 ? 2 : 1;
    return launched(cudaLaunchKernelEx(&config, kernel, args...));
}

inline bool is_dtype(int dt) { return dt == STAR_DTYPE_F32 || dt == STAR_DTYPE_BF16; }
inline int dtype_size(int dt) { return dt == STAR_DTYPE_BF16 ? 2 : 4; }

// A device buffer of an argument list: where it starts and how many bytes of
// address space it spans; of a matrix of several rows, also how far apart they
// are and how many bytes of each are its own.
struct Extent {
    uintptr_t begin = 0;
    uint64_t bytes = 0;
    uint64_t pitch = 0, width = 0;       // 0: one run of bytes
};

// Whether two buffers share memory.  Matrices with the same stride may lie side by
// side in the rows of one buffer: then their columns decide.  With different strides
// their address ranges do.
inline bool overlap(const Extent &a, const Extent &b)
{
    if (!a.bytes || !b.bytes || a.begin >= b.begin + b.bytes || b.begin >= a.begin + a.bytes) return false;
    const uint64_t pitch = a.pitch ? a.pitch : b.pitch;
    if (!pitch || (a.pitch && b.pitch && a.pitch != b.pitch)) return true;
    // Where b's rows start in a's, going round from row to row.
    const uint64_t at = b.begin >= a.begin ? (b.begin - a.begin) % pitch : (pitch - (a.begin - b.begin) % pitch) % pitch;
    return at < (a.pitch ? a.width : a.bytes) || at + (b.pitch ? b.width : b.bytes) > pitch;
}

inline Extent extent(const void *p, uint64_t bytes)
{
    return p ? Extent{reinterpret_cast<uintptr_t>(p), bytes, 0, 0} : Extent{};
}

// Largest byte count a matrix argument may span: far beyond any device's
// memory, and small enough that no sum of offsets overflows 64 bits.
constexpr uint64_t kMaxBytes = uint64_t{1} << 56;

// rows x cols elements of `size` bytes, `ld` elements from row to row.  Checks
// the pointer's alignment, the stride and the size; *out spans the matrix.
inline star_status_t check_matrix(const void *p, int64_t rows, int64_t cols, int64_t ld, int size, Extent *out)
{
    if (rows < 0 || cols < 0 || ld < cols) return STAR_ERR_INVALID_ARG;
    *out = Extent{};
    if (rows == 0 || cols == 0) return STAR_OK;
    if (!p) return STAR_ERR_NULL_POINTER;
    if (reinterpret_cast<uintptr_t>(p) % static_cast<unsigned>(size) != 0) return STAR_ERR_INVALID_ARG;
    if (static_cast<uint64_t>(ld) > kMaxBytes / static_cast<unsigned>(size) ||
        static_cast<uint64_t>(rows) > kMaxBytes / static_cast<unsigned>(size) / static_cast<uint64_t>(ld))
        return STAR_ERR_INVALID_ARG;
    *out = extent(p, (static_cast<uint64_t>(rows - 1) * static_cast<uint64_t>(ld) + static_cast<uint64_t>(cols)) *
                         static_cast<unsigned>(size));
    if (rows > 1) {
        out->pitch = static_cast<uint64_t>(ld) * static_cast<unsigned>(size);
        out->width = static_cast<uint64_t>(cols) * static_cast<unsigned>(size);
    }
    return STAR_OK;
}

// A vector of n elements; optional ones may be NULL.
inline star_status_t check_vector(const void *p, int64_t n, int size, bool optional, Extent *out)
{
    *out = Extent{};
    if (!p && optional) return STAR_OK;
    return check_matrix(p, 1, n, n, size, out);
}

// Whether a written buffer shares memory with any of the others.
inline bool overlaps_any(const Extent &written, const Extent *others, int n)
{
    for (int i = 0; i < n; ++i)
        if (overlap(written, others[i])) return true;
    return false;
}

}  // namespace star
