// What the entry points of the operators on rows of logits share on the host:
// argument checks, and how many clusters of a kernel the device holds.
#pragma once

#include <atomic>
#include <cmath>

#include "internal.h"
#include "rows.cuh"

namespace star {

constexpr int kMostKib = 224;        // shared memory of a block that keeps a row, beside little of its own

constexpr int kMaxDevices = 64;

// Clusters of a kernel that the device holds at once, per device, cluster size
// and shared memory (in KiB), asked once: the question takes longer than a small
// launch.
struct Held {
    std::atomic<int> clusters[kMaxDevices][4][kMostKib + 1];
};

template <typename Kernel> inline cudaError_t held_clusters(Kernel kernel, Held &known, int threads, int cluster, int kib, int *out, int most_kib = kMostKib)
{
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= kMaxDevices) return cudaErrorInvalidDevice;
    std::atomic<int> &slot = known.clusters[dev][cluster == 1 ? 0 : cluster == 2 ? 1 : cluster == 4 ? 2 : 3][kib];
    int n = slot.load(std::memory_order_relaxed);
    if (n == 0) {
        if (kib > 0) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, most_kib * 1024);
        if (e != cudaSuccess) return e;
        if (cluster == 1) {
            int sms = 0, per_sm = 0;
            e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
            if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, threads, static_cast<size_t>(kib) * 1024);
            n = sms * per_sm;
        } else {
            cudaLaunchConfig_t config{};
            config.gridDim = dim3(static_cast<unsigned>(cluster) * 64);
            config.blockDim = dim3(static_cast<unsigned>(threads));
            config.dynamicSmemBytes = static_cast<size_t>(kib) * 1024;
            cudaLaunchAttribute attribute{};
            attribute.id = cudaLaunchAttributeClusterDimension;
            attribute.val.clusterDim.x = static_cast<unsigned>(cluster);
            attribute.val.clusterDim.y = 1;
            attribute.val.clusterDim.z = 1;
            config.attrs = &attribute;
            config.numAttrs = 1;
            e = cudaOccupancyMaxActiveClusters(&n, kernel, &config);
        }
        if (e != cudaSuccess) return e;
        if (n < 1) return cudaErrorInvalidConfiguration;
        slot.store(n, std::memory_order_relaxed);
    }
    *out = n;
    return cudaSuccess;
}

// The checks that the operators share.  read[0] is the logits' extent, read[1] the labels'.
inline star_status_t check_rows(const void *logits, star_dtype_t dtype, int64_t rows, int64_t vocab, int64_t ld,
                                const int64_t *labels, float temperature, RowArgs *out, Extent *read, bool labels_optional = false)
{
    if (!is_dtype(dtype) || vocab < 0) return STAR_ERR_INVALID_ARG;
    if (vocab > 0x7fffffff) return STAR_ERR_UNSUPPORTED;
    if (!(temperature > 0.0f) || !std::isfinite(temperature) || !std::isfinite(1.0f / temperature) ||
        !std::isfinite(1.0f / temperature * kLog2e))
        return STAR_ERR_INVALID_ARG;
    star_status_t st = check_matrix(logits, rows, vocab, ld, dtype_size(dtype), &read[0]);
    if (st == STAR_OK) st = check_vector(labels, rows, 8, labels_optional, &read[1]);
    if (st != STAR_OK) return st;
    *out = RowArgs{logits, ld, rows, vocab, labels, nullptr, 1.0f / temperature};
    return STAR_OK;
}

// dlogits: its own memory, or exactly the logits.
inline star_status_t check_gradient(const void *dlogits, int64_t ld_dlogits, star_dtype_t dtype, const RowArgs &row,
                                    const Extent &logits, Extent *out)
{
    *out = Extent{};
    if (!dlogits) return STAR_OK;
    const star_status_t st = check_matrix(dlogits, row.rows, row.vocab, ld_dlogits, dtype_size(dtype), out);
    if (st != STAR_OK) return st;
    const bool in_place = dlogits == row.logits && (ld_dlogits == row.ld || row.rows <= 1);
    return !in_place && overlap(*out, logits) ? STAR_ERR_INVALID_ARG : STAR_OK;
}

// No written buffer may share memory with a read one or another written one.
inline star_status_t check_disjoint(const Extent *written, int n_written, const Extent *read, int n_read)
{
    for (int i = 0; i < n_written; ++i)
        if (overlaps_any(written[i], read, n_read) || overlaps_any(written[i], written, i)) return STAR_ERR_INVALID_ARG;
    return STAR_OK;
}

inline star_status_t check_workspace(const void *workspace, size_t have, int64_t rows, int64_t sequences, Extent *out)
{
    size_t need = 0;
    const star_status_t st = star_loss_workspace_bytes(rows, sequences, &need);
    if (st != STAR_OK) return st;
    if (!workspace) return STAR_ERR_NULL_POINTER;
    if (reinterpret_cast<uintptr_t>(workspace) % 16 != 0) return STAR_ERR_INVALID_ARG;
    if (have < need) return STAR_ERR_WORKSPACE_TOO_SMALL;
    *out = extent(workspace, need);
    return STAR_OK;
}

}  // namespace star
