// Entry point of the weight gradient: argument checks on the host, the shape of
// the launch, one kernel.
#include <algorithm>
#include <atomic>

#include "checkpoint_host.h"
#include "weight_grad.cuh"

namespace {

using namespace star;

constexpr int kMaxDevices = 64;

// cuTensorMapEncodeTiled, looked up once: the library links the runtime only.
using EncodeTiled = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                 const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                 CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiled encode_tiled()
{
    static std::atomic<void *> found{nullptr};
    void *f = found.load(std::memory_order_acquire);
    if (!f) {
        cudaDriverEntryPointQueryResult how = cudaDriverEntryPointSymbolNotFound;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &how) != cudaSuccess ||
            how != cudaDriverEntryPointSuccess) {
            cudaGetLastError();
            return nullptr;
        }
        found.store(f, std::memory_order_release);
    }
    return reinterpret_cast<EncodeTiled>(f);
}

// A row-major matrix of `rows` rows, `stride` bytes apart, read in tiles of
// `box_cols` x `box_rows`; what lies outside reads as zero.
bool make_map(CUtensorMap *map, CUtensorMapDataType type, const void *base, int64_t cols, int64_t rows, uint64_t stride,
              unsigned box_cols, unsigned box_rows, CUtensorMapSwizzle swizzle)
{
    const EncodeTiled encode = encode_tiled();
    if (!encode) return false;
    const cuuint64_t dims[2] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(rows)}, strides[1] = {stride};
    const cuuint32_t box[2] = {box_cols, box_rows}, steps[2] = {1, 1};
    return encode(map, type, 2, const_cast<void *>(base), dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle,
                  CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int BN, int STAGES>
star_status_t launch_tensor(const WeightGradTile &tile, const CUtensorMap &codes, const CUtensorMap &dy, bool dw_bf16, int parts,
                            cudaStream_t stream)
{
    const auto kernel = star_weight_grad_tensor_kernel<BN, STAGES>;
    constexpr int smem = GradSmem<BN, STAGES>::kDynamic;
    static std::atomic<bool> ready[kMaxDevices];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return cuda_failed(e);
    if (dev >= kMaxDevices) return STAR_ERR_UNSUPPORTED;
    if (!ready[dev].load(std::memory_order_acquire)) {
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
        if (e != cudaSuccess) return cuda_failed(e);
        ready[dev].store(true, std::memory_order_release);
    }
    cudaLaunchConfig_t config{};
    config.gridDim = dim3(static_cast<unsigned>((tile.a.kept.cols + kTileC - 1) / kTileC), static_cast<unsigned>((tile.a.outs + BN - 1) / BN),
                          static_cast<unsigned>(parts));
    config.blockDim = dim3(kGradThreads);
    config.dynamicSmemBytes = smem;
    config.stream = stream;
    cudaLaunchAttribute attribute{};
    attribute.id = cudaLaunchAttributeClusterDimension;
    attribute.val.clusterDim.x = 1;
    attribute.val.clusterDim.y = 1;
    attribute.val.clusterDim.z = static_cast<unsigned>(parts);
    config.attrs = &attribute;
    config.numAttrs = 1;
    e = cudaLaunchKernelEx(&config, kernel, tile, codes, dy, static_cast<int>(dw_bf16));
    if (e != cudaSuccess) return cuda_failed(e);
    return launched();
}

// Into how many parts the rows are split: enough blocks for the device, but at
// least 4 steps each.
int row_parts(int64_t tiles, int64_t steps)
{
    int parts = 1;
    while (parts < 8 && tiles * parts * 2 <= 148 && steps >= 4 * parts * 2) parts *= 2;
    return parts;
}

}  // namespace

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
    // The TMA reads dy in place: 16-byte aligned rows, coordinates of 32 bits.
    const bool tiled = y16 && rows > 0 && reinterpret_cast<uintptr_t>(dy) % 16 == 0 && ld_dy % 8 == 0 && rows < 0x7fffff00 &&
                       cols < 0x7fffff00 && outs < 0x7fffff00 && (outs + 255) / 256 <= 65535;
    if (tiled) {
        CUtensorMap codes_map, dy_map;
        if (!make_map(&codes_map, CU_TENSOR_MAP_DATA_TYPE_UINT8, codes, a.kept.pitch, rows, static_cast<uint64_t>(a.kept.pitch), kTileC,
                      kTileT, CU_TENSOR_MAP_SWIZZLE_NONE) ||
            !make_map(&dy_map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, dy, outs, rows, static_cast<uint64_t>(ld_dy) * 2, 64, kTileT,
                      CU_TENSOR_MAP_SWIZZLE_128B))
            return cuda_failed(cudaErrorInvalidValue);
        const int64_t steps = (rows + kTileT - 1) / kTileT;
        const WeightGradTile tile{a, static_cast<int>(steps)};
        const int64_t tiles = ((cols + kTileC - 1) / kTileC) * ((outs + 255) / 256);
        return launch_tensor<256, 4>(tile, codes_map, dy_map, w16, row_parts(tiles, steps), stream);
    }
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
