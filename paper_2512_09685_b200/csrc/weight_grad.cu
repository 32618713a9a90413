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

// The kernel comes in three shapes.  Shared memory and TMEM hold one block on an
// SM in all of them.
//   kWide   a pair of blocks, 256 columns x 512 outputs: a widened code serves 512
//           outputs, 0.73 us a step of 64 rows (1.47 PFLOP/s over 148 SMs)
//   kNarrow a pair, 256 x 256: 0.56 us, bound by the widening
//   kSingle a block, 128 x 256: 0.56 us
enum Shape { kWide = 0, kNarrow = 1, kSingle = 2, kShapes = 3 };
constexpr int kMostParts = 8;

template <int SHAPE> struct ShapeOf;
template <> struct ShapeOf<kWide> {
    static constexpr int kOuts = 512, kBlocks = 2;
    using Smem = GradSmem<512, 4, 3, true>;
    static constexpr auto kernel() { return star_weight_grad_tensor_kernel<512, 4, 3, true>; }
};
template <> struct ShapeOf<kNarrow> {
    static constexpr int kOuts = 256, kBlocks = 2;
    using Smem = GradSmem<256, 7, 3, true>;
    static constexpr auto kernel() { return star_weight_grad_tensor_kernel<256, 7, 3, true>; }
};
template <> struct ShapeOf<kSingle> {
    static constexpr int kOuts = 256, kBlocks = 1;
    using Smem = GradSmem<256, 4, 3, false>;
    static constexpr auto kernel() { return star_weight_grad_tensor_kernel<256, 4, 3, false>; }
};

void fill_config(cudaLaunchConfig_t *config, cudaLaunchAttribute *attribute, int64_t columns, int64_t down, int blocks, int parts,
                 int smem, cudaStream_t stream)
{
    *config = cudaLaunchConfig_t{};
    config->gridDim = dim3(static_cast<unsigned>(columns * blocks), static_cast<unsigned>(down), static_cast<unsigned>(parts));
    config->blockDim = dim3(kGradThreads);
    config->dynamicSmemBytes = static_cast<size_t>(smem);
    config->stream = stream;
    *attribute = cudaLaunchAttribute{};
    attribute->id = cudaLaunchAttributeClusterDimension;
    attribute->val.clusterDim.x = static_cast<unsigned>(blocks);
    attribute->val.clusterDim.y = 1;
    attribute->val.clusterDim.z = static_cast<unsigned>(parts);
    config->attrs = attribute;
    config->numAttrs = 1;
}

// Per device and shape: how many clusters of `parts` tiles the device holds at
// once (GPUs of one kind differ: their SMs come in groups of uneven size, and a
// cluster stays within a group).  0: not asked yet.
struct Device {
    std::atomic<int> clusters[kShapes][kMostParts + 1];
    std::atomic<bool> ready{false};
};
Device g_devices[kMaxDevices];

template <int SHAPE> cudaError_t prepare_shape(Device &d)
{
    using S = ShapeOf<SHAPE>;
    const auto kernel = S::kernel();
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, S::Smem::kDynamic);
    for (int parts = 1; e == cudaSuccess && parts * S::kBlocks <= 8; ++parts) {
        cudaLaunchConfig_t config;
        cudaLaunchAttribute attribute;
        fill_config(&config, &attribute, 64, 1, S::kBlocks, parts, S::Smem::kDynamic, nullptr);
        int n = 0;
        e = cudaOccupancyMaxActiveClusters(&n, kernel, &config);
        d.clusters[SHAPE][parts].store(n, std::memory_order_relaxed);
    }
    return e;
}

cudaError_t prepared_device(Device **out)
{
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= kMaxDevices) return cudaErrorInvalidDevice;
    Device &d = g_devices[dev];
    if (!d.ready.load(std::memory_order_acquire)) {
        e = prepare_shape<kWide>(d);
        if (e == cudaSuccess) e = prepare_shape<kNarrow>(d);
        if (e == cudaSuccess) e = prepare_shape<kSingle>(d);
        if (e != cudaSuccess) return e;
        d.ready.store(true, std::memory_order_release);
    }
    *out = &d;
    return cudaSuccess;
}

template <int SHAPE>
star_status_t launch_shape(const WeightGradTile &tile, const CUtensorMap &codes, const CUtensorMap &dy, bool dw_bf16, int parts,
                           cudaStream_t stream)
{
    using S = ShapeOf<SHAPE>;
    cudaLaunchConfig_t config;
    cudaLaunchAttribute attribute;
    constexpr int64_t columns = S::kBlocks * kTileC;
    fill_config(&config, &attribute, (tile.a.kept.cols + columns - 1) / columns, (tile.a.outs + S::kOuts - 1) / S::kOuts, S::kBlocks,
                parts, S::Smem::kDynamic, stream);
    const cudaError_t e = cudaLaunchKernelEx(&config, S::kernel(), tile, codes, dy, static_cast<int>(dw_bf16));
    return e == cudaSuccess ? launched() : cuda_failed(e);
}

// Shape and number of parts with the least expected time: the waves of tiles the
// device needs, each the steps of one part and what a tile costs beside them.
// Measured (us; 8 to 256 steps, 128 to 4096 columns): a step takes 0.73 / 0.56 /
// 0.56, the rest 5 and, split, 17 / 12 / 12 (accumulators through distributed
// shared memory).  16384 rows, 1024 -> 4096: kWide in 2 parts 114 us, in 1 part
// 191, kNarrow 150, kSingle 148.  8192 rows, 1024 -> 1024: kSingle in 4 parts 31
// us, in 1 part 77, kWide in 4 parts 41.
struct Plan {
    Shape shape;
    int parts;
};

Plan choose(const Device &d, int64_t cols, int64_t outs, int64_t steps)
{
    constexpr double step_us[kShapes] = {0.73, 0.56, 0.56}, split_us[kShapes] = {17.0, 12.0, 12.0};
    Plan best{kSingle, 1};
    double least = -1.0;
    for (int shape = kWide; shape < kShapes; ++shape) {
        const int blocks = shape == kSingle ? 1 : 2, outs_tile = shape == kWide ? 512 : 256;
        const int64_t tiles = ((cols + blocks * kTileC - 1) / (blocks * kTileC)) * ((outs + outs_tile - 1) / outs_tile);
        for (int parts = 1; parts * blocks <= 8 && parts <= steps; ++parts) {
            const int held = std::max(d.clusters[shape][parts].load(std::memory_order_relaxed), 1);
            const double waves = static_cast<double>((tiles + held - 1) / held);
            const double cost = waves * (static_cast<double>((steps + parts - 1) / parts) * step_us[shape] + (parts > 1 ? split_us[shape] : 5.0));
            if (least < 0.0 || cost < least) {
                least = cost;
                best = Plan{static_cast<Shape>(shape), parts};
            }
        }
    }
    return best;
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
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    const bool y16 = dy_dtype == STAR_DTYPE_BF16, w16 = dw_dtype == STAR_DTYPE_BF16;
    // The TMA reads dy in place: 16-byte aligned rows, coordinates of 32 bits.
    const bool tiled = y16 && rows > 0 && reinterpret_cast<uintptr_t>(dy) % 16 == 0 && ld_dy % 8 == 0 && rows < 0x7fffff00 &&
                       cols < 0x7fffff00 && outs < 0x7fffff00 && (outs + kTileO - 1) / kTileO <= 65535;
    if (tiled) {
        CUtensorMap codes_map, dy_map;
        if (!make_map(&codes_map, CU_TENSOR_MAP_DATA_TYPE_UINT8, codes, a.kept.pitch, rows, static_cast<uint64_t>(a.kept.pitch), kTileC,
                      kTileT, CU_TENSOR_MAP_SWIZZLE_NONE) ||
            !make_map(&dy_map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, dy, outs, rows, static_cast<uint64_t>(ld_dy) * 2, 64, kTileT,
                      CU_TENSOR_MAP_SWIZZLE_128B))
            return cuda_failed(cudaErrorInvalidValue);
        const int64_t steps = (rows + kTileT - 1) / kTileT;
        const WeightGradTile tile{a, static_cast<int>(steps)};
        Device *device = nullptr;
        const cudaError_t e = prepared_device(&device);
        if (e != cudaSuccess) return cuda_failed(e);
        const Plan plan = choose(*device, cols, outs, steps);
        switch (plan.shape) {
        case kWide: return launch_shape<kWide>(tile, codes_map, dy_map, w16, plan.parts, stream);
        case kNarrow: return launch_shape<kNarrow>(tile, codes_map, dy_map, w16, plan.parts, stream);
        default: return launch_shape<kSingle>(tile, codes_map, dy_map, w16, plan.parts, stream);
        }
    }
    const int64_t across = (cols + 31) / 32, down = (outs + 31) / 32;
    if (across > 0x7fffffff) return STAR_ERR_UNSUPPORTED;
    const dim3 grid(static_cast<unsigned>(across), static_cast<unsigned>(down < 65535 ? down : 65535));
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
