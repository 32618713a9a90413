// Entry point of the weight gradient: argument checks on the host, the shape of
// the launch, one kernel.
#include <algorithm>
#include <atomic>
#include <type_traits>

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

// The kernel's shapes.  Shared memory and TMEM hold one block on an SM in all of
// them.
//   kWide      a pair of blocks, 256 columns x 512 outputs: a widened code serves
//              512 outputs, 0.73 us a step of 64 rows (23 TFLOP/s a pair)
//   kNarrow    a pair, 256 x 256: 0.56 us, bound by the widening
//   kSingle    a block, 128 x 256: 0.56 us
//   kSmall     a block, 128 x 128, for few rows and few tiles
//   kNarrowSum, kSingleSum      with a running sum, for a dw in fp32 and for many rows
//   kLoosePair, kLooseSingle    dy in bf16 off the 16-byte grid: 256 x 128 by a
//              pair, 128 x 128 by a block
//   kCutPair, kCutSingle        dy in fp32, three terms: the same
// Each in its best number of parts, us, in bursts of 20 launches (bf16; rows, columns ->
// outputs; launched without a pause the first takes 128, under the power cap):
//                          kWide  kNarrow  kSingle  kSmall
//   16384, 1024 -> 4096    107    148      142      273
//    8192, 4096 -> 4096    199    302      292      490
//    8192, 1024 -> 1024     38     34       28       41
//     515, 1024 -> 1024     14.8   11.9     10.7      9.7
//     100,  256 ->  256     10.3    7.5      6.5      5.5
// dw in fp32, kNarrowSum 202 and kSingleSum 203 for the first, 43 and 35 for the
// third (kSingle in parts of 2048 rows: 28.5).  By pair / by block: loose dy 407 / 539
// for the first, 58 / 75 for the third, 13.9 / 12.1 for 2048, 128 -> 1024; fp32 dy 580 / 731,
// 80 / 99 and 17.3 / 15.7.
enum Shape { kWide, kNarrow, kSingle, kSmall, kNarrowSum, kSingleSum, kLoosePair, kLooseSingle, kCutPair, kCutSingle, kShapes };
constexpr int kMostParts = 8;

template <int SHAPE> struct ShapeOf;
template <int BN, int LOADS, int WIDE, bool PAIR, int TERMS, bool FLUSH> struct ShapeBase {
    static constexpr int kOuts = BN, kBlocks = PAIR ? 2 : 1;
    using Smem = GradSmem<BN, LOADS, WIDE, PAIR, TERMS>;
    static constexpr auto kernel() { return star_weight_grad_tensor_kernel<BN, LOADS, WIDE, PAIR, TERMS, FLUSH>; }
};
template <> struct ShapeOf<kWide> : ShapeBase<512, 4, 3, true, 0, false> {};
template <> struct ShapeOf<kNarrow> : ShapeBase<256, 7, 3, true, 0, false> {};
template <> struct ShapeOf<kSingle> : ShapeBase<256, 4, 3, false, 0, false> {};
template <> struct ShapeOf<kSmall> : ShapeBase<128, 6, 4, false, 0, false> {};
template <> struct ShapeOf<kNarrowSum> : ShapeBase<256, 7, 3, true, 0, true> {};
template <> struct ShapeOf<kSingleSum> : ShapeBase<256, 4, 3, false, 0, true> {};
template <> struct ShapeOf<kLoosePair> : ShapeBase<128, 6, 5, true, 1, true> {};
template <> struct ShapeOf<kLooseSingle> : ShapeBase<128, 4, 4, false, 1, true> {};
template <> struct ShapeOf<kCutPair> : ShapeBase<128, 5, 4, true, 3, true> {};
template <> struct ShapeOf<kCutSingle> : ShapeBase<128, 4, 3, false, 3, true> {};

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
        cudaLaunchConfig_t config{};
        cudaLaunchAttribute attribute{};
        config.gridDim = dim3(static_cast<unsigned>(64 * S::kBlocks), 1, static_cast<unsigned>(parts));
        config.blockDim = dim3(kGradThreads);
        config.dynamicSmemBytes = S::Smem::kDynamic;
        attribute.id = cudaLaunchAttributeClusterDimension;
        attribute.val.clusterDim.x = S::kBlocks;
        attribute.val.clusterDim.y = 1;
        attribute.val.clusterDim.z = static_cast<unsigned>(parts);
        config.attrs = &attribute;
        config.numAttrs = 1;
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
        if (e == cudaSuccess) e = prepare_shape<kSmall>(d);
        if (e == cudaSuccess) e = prepare_shape<kNarrowSum>(d);
        if (e == cudaSuccess) e = prepare_shape<kSingleSum>(d);
        if (e == cudaSuccess) e = prepare_shape<kLoosePair>(d);
        if (e == cudaSuccess) e = prepare_shape<kLooseSingle>(d);
        if (e == cudaSuccess) e = prepare_shape<kCutPair>(d);
        if (e == cudaSuccess) e = prepare_shape<kCutSingle>(d);
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
    constexpr int64_t columns = S::kBlocks * kTileC;
    const dim3 grid(static_cast<unsigned>((tile.a.kept.cols + columns - 1) / columns * S::kBlocks),
                    static_cast<unsigned>((tile.a.outs + S::kOuts - 1) / S::kOuts), static_cast<unsigned>(parts));
    return launch(S::kernel(), grid, kGradThreads, S::Smem::kDynamic, dim3(S::kBlocks, 1, static_cast<unsigned>(parts)), stream, tile,
                  codes, dy, static_cast<int>(dw_bf16));
}

// Shape and number of parts with the least expected time: the waves of tiles the
// device needs, each the steps of one part and what a tile costs beside them.
// Measured (us; 8 to 256 steps, 128 to 4096 columns): the rest beside the steps
// takes 5 and, split, 17 with 512 outputs and 12 with 256 or fewer (accumulators
// through distributed shared memory).  16384 rows, 1024 -> 4096: kWide in 2 parts
// 107 us, in 1 part 185.  8192 rows, 1024 -> 1024: kSingle in 4 parts 29 us, in 1
// part 75.
struct Plan {
    Shape shape;
    int parts;
    double us;
};

struct Candidate {
    Shape shape;
    int blocks, outs;
    double step_us, split_us;
    int most_steps;              // in one part; 0: any number
};

template <size_t N> Plan choose(const Device &d, const Candidate (&candidates)[N], int64_t cols, int64_t outs, int64_t steps)
{
    Plan best{candidates[0].shape, 1, -1.0};
    for (const Candidate &c : candidates) {
        const int64_t tiles = ((cols + c.blocks * kTileC - 1) / (c.blocks * kTileC)) * ((outs + c.outs - 1) / c.outs);
        for (int parts = 1; parts * c.blocks <= 8 && (parts <= steps || parts == 1); ++parts) {
            if (c.most_steps > 0 && (steps + parts - 1) / parts > c.most_steps) continue;
            const int held = std::max(d.clusters[c.shape][parts].load(std::memory_order_relaxed), 1);
            const double waves = static_cast<double>((tiles + held - 1) / held);
            const double cost = waves * (static_cast<double>((steps + parts - 1) / parts) * c.step_us + (parts > 1 ? c.split_us : 5.0));
            if (best.us < 0.0 || cost < best.us) best = Plan{c.shape, parts, cost};
        }
    }
    return best;
}

// One accumulator over at most 16384 rows: it cuts 4.1e-5 of a sum of one sign, a hundredth of what
// a bf16 result is rounded by (65536 rows 2.7e-4).  More go by a running sum.
constexpr int kLongSteps = 16384 / kTileT;
constexpr Candidate kPlain[6] = {{kWide, 2, 512, 0.73, 17.0, kLongSteps},   {kNarrow, 2, 256, 0.56, 12.0, kLongSteps},
                                 {kSingle, 1, 256, 0.56, 12.0, kLongSteps}, {kSmall, 1, 128, 0.52, 10.0, kLongSteps},
                                 {kNarrowSum, 2, 256, 0.76, 12.0, 0},       {kSingleSum, 1, 256, 0.76, 12.0, 0}};
// A dw in fp32 takes the same shapes for parts of at most 2048 rows, which cut 2.3e-6 of a sum of one
// sign and 4.8e-7 of one of random signs (2048 rows, 4096 -> 4096: 82 us; in parts no longer than a
// run of the running sum, 1.2e-6 at most, 131 us).
constexpr int kShortSteps = 2048 / kTileT;
constexpr Candidate kSummed[6] = {{kNarrowSum, 2, 256, 0.76, 12.0, 0},          {kSingleSum, 1, 256, 0.76, 12.0, 0},
                                  {kWide, 2, 512, 0.73, 17.0, kShortSteps},     {kNarrow, 2, 256, 0.56, 12.0, kShortSteps},
                                  {kSingle, 1, 256, 0.56, 12.0, kShortSteps},   {kSmall, 1, 128, 0.52, 10.0, kShortSteps}};
constexpr Candidate kLooseDy[2] = {{kLoosePair, 2, 128, 0.9, 10.0, 0}, {kLooseSingle, 1, 128, 0.9, 10.0, 0}};
constexpr Candidate kCutDy[2] = {{kCutPair, 2, 128, 1.0, 10.0, 0}, {kCutSingle, 1, 128, 1.2, 10.0, 0}};

// Few rows on the ordinary units, where that takes less than the tensor cores.  Here: waves
// of tiles, two to an SM, each of 2 us and 0.25 us a row (0.3 transposed).  There: `us`, as chosen
// above, or, where few steps leave the time to the stores, 5 us and 0.8 us a million results in
// bf16 (0.9), 1.1 in fp32 (1.3), 2.9 from a dy in fp32 (narrower tiles).  Here / tensor cores, us:
//                        1 row         2         4         8        16        32
//   bf16 4096 x 4096  10.2/18.7 12.2/19.0 15.4/18.7 18.1/18.6 22.5/18.2 38.3/18.1
//   bf16 1024 x 4096   4.4/7.9   4.9/8.1   6.2/8.0   6.3/8.0   8.1/7.9  12.8/7.9
//   bf16 1024 x 1024   2.6/5.1   3.1/5.3   3.6/5.1   3.7/5.1   4.7/5.1   7.3/5.0
//   dw in fp32, 4096 x 4096      14.7/24.2 16.3/24.0 19.7/24.1 22.1/24.0 27.4/23.6 42.6/23.6
//   dy and dw in fp32, the same  14.5/52.3 16.2/52.4 19.5/52.5 21.8/52.6 27.2/52.8 42.4/53.9
bool few_rows(int64_t rows, int64_t cols, int64_t outs, bool transposed, bool y16, bool w16, double us)
{
    const int64_t inner = transposed ? outs : cols, outer = transposed ? cols : outs;
    const int64_t tiles = ((inner + kFewInner - 1) / kFewInner) * ((outer + kFewOuter - 1) / kFewOuter);
    const double millions = static_cast<double>(cols) * static_cast<double>(outs) * 1e-6;
    const double stores = 5.0 + millions * (!y16 ? 2.9 : w16 ? (transposed ? 0.9 : 0.8) : (transposed ? 1.3 : 1.1));
    const double row = transposed ? 0.3 : 0.25;
    return 2.0 + static_cast<double>((tiles + 295) / 296) * (2.0 + row * static_cast<double>(rows)) < std::max(us, stores);
}

template <typename GY, typename GW> star_status_t launch_few(const WeightGradArgs &a, bool transposed, cudaStream_t stream)
{
    const int64_t inner = transposed ? a.outs : a.kept.cols, outer = transposed ? a.kept.cols : a.outs;
    const int64_t ld = transposed ? a.stride_c : a.stride_o;
    const int vector = reinterpret_cast<uintptr_t>(a.dw) % (4 * GW::kBytes) == 0 && ld % 4 == 0;
    const dim3 grid(static_cast<unsigned>((inner + kFewInner - 1) / kFewInner), static_cast<unsigned>((outer + kFewOuter - 1) / kFewOuter));
    if (transposed)
        return launch(star_weight_grad_few_kernel<GY, GW, true>, grid, kFewThreads, 0, dim3(1), stream, a, vector);
    return launch(star_weight_grad_few_kernel<GY, GW, false>, grid, kFewThreads, 0, dim3(1), stream, a, vector);
}

}  // namespace

cudaError_t star::weight_grad_expired(cudaStream_t stream, int *expired) { return take_expired(stream, expired); }

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
    if (rows >= 0x7fffff00 || cols >= 0x7fffff00 || outs >= 0x7fffff00 || std::max(cols, outs) > int64_t{65535} * kFewOuter) return STAR_ERR_UNSUPPORTED;
    // The TMA reads dy in place: rows on the 16-byte grid, strides of up to 40 bits.
    const bool tiled = y16 && reinterpret_cast<uintptr_t>(dy) % 16 == 0 && ld_dy % 8 == 0 && ld_dy < (int64_t{1} << 38);
    Device *device = nullptr;
    const cudaError_t e = prepared_device(&device);
    if (e != cudaSuccess) return cuda_failed(e);
    const int64_t steps = (rows + kTileT - 1) / kTileT;
    const Plan plan = !y16     ? choose(*device, kCutDy, cols, outs, steps)
                      : !tiled ? choose(*device, kLooseDy, cols, outs, steps)
                      : w16    ? choose(*device, kPlain, cols, outs, steps)
                               : choose(*device, kSummed, cols, outs, steps);
    if (rows == 0 || few_rows(rows, cols, outs, transposed != 0, y16, w16, plan.us)) {
        if (y16) return w16 ? launch_few<GradBF16, GradBF16>(a, transposed != 0, stream) : launch_few<GradBF16, GradF32>(a, transposed != 0, stream);
        return w16 ? launch_few<GradF32, GradBF16>(a, transposed != 0, stream) : launch_few<GradF32, GradF32>(a, transposed != 0, stream);
    }
    CUtensorMap codes_map{}, dy_map{};
    if (!make_map(&codes_map, CU_TENSOR_MAP_DATA_TYPE_UINT8, codes, a.kept.pitch, rows, static_cast<uint64_t>(a.kept.pitch), kTileC, kTileT,
                  CU_TENSOR_MAP_SWIZZLE_NONE))
        return cuda_failed(cudaErrorInvalidValue);
    if (tiled && !make_map(&dy_map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, dy, outs, rows, static_cast<uint64_t>(ld_dy) * 2, 64, kTileT,
                           CU_TENSOR_MAP_SWIZZLE_128B))
        return cuda_failed(cudaErrorInvalidValue);
    const WeightGradTile tile{a, static_cast<int>(steps), wait_attempts()};
    const auto run = [&](auto shape) { return launch_shape<decltype(shape)::value>(tile, codes_map, dy_map, w16, plan.parts, stream); };
    switch (plan.shape) {
    case kWide: return run(std::integral_constant<int, kWide>());
    case kNarrow: return run(std::integral_constant<int, kNarrow>());
    case kSmall: return run(std::integral_constant<int, kSmall>());
    case kNarrowSum: return run(std::integral_constant<int, kNarrowSum>());
    case kSingleSum: return run(std::integral_constant<int, kSingleSum>());
    case kLoosePair: return run(std::integral_constant<int, kLoosePair>());
    case kLooseSingle: return run(std::integral_constant<int, kLooseSingle>());
    case kCutPair: return run(std::integral_constant<int, kCutPair>());
    case kCutSingle: return run(std::integral_constant<int, kCutSingle>());
    default: return run(std::integral_constant<int, kSingle>());
    }
}
