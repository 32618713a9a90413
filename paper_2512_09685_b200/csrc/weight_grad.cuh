// Device code of the weight gradient whose input was kept in 8 bits, on the
// 5th-generation tensor cores (sm_100a).
//
// dW[o][c] = sum_t dy[t][o] * value[t][c] is a matrix product over the rows t
// of the step.  A block of threads owns 128 columns c (the accumulator's 128
// lanes) and BN outputs o (its columns), and walks the rows in steps of 64:
//   - one thread fetches the step's codes, scale bytes and dy tile by TMA;
//   - eight warps widen the codes to bf16, which holds code * 2^e exactly, and
//     write them as the A operand; the dy tile is the B operand as it lies in
//     memory (both operands have the summed index t slowest: "MN-major");
//   - one thread issues the matrix instructions, which accumulate in TMEM.
// Products are exact; the sums are binary32.  With few output tiles the rows are
// split over the blocks of a cluster, which add their accumulators through
// distributed shared memory in a fixed order.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "checkpoint.cuh"

namespace star {

constexpr int kTileC = 128;          // columns (M of the matrix instruction)
constexpr int kTileT = 64;           // rows per step
constexpr int kConvertWarps = 8;
constexpr int kFirstConvert = 4;     // warps 0: TMA, 1: matrix instructions, 2: TMEM, 3: idle
constexpr int kGradThreads = 32 * (kFirstConvert + kConvertWarps);

struct WeightGradTile {
    WeightGradArgs a;
    int steps;                       // of kTileT rows
};

// ---------------------------------------------------------------------------
// Barriers in shared memory.  Every wait ends: after kWaitNs it reports failure,
// the block stops issuing, drains its copies, and leaves without a result.
// ---------------------------------------------------------------------------
constexpr uint64_t kWaitNs = 4000000000ull;
__device__ int g_wait_expired;       // set by a block that gave up waiting

__device__ __forceinline__ uint32_t smem_address(const void *p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }

__device__ __forceinline__ void barrier_init(uint32_t bar, uint32_t count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" :: "r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void barrier_expect(uint32_t bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" :: "r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void barrier_arrive(uint32_t bar)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" :: "r"(bar) : "memory");
}
__device__ __forceinline__ bool barrier_try(uint32_t bar, uint32_t parity)
{
    uint32_t done;
    asm volatile("{\n\t.reg .pred p;\n\t"
                 "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
                 "selp.u32 %0, 1, 0, p;\n\t}" : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    return done != 0;
}
__device__ __forceinline__ uint64_t now_ns()
{
    uint64_t t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
    return t;
}
__device__ __noinline__ bool barrier_wait_long(uint32_t bar, uint32_t parity)
{
    const uint64_t start = now_ns();
    while (now_ns() - start < kWaitNs)
        for (int i = 0; i < 64; ++i)
            if (barrier_try(bar, parity)) return true;
    atomicExch(&g_wait_expired, 1);
    return false;
}
__device__ __forceinline__ bool barrier_wait(uint32_t bar, uint32_t parity)
{
    for (int i = 0; i < 32; ++i)
        if (barrier_try(bar, parity)) return true;
    return barrier_wait_long(bar, parity);
}

// ---------------------------------------------------------------------------
// Copies and matrix instructions.
// ---------------------------------------------------------------------------
__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap *map, int x, int y, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 :: "r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}
__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 :: "r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}

// Descriptor of an operand tile stored as 128-byte rows (64 bf16 of one t), 64
// rows to a chunk of 64 columns, 128-byte swizzle.  Leading offset: from chunk
// to chunk; stride offset: from 8 rows to the next 8.
__device__ __forceinline__ uint64_t operand_descriptor(uint32_t address)
{
    constexpr uint64_t leading = (kTileT * 128) >> 4, stride = (8 * 128) >> 4;
    return static_cast<uint64_t>((address >> 4) & 0x3fff) | leading << 16 | stride << 32 | uint64_t{1} << 46 | uint64_t{2} << 61;
}

// bf16 x bf16 -> fp32, both operands MN-major, M = 128.
template <int BN> __device__ __forceinline__ constexpr uint32_t instruction_descriptor()
{
    return 1u << 4 | 1u << 7 | 1u << 10 | 1u << 15 | 1u << 16 | static_cast<uint32_t>(BN / 8) << 17 | static_cast<uint32_t>(kTileC / 16) << 24;
}

__device__ __forceinline__ void matrix_multiply(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool accumulate)
{
    asm volatile("{\n\t.reg .pred p;\n\t"
                 "setp.ne.u32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 :: "r"(d), "l"(a), "l"(b), "r"(idesc), "r"(static_cast<uint32_t>(accumulate)) : "memory");
}
// The barrier's phase advances once every matrix instruction issued so far is done.
__device__ __forceinline__ void matrix_commit(uint32_t bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" :: "r"(bar) : "memory");
}
__device__ __forceinline__ void tensor_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tensor_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// 32 columns of the warp's 32 accumulator lanes: out[i] = column i of this thread's lane.
__device__ __forceinline__ void load_accumulator(uint32_t address, float (&out)[32])
{
    uint32_t r[32];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 "
                 "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
                 "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
                   "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
                   "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
                   "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
                 : "r"(address));
    // The registers go through the wait, so that nothing reads them before it.
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
                   "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]),
                   "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]),
                   "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31])
                 :: "memory");
#pragma unroll
    for (int i = 0; i < 32; ++i) out[i] = __uint_as_float(r[i]);
}

// ---------------------------------------------------------------------------
// Widening.  With u = code + 128 in 0 .. 255, the float with bits 0x4b0000uu is
// 2^23 + u; fma(that, 2^e, -(2^23 + 128) 2^e) = code * 2^e, exact, and exact in
// bf16: its upper half.  A byte permutation, an fma per code and half a
// permutation to pack: 2.5 instructions a code.
// ---------------------------------------------------------------------------
__device__ __forceinline__ uint2 widen_codes(uint32_t four, float scale)
{
    const uint32_t u = four ^ 0x80808080u;
    const float off = __fmul_rn(scale, -8388736.0f);
    float f[4];
    f[0] = __fmaf_rn(__uint_as_float(__byte_perm(u, 0x4b000000u, 0x7650)), scale, off);
    f[1] = __fmaf_rn(__uint_as_float(__byte_perm(u, 0x4b000000u, 0x7651)), scale, off);
    f[2] = __fmaf_rn(__uint_as_float(__byte_perm(u, 0x4b000000u, 0x7652)), scale, off);
    f[3] = __fmaf_rn(__uint_as_float(__byte_perm(u, 0x4b000000u, 0x7653)), scale, off);
    return make_uint2(__byte_perm(__float_as_uint(f[0]), __float_as_uint(f[1]), 0x7632),
                      __byte_perm(__float_as_uint(f[2]), __float_as_uint(f[3]), 0x7632));
}

// Shared memory of a block, from a 1024-byte aligned base.
template <int BN, int STAGES> struct GradSmem {
    static constexpr int kA = kTileC * kTileT * 2;
    static constexpr int kB = BN * kTileT * 2;
    static constexpr int kRaw = kTileC * kTileT;
    static constexpr int kScale = kTileT * 4;
    static constexpr int kOffB = STAGES * kA;
    static constexpr int kOffRaw = kOffB + STAGES * kB;
    static constexpr int kOffScale = kOffRaw + STAGES * kRaw;
    static constexpr int kOffBarrier = kOffScale + STAGES * kScale;
    static constexpr int kBytes = kOffBarrier + 256;
    static constexpr int kDynamic = kBytes + 1024;               // room to align the base
    static_assert(kTileC * BN * 4 <= kOffBarrier, "the accumulators of a split tile reuse the stages");
    static_assert(kDynamic <= 232448, "more shared memory than a block may have");
};

__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t peer_address(uint32_t address, uint32_t rank)
{
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(address), "r"(rank));
    return r;
}
__device__ __forceinline__ float peer_load(uint32_t address)
{
    float x;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(x) : "r"(address) : "memory");
    return x;
}

__device__ __forceinline__ void store_weight(const WeightGradArgs &a, bool bf16, int64_t o, int64_t c, float x)
{
    const int64_t at = o * a.stride_o + c * a.stride_c;
    if (bf16) {
        if (a.accumulate) x = __fadd_rn(x, load_value<GradBF16>(a.dw, at));
        store_value<GradBF16>(a.dw, at, x);
    } else {
        if (a.accumulate) x = __fadd_rn(x, load_value<GradF32>(a.dw, at));
        store_value<GradF32>(a.dw, at, x);
    }
}

// grid: (column tiles, output tiles, parts of the rows); cluster: (1, 1, parts).
template <int BN, int STAGES>
__global__ void __launch_bounds__(kGradThreads, 1)
star_weight_grad_tensor_kernel(const __grid_constant__ WeightGradTile p, const __grid_constant__ CUtensorMap codes_map,
                               const __grid_constant__ CUtensorMap dy_map, int dw_bf16)
{
    using S = GradSmem<BN, STAGES>;
    extern __shared__ uint8_t dynamic[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(dynamic) + 1023) & ~uintptr_t{1023});
    const uint32_t base = smem_address(smem);
    const uint32_t bars = base + S::kOffBarrier;
    const auto loaded = [&](int s) { return bars + 8 * s; };                     // the step's copies have landed
    const auto widened = [&](int s) { return bars + 8 * (STAGES + s); };         // its A operand is written
    const auto used = [&](int s) { return bars + 8 * (2 * STAGES + s); };        // its matrix instructions are done
    const uint32_t finished = bars + 8 * (3 * STAGES);
    uint32_t *tmem_at = reinterpret_cast<uint32_t *>(smem + S::kOffBarrier + 8 * (3 * STAGES + 1));
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;

    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) {
            barrier_init(loaded(s), 1);
            barrier_init(widened(s), kConvertWarps);
            barrier_init(used(s), 1);
        }
        barrier_init(finished, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 2) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                     :: "r"(smem_address(tmem_at)), "n"(BN) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    tensor_fence_before();
    __syncthreads();
    tensor_fence_after();
    const uint32_t tmem = *tmem_at;

    const int64_t c0 = static_cast<int64_t>(blockIdx.x) * kTileC, o0 = static_cast<int64_t>(blockIdx.y) * BN;
    const int parts = static_cast<int>(gridDim.z), part = static_cast<int>(blockIdx.z);
    const int first = static_cast<int>(static_cast<int64_t>(p.steps) * part / parts);
    const int last = static_cast<int>(static_cast<int64_t>(p.steps) * (part + 1) / parts);
    bool ok = true;

    if (warp == 0) {
        if (lane == 0) {
            int issued = 0;
            for (int k = first; k < last; ++k) {
                const int i = k - first, s = i % STAGES;
                if (i >= STAGES && !barrier_wait(used(s), (i / STAGES - 1) & 1)) break;
                barrier_expect(loaded(s), S::kRaw + S::kScale + S::kB);
                const int t = k * kTileT;
                tma_load_2d(base + S::kOffRaw + s * S::kRaw, &codes_map, static_cast<int>(c0), t, loaded(s));
                bulk_load(base + S::kOffScale + s * S::kScale, p.a.kept.scales + (blockIdx.x * p.a.kept.tall + t) * 4, S::kScale, loaded(s));
#pragma unroll
                for (int q = 0; q < BN / 64; ++q)
                    tma_load_2d(base + S::kOffB + s * S::kB + q * (kTileT * 128), &dy_map, static_cast<int>(o0) + 64 * q, t, loaded(s));
                issued = i + 1;
            }
            // Copies still in flight land before the block goes on (they have, unless a wait ran out).
            for (int i = issued > STAGES ? issued - STAGES : 0; i < issued; ++i) barrier_wait(loaded(i % STAGES), (i / STAGES) & 1);
        }
    } else if (warp == 1) {
        if (lane == 0) {
            constexpr uint32_t idesc = instruction_descriptor<BN>();
            for (int k = first; k < last && ok; ++k) {
                const int i = k - first, s = i % STAGES;
                const uint32_t parity = (i / STAGES) & 1;
                ok = barrier_wait(loaded(s), parity) && barrier_wait(widened(s), parity);
                if (!ok) break;
                tensor_fence_after();
                const uint32_t as = base + s * S::kA, bs = base + S::kOffB + s * S::kB;
#pragma unroll
                for (int q = 0; q < kTileT / 16; ++q)                // 16 rows an instruction
                    matrix_multiply(tmem, operand_descriptor(as + q * 2048), operand_descriptor(bs + q * 2048), idesc, i > 0 || q > 0);
                matrix_commit(used(s));
            }
            if (last > first) matrix_commit(finished);
        }
    } else if (warp >= kFirstConvert) {
        const int w = threadIdx.x - 32 * kFirstConvert;
        for (int k = first; k < last; ++k) {
            const int i = k - first, s = i % STAGES;
            ok = barrier_wait(loaded(s), (i / STAGES) & 1);
            if (!ok) break;
            const uint8_t *raw = smem + S::kOffRaw + s * S::kRaw, *scale = smem + S::kOffScale + s * S::kScale;
            uint8_t *as = smem + s * S::kA;
#pragma unroll
            for (int h = 0; h < kTileT * 8 / (32 * kConvertWarps); ++h) {
                const int unit = w + h * 32 * kConvertWarps, t = unit / 8, j = unit % 8;       // 16 codes of row t
                const uint4 codes = *reinterpret_cast<const uint4 *>(raw + t * kTileC + j * 16);
                // Rows past the end have codes 0 and no scale.
                const float f = static_cast<int64_t>(k) * kTileT + t < p.a.kept.rows ? scale_value(scale[t * 4 + j / 2]) : 0.0f;
                const uint2 q0 = widen_codes(codes.x, f), q1 = widen_codes(codes.y, f), q2 = widen_codes(codes.z, f), q3 = widen_codes(codes.w, f);
                const uint4 lo = make_uint4(q0.x, q0.y, q1.x, q1.y), hi = make_uint4(q2.x, q2.y, q3.x, q3.y);
                // Eight neighbouring threads fill one 128-byte row in each half; the upper
                // half starts with its odd 16 bytes, so that no bank is hit twice.
                uint8_t *row = as + (j / 4) * (kTileT * 128) + t * 128;
                const int odd = j / 4, even_at = ((2 * (j % 4)) ^ (t % 8)) * 16, odd_at = ((2 * (j % 4) + 1) ^ (t % 8)) * 16;
                *reinterpret_cast<uint4 *>(row + (odd ? odd_at : even_at)) = odd ? hi : lo;
                *reinterpret_cast<uint4 *>(row + (odd ? even_at : odd_at)) = odd ? lo : hi;
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) barrier_arrive(widened(s));
        }
    }

    // The result: every warp waits for the last matrix instruction itself.
    const bool any = last > first;
    __syncwarp();                        // the idle lanes of a role do not spin beside it
    if (any) ok = barrier_wait(finished, 0) && ok;
    const bool whole = __syncthreads_and(ok);
    tensor_fence_after();
    if (parts == 1) {
        if (whole && warp >= kFirstConvert) {
            const int quarter = warp % 4, half = (warp - kFirstConvert) / 4;
            const int64_t c = c0 + quarter * 32 + lane;
            for (int col = half * (BN / 2); col < (half + 1) * (BN / 2); col += 32) {
                float x[32];
                if (any) {
                    load_accumulator(tmem + (static_cast<uint32_t>(quarter * 32) << 16) + col, x);
                } else {
#pragma unroll
                    for (int r = 0; r < 32; ++r) x[r] = 0.0f;
                }
                if (c < p.a.kept.cols) {
#pragma unroll
                    for (int r = 0; r < 32; ++r)
                        if (o0 + col + r < p.a.outs) store_weight(p.a, dw_bf16, o0 + col + r, c, x[r]);
                }
            }
        }
    } else {
        float *sums = reinterpret_cast<float *>(smem);               // [BN][kTileC]
        if (warp >= kFirstConvert) {
            const int quarter = warp % 4, half = (warp - kFirstConvert) / 4;
            for (int col = half * (BN / 2); col < (half + 1) * (BN / 2); col += 32) {
                float x[32];
                load_accumulator(tmem + (static_cast<uint32_t>(quarter * 32) << 16) + col, x);
#pragma unroll
                for (int r = 0; r < 32; ++r) sums[(col + r) * kTileC + quarter * 32 + lane] = x[r];
            }
        }
        __syncthreads();
        cluster_sync();
        const int mine = BN / parts;
        const uint32_t rank = cluster_rank();
        if (whole) {
            for (int i = threadIdx.x; i < mine * kTileC; i += kGradThreads) {
                const int col = static_cast<int>(rank) * mine + i / kTileC, r = i % kTileC;
                const uint32_t at = base + static_cast<uint32_t>(col * kTileC + r) * 4;
                float x = peer_load(peer_address(at, 0));
                for (int q = 1; q < parts; ++q) x = __fadd_rn(x, peer_load(peer_address(at, q)));
                if (c0 + r < p.a.kept.cols && o0 + col < p.a.outs) store_weight(p.a, dw_bf16, o0 + col, c0 + r, x);
            }
        }
        __syncthreads();
        cluster_sync();                                              // nobody leaves while its memory is read
    }
    tensor_fence_before();
    __syncthreads();
    if (warp == 2)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" :: "r"(tmem), "n"(BN));
}

}  // namespace star
