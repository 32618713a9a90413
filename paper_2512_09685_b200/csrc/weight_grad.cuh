// Device code of the weight gradient whose input was kept in 8 bits, on the
// 5th-generation tensor cores (sm_100a).
//
// dW[o][c] = sum_t dy[t][o] * value[t][c] is a matrix product over the rows t
// of the step.  A block of threads owns 128 columns c (the accumulator's 128
// lanes) and BN outputs o (its columns), and walks the rows in steps of 64:
//   - one thread fetches the step's codes, scale bytes and dy tile by TMA;
//   - two groups of eight warps, in turn, widen the codes to bf16, which holds
//     code * 2^e exactly, and write them as the A operand; the dy tile is the B
//     operand as it lies in memory (both operands have the summed index t slowest:
//     "MN-major");
//   - one thread issues the matrix instructions, which accumulate in TMEM.
// With few output tiles the rows are split over the blocks of a cluster, which add
// their accumulators through distributed shared memory in a fixed order.
//
// Precision.  Products are exact.  A dy in fp32 is cut into three bf16 terms of 8
// bits each, which together are it, and multiplied three times.  The tensor
// cores' binary32 additions cut instead of rounding: a sum of one sign in one
// accumulator is off towards zero by 2.3e-6 of itself after 2048 rows, 1.7e-5 after 8192,
// 4.1e-5 after 16384 and 2.7e-4 after 65536, one of random signs by 4.8e-7 after 2048
// (measured).  For a dw in bf16 that stays far below its own rounding up to the 16384
// rows that go into one; for a dw in fp32 the accumulator is added to a running sum, with
// rounding, every 1280 rows (FLUSH): 1.2e-6 and 2.8e-7 for any number of rows, where a binary32
// product on the ordinary units has 1.9e-6 and 5.4e-7 after 16384.  Every 2048 rows would be
// 2.3e-6 and 4.8e-7 and 0 to 5 % faster.  The lower terms of an fp32 dy have an accumulator of
// their own, beside sums 2^8 and 2^16 times their size most of their bits would be cut: 1.5e-6 and
// 3.6e-7.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "checkpoint.cuh"

namespace star {

constexpr int kTileC = 128;          // columns (M of the matrix instruction)
constexpr int kTileT = 64;           // rows per step
constexpr int kTileO = 256;          // most outputs (N) of one matrix instruction
constexpr int kGroups = 2;           // groups of converting warps, taking the steps in turn
constexpr int kGroupWarps = 8;
constexpr int kConvertWarps = kGroups * kGroupWarps;
constexpr int kFirstConvert = 4;     // warps 0: TMA, 1: matrix instructions, 2: TMEM, 3: idle
constexpr int kGradThreads = 32 * (kFirstConvert + kConvertWarps);

struct WeightGradTile {
    WeightGradArgs a;
    int steps;                       // of kTileT rows
    int tries;                       // of a wait
};

// ---------------------------------------------------------------------------
// Copies and matrix instructions.
// ---------------------------------------------------------------------------
__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap *map, int x, int y, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 :: "r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}
// Descriptor of an operand tile stored as 128-byte rows (64 bf16 of one t), 64
// rows to a chunk of 64 columns, 128-byte swizzle.  Leading offset: from chunk
// to chunk; stride offset: from 8 rows to the next 8.
__device__ __forceinline__ uint64_t operand_descriptor(uint32_t address)
{
    constexpr uint64_t leading = (kTileT * 128) >> 4, stride = (8 * 128) >> 4;
    return static_cast<uint64_t>((address >> 4) & 0x3fff) | leading << 16 | stride << 32 | uint64_t{1} << 46 | uint64_t{2} << 61;
}

// bf16 x bf16 -> fp32, both operands MN-major, N columns.  M = 128, or 256 over a pair of blocks.
template <int N, bool PAIR> __device__ __forceinline__ constexpr uint32_t instruction_descriptor()
{
    return 1u << 4 | 1u << 7 | 1u << 10 | 1u << 15 | 1u << 16 | static_cast<uint32_t>(N / 8) << 17 |
           static_cast<uint32_t>((PAIR ? 2 : 1) * kTileC / 16) << 24;
}

template <bool PAIR> __device__ __forceinline__ void matrix_multiply(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool accumulate)
{
    if constexpr (PAIR)
        asm volatile("{\n\t.reg .pred p;\n\t"
                     "setp.ne.u32 p, %4, 0;\n\t"
                     "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                     :: "r"(d), "l"(a), "l"(b), "r"(idesc), "r"(static_cast<uint32_t>(accumulate)) : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\t"
                     "setp.ne.u32 p, %4, 0;\n\t"
                     "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                     :: "r"(d), "l"(a), "l"(b), "r"(idesc), "r"(static_cast<uint32_t>(accumulate)) : "memory");
}
// The barrier's phase advances once every matrix instruction issued so far is
// done; in a pair, that of the barrier at the same place in both blocks (mask).
template <bool PAIR> __device__ __forceinline__ void matrix_commit(uint32_t bar, uint32_t mask)
{
    if constexpr (PAIR)
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                     :: "r"(bar), "h"(static_cast<uint16_t>(mask)) : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" :: "r"(bar) : "memory");
}
// Accumulator memory of BN columns; whole warps, both blocks of a pair.
template <int BN, bool PAIR> __device__ __forceinline__ void tensor_alloc(uint32_t at)
{
    if constexpr (PAIR) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" :: "r"(at), "n"(BN) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    } else {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" :: "r"(at), "n"(BN) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
}
template <int BN, bool PAIR> __device__ __forceinline__ void tensor_free(uint32_t tmem)
{
    if constexpr (PAIR)
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" :: "r"(tmem), "n"(BN));
    else
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" :: "r"(tmem), "n"(BN));
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

__device__ __forceinline__ void store_accumulator(uint32_t address, const float (&x)[32])
{
    uint32_t r[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) r[i] = __float_as_uint(x[i]);
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
                 "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
                 "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};"
                 :: "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
                    "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]),
                    "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]),
                    "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]), "r"(address)
                 : "memory");
    asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}

// ---------------------------------------------------------------------------
// Widening.  With u = code + 128 in 0 .. 255, the float with bits 0x4b0000uu is
// 2^23 + u; fma(that, 2^e, -(2^23 + 128) 2^e) = code * 2^e, exact, and exact in
// bf16: its upper half.  A byte permutation, an fma per code and half a
// permutation to pack: 2.75 instructions a code.
// ---------------------------------------------------------------------------
__device__ __forceinline__ uint2 widen_codes(uint32_t four, float scale, float off)
{
    const uint32_t u = four ^ 0x80808080u;
    float f[4];
    f[0] = __fmaf_rn(__uint_as_float(__byte_perm(u, 0x4b000000u, 0x7650)), scale, off);
    f[1] = __fmaf_rn(__uint_as_float(__byte_perm(u, 0x4b000000u, 0x7651)), scale, off);
    f[2] = __fmaf_rn(__uint_as_float(__byte_perm(u, 0x4b000000u, 0x7652)), scale, off);
    f[3] = __fmaf_rn(__uint_as_float(__byte_perm(u, 0x4b000000u, 0x7653)), scale, off);
    return make_uint2(__byte_perm(__float_as_uint(f[0]), __float_as_uint(f[1]), 0x7632),
                      __byte_perm(__float_as_uint(f[2]), __float_as_uint(f[3]), 0x7632));
}
__device__ __forceinline__ uint4 widen_codes(uint2 eight, float scale, float off)
{
    const uint2 a = widen_codes(eight.x, scale, off), b = widen_codes(eight.y, scale, off);
    return make_uint4(a.x, a.y, b.x, b.y);
}

// ---------------------------------------------------------------------------
// A dy that the TMA does not read as it is: fp32 (three terms) or rows off the
// 16-byte grid.  The widening warps fetch it themselves, eight neighbouring
// outputs of a row a thread.
// ---------------------------------------------------------------------------
struct DyEight {
    uint32_t w[8];       // fp32: the values; bf16: the first four words, or two 16-byte loads around them
};

// bf16 off the 16-byte grid: eight values lie within two aligned 16-byte pieces.
// Where those are inside the matrix, *shift is the values' offset in them; -1 if not.
__device__ __forceinline__ const uint4 *around_eight(const WeightGradArgs &a, int64_t t, int64_t o, int *shift)
{
    const uintptr_t p = reinterpret_cast<uintptr_t>(a.dy) + static_cast<uintptr_t>((t * a.ld_dy + o) * 2), at = p & ~uintptr_t{15};
    const uintptr_t from = reinterpret_cast<uintptr_t>(a.dy), to = from + static_cast<uintptr_t>(((a.kept.rows - 1) * a.ld_dy + a.outs) * 2);
    const bool inside = t < a.kept.rows && o + 8 <= a.outs && at >= from && at + 32 <= to;
    *shift = inside ? static_cast<int>(p & 15u) : -1;
    return reinterpret_cast<const uint4 *>(at);
}

template <int TERMS> __device__ __forceinline__ void load_dy(const WeightGradArgs &a, int64_t t, int64_t o, bool vector, DyEight &r)
{
    using G = std::conditional_t<TERMS == 3, GradF32, GradBF16>;
    const char *p = static_cast<const char *>(a.dy) + (t * a.ld_dy + o) * G::kBytes;
    if constexpr (TERMS == 1) {
        int shift;
        const uint4 *at = around_eight(a, t, o, &shift);
        if (shift >= 0) {
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const uint4 v = at[q];
                r.w[4 * q] = v.x; r.w[4 * q + 1] = v.y; r.w[4 * q + 2] = v.z; r.w[4 * q + 3] = v.w;
            }
            return;
        }
    } else if (vector && t < a.kept.rows && o + 8 <= a.outs) {
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const uint4 v = reinterpret_cast<const uint4 *>(p)[q];
            r.w[4 * q] = v.x; r.w[4 * q + 1] = v.y; r.w[4 * q + 2] = v.z; r.w[4 * q + 3] = v.w;
        }
        return;
    }
    const int left = t < a.kept.rows ? static_cast<int>(min(a.outs - o, int64_t{8})) : 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) r.w[e] = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if (e < left) {
            if constexpr (TERMS == 3)
                r.w[e] = reinterpret_cast<const uint32_t *>(p)[e];
            else
                r.w[e / 2] |= static_cast<uint32_t>(reinterpret_cast<const unsigned short *>(p)[e]) << (e % 2 * 16);
        }
    }
}

// The eight bf16 of what load_dy<1> fetched.
__device__ __forceinline__ uint4 eight_bf16(const WeightGradArgs &a, int64_t t, int64_t o, DyEight r)
{
    int shift;
    around_eight(a, t, o, &shift);
    if (shift > 0) {
#pragma unroll
        for (int e = 0; e < 6; ++e) r.w[e] = shift & 8 ? r.w[e + 2] : r.w[e];
#pragma unroll
        for (int e = 0; e < 5; ++e) r.w[e] = shift & 4 ? r.w[e + 1] : r.w[e];
#pragma unroll
        for (int e = 0; e < 4; ++e) r.w[e] = __funnelshift_r(r.w[e], r.w[e + 1], (shift & 2) * 8);
    }
    return make_uint4(r.w[0], r.w[1], r.w[2], r.w[3]);
}

// Cuts eight fp32 into three bf16 each: the upper half of the value, of what is
// left, and of what is then left.  A value that is not finite is its first term
// (a NaN stays one: its quiet bit lies in the upper half).
__device__ __forceinline__ void cut_dy(const DyEight &v, uint4 (&term)[3])
{
    uint32_t first[8], second[8], third[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float x = __uint_as_float(v.w[e]);
        const bool finite = fabsf(x) < INFINITY;
        first[e] = x != x ? v.w[e] | 0x00400000u : v.w[e];
        const float rest = finite ? __fsub_rn(x, __uint_as_float(v.w[e] & 0xffff0000u)) : 0.0f;
        second[e] = __float_as_uint(rest);
        third[e] = __float_as_uint(__fsub_rn(rest, __uint_as_float(second[e] & 0xffff0000u)));
    }
    const auto upper = [](const uint32_t (&w)[8]) {
        return make_uint4(__byte_perm(w[0], w[1], 0x7632), __byte_perm(w[2], w[3], 0x7632), __byte_perm(w[4], w[5], 0x7632),
                          __byte_perm(w[6], w[7], 0x7632));
    };
    term[0] = upper(first);
    term[1] = upper(second);
    term[2] = upper(third);
}

// Shared memory of a block, from a 1024-byte aligned base: a ring of LOADS steps
// as they are fetched (codes, scale bytes, dy), and a shorter one of WIDE steps
// of the widened operand.  A step's copies take a microsecond or more under load
// and its products a quarter of one, so the first ring has to be deep.  TERMS = 0:
// dy comes by TMA and is an operand as it lies; otherwise its TERMS terms are
// written beside the widened operand.
template <int BN, int LOADS, int WIDE, bool PAIR, int TERMS> struct GradSmem {
    static constexpr int kN = BN < kTileO ? BN : kTileO;         // outputs of one matrix instruction
    static_assert(BN % kN == 0, "whole instructions");
    static constexpr int kOuts = PAIR ? BN / 2 : BN;             // outputs whose dy this block holds
    static constexpr int kRun = PAIR ? kN / 2 : kN;              // of them, side by side: this block's share of one instruction
    static constexpr int kA = kTileC * kTileT * 2;
    static constexpr int kB = kOuts * kTileT * 2;
    static constexpr int kBSlots = TERMS == 0 ? LOADS : WIDE * TERMS;
    static constexpr int kRaw = kTileC * kTileT;
    static constexpr int kScale = kTileT * 4;
    static constexpr int kOffB = WIDE * kA;
    static constexpr int kOffRaw = kOffB + kBSlots * kB;
    static constexpr int kOffScale = kOffRaw + LOADS * kRaw;
    static constexpr int kOffBarrier = kOffScale + LOADS * kScale;
    static constexpr int kBytes = kOffBarrier + 256;
    static constexpr int kDynamic = kBytes + 1024;               // room to align the base
    static_assert(WIDE <= LOADS && 8 * (2 * LOADS + WIDE + 4) <= 256, "barriers");
    static_assert(kTileC * kN * 4 <= kOffBarrier, "the accumulators of a split tile reuse the rings");
    static_assert(kDynamic <= 232448, "more shared memory than a block may have");
};

__device__ __forceinline__ float4 peer_load(uint32_t address)
{
    float4 x;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(x.x), "=f"(x.y), "=f"(x.z), "=f"(x.w) : "r"(address));
    return x;
}

// The sums of a split tile: part `part` adds its share of the columns over the
// parts' accumulators (in their shared memory, N * kTileC values), in the order of
// the parts, all loads of a sum in flight together.  store(i, x): the i-th four.
template <int PARTS, int N, typename Store>
__device__ __forceinline__ void join_parts(uint32_t sums, int part, uint32_t of_pair, uint32_t blocks, Store store)
{
    const int first = N * part / PARTS, last = N * (part + 1) / PARTS;
    for (int i = first * (kTileC / 4) + threadIdx.x; i < last * (kTileC / 4); i += kGradThreads) {
        float4 x[PARTS];
#pragma unroll
        for (int q = 0; q < PARTS; ++q) x[q] = peer_load(peer_address(sums + static_cast<uint32_t>(i) * 16, of_pair + blocks * q));
#pragma unroll
        for (int q = 1; q < PARTS; ++q) {
            x[0].x = __fadd_rn(x[0].x, x[q].x);
            x[0].y = __fadd_rn(x[0].y, x[q].y);
            x[0].z = __fadd_rn(x[0].z, x[q].z);
            x[0].w = __fadd_rn(x[0].w, x[q].w);
        }
        store(i, x[0]);
    }
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

// dst[0 .. 32) = x, or += x, in 32-byte accesses; values of BYTES each.
template <int BYTES> __device__ __forceinline__ void add_and_store(char *dst, const float (&x)[32], bool accumulate)
{
#pragma unroll
    for (int half = 0; half < BYTES / 2; ++half, dst += 64) {            // two accesses at a time
        uint32_t before[2][8];
        if (accumulate) {
            load_words(dst, before[0]);
            load_words(dst + 32, before[1]);
        }
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            uint32_t w[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if constexpr (BYTES == 4) {
                    const float v = x[16 * half + 8 * q + e];
                    w[e] = __float_as_uint(accumulate ? __fadd_rn(v, __uint_as_float(before[q][e])) : v);
                } else {
                    float lo = x[16 * q + 2 * e], hi = x[16 * q + 2 * e + 1];
                    if (accumulate) {
                        lo = __fadd_rn(lo, __uint_as_float(before[q][e] << 16));
                        hi = __fadd_rn(hi, __uint_as_float(before[q][e] & 0xffff0000u));
                    }
                    w[e] = pack_bf16(lo, hi);
                }
            }
            store_words(dst + 32 * q, w);
        }
    }
}

// A warp's 32 columns c0 .. and 32 outputs o0 .. (x[r]: output o0 + r of this
// lane's column).  `words`: pairs of bf16 at even columns lie on whole words.
// Plain layout: neighbouring lanes trade halves, so that each stores two columns
// of every other output; fp32 needs no trade.  Transposed, a lane's outputs are
// neighbours in memory (2048 rows, 4096 -> 4096, fp32: 32-byte accesses 73 us, words
// 161).  What is added to is loaded ahead of the stores, 16 words at a time: the compiler cannot move a load
// over a store that might change it.
__device__ __forceinline__ void store_block(const WeightGradArgs &a, bool bf16, bool words, int64_t o0, int64_t c0, int lane, const float (&x)[32])
{
    const int64_t c = c0 + lane;
    if (bf16 && words && a.stride_c == 1 && o0 + 32 <= a.outs && c0 + 32 <= a.kept.cols) {
        const int odd = lane & 1;
        uint32_t *dst = reinterpret_cast<uint32_t *>(static_cast<unsigned short *>(a.dw) + (o0 + odd) * a.stride_o + (c - odd));
        const int64_t two_rows = a.stride_o;                     // two outputs further, in words
        uint32_t before[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) before[r] = a.accumulate ? dst[r * two_rows] : 0u;
#pragma unroll
        for (int r = 0; r < 32; r += 2, dst += two_rows) {
            const float mine = odd ? x[r + 1] : x[r], theirs = __shfl_xor_sync(0xffffffffu, odd ? x[r] : x[r + 1], 1);
            float lo = odd ? theirs : mine, hi = odd ? mine : theirs;
            if (a.accumulate) {
                lo = __fadd_rn(lo, __uint_as_float(before[r / 2] << 16));
                hi = __fadd_rn(hi, __uint_as_float(before[r / 2] & 0xffff0000u));
            }
            *dst = pack_bf16(lo, hi);
        }
        return;
    }
    if (a.stride_o == 1 && o0 + 32 <= a.outs) {
        if (c >= a.kept.cols) return;
        char *dst = static_cast<char *>(a.dw) + (o0 + c * a.stride_c) * (bf16 ? 2 : 4);
        if (reinterpret_cast<uintptr_t>(dst) % 32 == 0) {        // whole sectors: a lane's outputs are neighbours
            if (bf16)
                add_and_store<2>(dst, x, a.accumulate);
            else
                add_and_store<4>(dst, x, a.accumulate);
            return;
        }
    }
    if (c >= a.kept.cols) return;
    const int left = static_cast<int>(min(a.outs - o0, int64_t{32}));
    if (!bf16) {
        float *dst = static_cast<float *>(a.dw) + o0 * a.stride_o + c * a.stride_c;
#pragma unroll
        for (int r0 = 0; r0 < 32; r0 += 16, dst += 16 * a.stride_o) {
            float before[16];
#pragma unroll
            for (int r = 0; r < 16; ++r) before[r] = a.accumulate && r0 + r < left ? dst[r * a.stride_o] : 0.0f;
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (r0 + r < left) dst[r * a.stride_o] = a.accumulate ? __fadd_rn(x[r0 + r], before[r]) : x[r0 + r];
        }
        return;
    }
#pragma unroll
    for (int r = 0; r < 32; ++r)
        if (r < left) store_weight(a, true, o0 + r, c, x[r]);
}

// Four neighbours along dw's rows: columns c .. of an output or, `swapped`, outputs
// o .. of a column.
__device__ __forceinline__ void store_four(const WeightGradArgs &a, bool bf16, bool words, bool swapped, int64_t o, int64_t c, float4 v)
{
    const int64_t left = swapped ? a.outs - o : a.kept.cols - c;
    if (left <= 0 || (swapped ? c >= a.kept.cols : o >= a.outs)) return;
    const int64_t at = o * a.stride_o + c * a.stride_c;
    if (bf16 && words && left >= 4) {
        uint32_t *dst = reinterpret_cast<uint32_t *>(static_cast<unsigned short *>(a.dw) + at);
        if (a.accumulate) {
            const uint32_t lo = dst[0], hi = dst[1];
            v.x = __fadd_rn(v.x, __uint_as_float(lo << 16));
            v.y = __fadd_rn(v.y, __uint_as_float(lo & 0xffff0000u));
            v.z = __fadd_rn(v.z, __uint_as_float(hi << 16));
            v.w = __fadd_rn(v.w, __uint_as_float(hi & 0xffff0000u));
        }
        dst[0] = pack_bf16(v.x, v.y);
        dst[1] = pack_bf16(v.z, v.w);
        return;
    }
    if (!bf16 && left >= 4) {
        float *dst = static_cast<float *>(a.dw) + at;
        if (reinterpret_cast<uintptr_t>(dst) % 16 == 0) {
            if (a.accumulate) {
                const float4 before = *reinterpret_cast<const float4 *>(dst);
                v = make_float4(__fadd_rn(v.x, before.x), __fadd_rn(v.y, before.y), __fadd_rn(v.z, before.z), __fadd_rn(v.w, before.w));
            }
            *reinterpret_cast<float4 *>(dst) = v;
            return;
        }
    }
    const float x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (e < left) store_weight(a, bf16, swapped ? o + e : o, swapped ? c : c + e, x[e]);
}

// grid: (column tiles, output tiles, parts of the rows); cluster: (1 or 2, 1, parts).
// Every part has a step at least.
//
// PAIR: two blocks with neighbouring column tiles work as one (cta_group::2).
// Each widens its own 128 columns and fetches half of the dy tile; the matrix
// instructions, issued by the first of the two, read both halves from both
// blocks.  One block alone is bound by its shared memory: per step of 64 rows
// the matrix instructions read 48 KB, the copies write 40 KB and the widening
// moves 24 KB, 112 KB where 128 B a cycle give 64 KB in the 512 cycles of the
// products.  In a pair that is 80 KB.
// FLUSH: the accumulator, and that of the lower terms, is added to a running sum beside
// it in TMEM every kFlushSteps steps.
constexpr int kFlushSteps = 20;

template <int BN, int LOADS, int WIDE, bool PAIR, int TERMS, bool FLUSH>
__global__ void __launch_bounds__(kGradThreads, 1)
star_weight_grad_tensor_kernel(const __grid_constant__ WeightGradTile p, const __grid_constant__ CUtensorMap codes_map,
                               const __grid_constant__ CUtensorMap dy_map, int dw_bf16)
{
    using S = GradSmem<BN, LOADS, WIDE, PAIR, TERMS>;
    // Columns of TMEM: the accumulator, the running sum, the lower terms' accumulator; a power of two.
    constexpr int kTmem = TERMS == 3 ? 4 * BN : FLUSH ? 2 * BN : BN, kLower = 2 * BN;
    static_assert(TERMS != 3 || (FLUSH && BN == S::kN), "one instruction's columns, summed");
    constexpr int kShare = BN / (kConvertWarps / 4);             // accumulator columns a converting warp reads at the end
    static_assert(kShare % 32 == 0, "whole loads");
    constexpr uint32_t kBlocks = PAIR ? 2 : 1;
    extern __shared__ uint8_t dynamic[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(dynamic) + 1023) & ~uintptr_t{1023});
    const uint32_t base = smem_address(smem);
    const uint32_t bars = base + S::kOffBarrier;
    const auto loaded = [&](int i) { return bars + 8 * (i % LOADS); };                       // step i's copies have landed
    const auto used = [&](int i) { return bars + 8 * (LOADS + i % LOADS); };                 // its matrix instructions are done
    const auto widened = [&](int i) { return bars + 8 * (2 * LOADS + i % WIDE); };           // its A operand is written (in both blocks)
    const auto load_phase = [](int i) { return static_cast<uint32_t>(i / LOADS) & 1; };
    const auto wide_phase = [](int i) { return static_cast<uint32_t>(i / WIDE) & 1; };
    const uint32_t finished = bars + 8 * (2 * LOADS + WIDE);
    const uint32_t summed = finished + 8;                        // FLUSH: a run's matrix instructions are done
    const uint32_t drained = finished + 16;                      // and its accumulator is read (in both blocks)
    uint32_t *tmem_at = reinterpret_cast<uint32_t *>(smem + S::kOffBarrier + 8 * (2 * LOADS + WIDE + 3));
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const uint32_t rank = cluster_rank(), of_pair = rank % kBlocks, leader = rank - of_pair;
    const uint32_t mask = 3u << leader;

    if (threadIdx.x == 0) {
        for (int i = 0; i < LOADS; ++i) {
            barrier_init(loaded(i), 1);
            barrier_init(used(i), 1);
        }
        for (int i = 0; i < WIDE; ++i) barrier_init(widened(i), kBlocks * kGroupWarps);
        barrier_init(finished, 1);
        barrier_init(summed, 1);
        barrier_init(drained, kBlocks * kConvertWarps);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    // Taking TMEM waits without limit for whoever holds it, so a block that waits for the
    // kernel in front must not hold any that that kernel may still ask for.
    wait_for_primary();
    if (warp == 2) tensor_alloc<kTmem, PAIR>(smem_address(tmem_at));
    tensor_fence_before();
    __syncthreads();
    if constexpr (PAIR) cluster_sync();                          // the other block's barriers are ready
    tensor_fence_after();
    const uint32_t tmem = *tmem_at;

    const int64_t c0 = static_cast<int64_t>(blockIdx.x) * kTileC, o0 = static_cast<int64_t>(blockIdx.y) * BN;
    const int parts = static_cast<int>(gridDim.z), part = static_cast<int>(blockIdx.z);
    const int first = static_cast<int>(static_cast<int64_t>(p.steps) * part / parts);
    const int last = static_cast<int>(static_cast<int64_t>(p.steps) * (part + 1) / parts);
    bool ok = true;

    if (warp == 0) {
        if (lane == 0) {
            // The second block of a pair may lie past the last column tile: its
            // codes read as zero, its scales are those of the last tile.
            const int64_t scale_tile = min(static_cast<int64_t>(blockIdx.x), (p.a.kept.cols - 1) / kTileC);
            const uint8_t *scales = p.a.kept.scales + scale_tile * p.a.kept.tall * 4;
            const int outs0 = static_cast<int>(o0) + static_cast<int>(of_pair) * S::kRun;
            int issued = 0;
            for (int k = first; k < last; ++k) {
                const int i = k - first, s = i % LOADS;
                if (i >= LOADS && !barrier_wait(used(i - LOADS), load_phase(i - LOADS), p.tries)) break;
                barrier_expect(loaded(i), S::kRaw + S::kScale + (TERMS == 0 ? S::kB : 0));
                const int t = k * kTileT;
                tma_load_2d(base + S::kOffRaw + s * S::kRaw, &codes_map, static_cast<int>(c0), t, loaded(i));
                bulk_load(base + S::kOffScale + s * S::kScale, scales + static_cast<int64_t>(t) * 4, S::kScale, loaded(i));
                if constexpr (TERMS == 0) {
#pragma unroll
                    for (int q = 0; q < S::kOuts / 64; ++q)
                        tma_load_2d(base + S::kOffB + s * S::kB + q * (kTileT * 128), &dy_map,
                                    outs0 + 64 * q / S::kRun * S::kN + 64 * q % S::kRun, t, loaded(i));
                }
                issued = i + 1;
            }
            // Copies still in flight land before the block goes on (they have, unless a wait ran out).
            for (int i = issued > LOADS ? issued - LOADS : 0; i < issued; ++i) barrier_wait(loaded(i), load_phase(i), kWaitTries);
        }
    } else if (warp == 1) {
        if (lane == 0 && of_pair == 0) {
            constexpr uint32_t idesc = instruction_descriptor<S::kN, PAIR>();
            for (int k = first; k < last && ok; ++k) {
                const int i = k - first, in_run = FLUSH ? i % kFlushSteps : i;
                if (FLUSH && i > 0 && in_run == 0) ok = barrier_wait(drained, (i / kFlushSteps - 1) & 1, p.tries);
                // The widening warps of both blocks have seen their block's copies land.
                ok = ok && barrier_wait(loaded(i), load_phase(i), p.tries) && barrier_wait(widened(i), wide_phase(i), p.tries);
                if (!ok) break;
                tensor_fence_after();
                const uint32_t as = base + (i % WIDE) * S::kA;
                const uint32_t bs = base + S::kOffB + (TERMS == 0 ? i % LOADS : i % WIDE * TERMS) * S::kB;
#pragma unroll
                for (int q = 0; q < kTileT / 16; ++q)                // 16 rows an instruction
#pragma unroll
                    for (int n = 0; n < BN / S::kN; ++n)
#pragma unroll
                        for (int term = 0; term < (TERMS == 0 ? 1 : TERMS); ++term)
                            matrix_multiply<PAIR>(tmem + n * S::kN + (term > 0 ? kLower : 0), operand_descriptor(as + q * 2048),
                                                  operand_descriptor(bs + term * S::kB + n * (S::kRun * kTileT * 2) + q * 2048), idesc,
                                                  in_run > 0 || q > 0 || term > 1);
                matrix_commit<PAIR>(used(i), mask);
                if (FLUSH && in_run == kFlushSteps - 1 && k + 1 < last) matrix_commit<PAIR>(summed, mask);
            }
            matrix_commit<PAIR>(finished, mask);
        }
    } else if (warp >= kFirstConvert) {
        // Thread w of a group widens 16 codes of rows w / 8 + 32 h: their place is the
        // same in every step.  Eight neighbouring threads fill one 128-byte row in
        // each half of the operand; those of the upper half start with their second
        // eight codes, so that no bank is hit twice.
        constexpr int kRows = 32 * kGroupWarps / 8;
        const int w = (threadIdx.x - 32 * kFirstConvert) % (32 * kGroupWarps), t0 = w / 8, j = w % 8, swap = j / 4;
        static_assert(kRows % 8 == 0, "the swizzle depends on the row modulo 8");
        const int from = t0 * kTileC + j * 16, to = swap * (kTileT * 128) + t0 * 128;
        const int to0 = to + (((2 * (j % 4) + swap) ^ (t0 % 8)) << 4), to1 = to + (((2 * (j % 4) + 1 - swap) ^ (t0 % 8)) << 4);
        // FLUSH: adds this warp's part of run `run`'s accumulator to the running sum.
        const int quarter = warp % 4, share = (warp - kFirstConvert) / 4;
        int run = 0;
        const auto drain = [&] {
            if (!barrier_wait(summed, run & 1, p.tries)) return false;
            tensor_fence_after();
            for (int col = share * kShare; col < (share + 1) * kShare; col += 32) {
                const uint32_t at = tmem + (static_cast<uint32_t>(quarter * 32) << 16) + col;
                float x[32];
                load_accumulator(at, x);
                if constexpr (TERMS == 3) {
                    float lower[32];
                    load_accumulator(at + kLower, lower);
#pragma unroll
                    for (int r = 0; r < 32; ++r) x[r] = __fadd_rn(x[r], lower[r]);
                }
                if (run > 0) {
                    float sum[32];
                    load_accumulator(at + BN, sum);
#pragma unroll
                    for (int r = 0; r < 32; ++r) x[r] = __fadd_rn(x[r], sum[r]);
                }
                store_accumulator(at + BN, x);
            }
            tensor_fence_before();
            __syncwarp();
            if (lane == 0) barrier_arrive(peer_address(drained, leader));
            ++run;
            return true;
        };
        const int runs = FLUSH ? (last - first + kFlushSteps - 1) / kFlushSteps : 1;
        const bool vector = TERMS == 0 || (reinterpret_cast<uintptr_t>(p.a.dy) % 16 == 0 && p.a.ld_dy * (TERMS == 3 ? 4 : 2) % 16 == 0);
        constexpr int kEights = TERMS == 0 ? 1 : S::kOuts * kTileT / 8 / (32 * kGroupWarps);
        DyEight dy[kEights];
        const auto fetch_dy = [&](int k) {
#pragma unroll
            for (int h = 0; h < kEights; ++h) {
                const int unit = w + h * 32 * kGroupWarps, t = unit / (S::kOuts / 8), j = unit % (S::kOuts / 8);
                load_dy<TERMS>(p.a, static_cast<int64_t>(k) * kTileT + t, o0 + of_pair * S::kRun + j * 8, vector, dy[h]);
            }
        };
        for (int k = first + (warp - kFirstConvert) / kGroupWarps; k < last; k += kGroups) {
            const int i = k - first, s = i % LOADS;
            if constexpr (FLUSH) {
                while (ok && run < i / kFlushSteps) ok = drain();
                if (!ok) break;
            }
            // TERMS > 0: the step's dy is on its way while the codes are widened.
            if constexpr (TERMS > 0) fetch_dy(k);
            ok = (i < WIDE || barrier_wait(used(i - WIDE), load_phase(i - WIDE), p.tries)) && barrier_wait(loaded(i), load_phase(i), p.tries);
            if (!ok) break;
            const uint8_t *raw = smem + S::kOffRaw + s * S::kRaw + from, *scale = smem + S::kOffScale + s * S::kScale + t0 * 4 + j / 2;
            uint8_t *as = smem + (i % WIDE) * S::kA;
            const int64_t left = p.a.kept.rows - static_cast<int64_t>(k) * kTileT;   // rows past the end have codes 0 and no scale
            const int rows = static_cast<int>(min(left, static_cast<int64_t>(kTileT)));
#pragma unroll
            for (int h = 0; h < kTileT / kRows; ++h) {
                const uint2 c0 = *reinterpret_cast<const uint2 *>(raw + h * kRows * kTileC + 8 * swap);
                const uint2 c1 = *reinterpret_cast<const uint2 *>(raw + h * kRows * kTileC + 8 - 8 * swap);
                const float f = t0 + h * kRows < rows ? scale_value(scale[h * kRows * 4]) : 0.0f, off = __fmul_rn(f, -8388736.0f);
                *reinterpret_cast<uint4 *>(as + h * kRows * 128 + to0) = widen_codes(c0, f, off);
                *reinterpret_cast<uint4 *>(as + h * kRows * 128 + to1) = widen_codes(c1, f, off);
            }
            if constexpr (TERMS > 0) {
                uint8_t *bs = smem + S::kOffB + (i % WIDE) * TERMS * S::kB;
#pragma unroll
                for (int h = 0; h < kEights; ++h) {
                    const int unit = w + h * 32 * kGroupWarps, t = unit / (S::kOuts / 8), j = unit % (S::kOuts / 8);
                    uint4 *at = reinterpret_cast<uint4 *>(bs + j / 8 * (kTileT * 128) + t * 128 + ((j % 8) ^ (t % 8)) * 16);
                    if constexpr (TERMS == 3) {
                        uint4 term[3];
                        cut_dy(dy[h], term);
#pragma unroll
                        for (int q = 0; q < 3; ++q) at[q * (S::kB / 16)] = term[q];
                    } else {
                        *at = eight_bf16(p.a, static_cast<int64_t>(k) * kTileT + t, o0 + of_pair * S::kRun + j * 8, dy[h]);
                    }
                }
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) barrier_arrive(peer_address(widened(i), leader));
        }
        if constexpr (FLUSH)
            while (ok && run + 1 < runs) ok = drain();
    }

    // The result: every warp waits for the last matrix instruction itself, also where
    // other waits ran out.
    __syncwarp();                        // the idle lanes of a role do not spin beside it
    ok = barrier_wait(finished, 0, kWaitTries) && ok;
    const bool whole = __syncthreads_and(ok);
    tensor_fence_after();
    const int quarter = warp % 4, share = (warp - kFirstConvert) / 4;            // of a converting warp
    const bool words = reinterpret_cast<uintptr_t>(p.a.dw) % 4 == 0 && (p.a.stride_c == 1 ? p.a.stride_o : p.a.stride_c) % 2 == 0;
    // 32 columns of the result in this warp's lanes, from column `col` on.
    const auto result = [&](int col, float (&x)[32]) {
        const uint32_t at = tmem + (static_cast<uint32_t>(quarter * 32) << 16) + col;
        load_accumulator(at, x);
        if (FLUSH && last - first > kFlushSteps) {
            float sum[32];
            load_accumulator(at + BN, sum);
#pragma unroll
            for (int r = 0; r < 32; ++r) x[r] = __fadd_rn(x[r], sum[r]);
        }
        if constexpr (TERMS == 3) {
            float lower[32];
            load_accumulator(at + kLower, lower);
#pragma unroll
            for (int r = 0; r < 32; ++r) x[r] = __fadd_rn(x[r], lower[r]);
        }
    };
    if (parts == 1) {
        if (whole && warp >= kFirstConvert) {
            for (int col = share * kShare; col < (share + 1) * kShare; col += 32) {
                float x[32];
                result(col, x);
                store_block(p.a, dw_bf16, words, o0 + col, c0 + quarter * 32, lane, x);
            }
        }
    } else {
        // [kN][kTileC], or [kTileC][kN] in fours that trade places within eight, so
        // that neither these stores nor the loads of the join collide in the banks.
        float *sums = reinterpret_cast<float *>(smem);
        const bool swapped = p.a.stride_o == 1 && p.a.stride_c != 1;
        constexpr int kPart = S::kN / (kConvertWarps / 4);
        for (int n = 0; n < BN / S::kN; ++n) {
            if (warp >= kFirstConvert) {
                for (int col = share * kPart; col < (share + 1) * kPart; col += 32) {
                    float x[32];
                    result(n * S::kN + col, x);
                    const int c = quarter * 32 + lane;
                    if (swapped) {
                        float4 *row = reinterpret_cast<float4 *>(sums + c * S::kN);
#pragma unroll
                        for (int r = 0; r < 8; ++r) row[(col / 4 + r) ^ (c & 7)] = make_float4(x[4 * r], x[4 * r + 1], x[4 * r + 2], x[4 * r + 3]);
                    } else {
#pragma unroll
                        for (int r = 0; r < 32; ++r) sums[(col + r) * kTileC + c] = x[r];
                    }
                }
            }
            __syncthreads();
            cluster_sync();
            if (whole) {
                const auto store = [&](int i, float4 x) {
                    const int c = swapped ? i / (S::kN / 4) : i % (kTileC / 4) * 4;
                    const int o = swapped ? (i % (S::kN / 4) ^ (c & 7)) * 4 : i / (kTileC / 4);
                    store_four(p.a, dw_bf16, words, swapped, o0 + n * S::kN + o, c0 + c, x);
                };
                switch (parts) {
                case 2: join_parts<2, S::kN>(base, part, of_pair, kBlocks, store); break;
                case 3: join_parts<3, S::kN>(base, part, of_pair, kBlocks, store); break;
                case 4: join_parts<4, S::kN>(base, part, of_pair, kBlocks, store); break;
                case 5: join_parts<5, S::kN>(base, part, of_pair, kBlocks, store); break;
                case 6: join_parts<6, S::kN>(base, part, of_pair, kBlocks, store); break;
                case 7: join_parts<7, S::kN>(base, part, of_pair, kBlocks, store); break;
                default: join_parts<8, S::kN>(base, part, of_pair, kBlocks, store); break;
                }
            }
            if (n + 1 < BN / S::kN) {
                __syncthreads();
                cluster_sync();                                      // the sums are read before the next ones come
            }
        }
    }
    tensor_fence_before();
    __syncthreads();
    if (PAIR || parts > 1) cluster_sync();                           // nobody leaves while a peer reads its memory or signals it
    if (warp == 2) tensor_free<kTmem, PAIR>(tmem);
}

// ---------------------------------------------------------------------------
// Few rows: the time goes into writing dw, and a tile of the tensor cores would
// cost more in its preparation than in its products.  Outer products in binary32
// on the ordinary units: a block makes 64 x 256 results, a thread 8 x 8 of them,
// rows 32 at a time in shared memory.  The result's inner index, along which dw
// is stored, runs over the lanes: columns, or outputs where dw is transposed.
// 4096 x 4096 from 1 row: bf16 10 us (3.3 TB/s), fp32 14.5 (4.6 TB/s); added to 12.7 and 16.1.
// ---------------------------------------------------------------------------
constexpr int kFewRows = 32, kFewOuter = 64, kFewInner = 256, kFewThreads = 256;

// dw[at .. at + left) as four values, 0 beyond.
template <typename GW> __device__ __forceinline__ void load_four(const void *dw, int64_t at, bool whole, int left, float (&x)[4])
{
    if (whole) {
        if constexpr (GW::kBytes == 2) {
            const uint2 w = *reinterpret_cast<const uint2 *>(static_cast<const unsigned short *>(dw) + at);
            x[0] = __uint_as_float(w.x << 16);
            x[1] = __uint_as_float(w.x & 0xffff0000u);
            x[2] = __uint_as_float(w.y << 16);
            x[3] = __uint_as_float(w.y & 0xffff0000u);
        } else {
            const float4 w = *reinterpret_cast<const float4 *>(static_cast<const float *>(dw) + at);
            x[0] = w.x;
            x[1] = w.y;
            x[2] = w.z;
            x[3] = w.w;
        }
    } else {
#pragma unroll
        for (int q = 0; q < 4; ++q) x[q] = q < left ? load_value<GW>(dw, at + q) : 0.0f;
    }
}

template <typename GY, typename GW, bool TRANSPOSED>
__global__ void __launch_bounds__(kFewThreads, 2) star_weight_grad_few_kernel(const __grid_constant__ WeightGradArgs a, int vector)
{
    __shared__ alignas(16) float outer[kFewRows][kFewOuter], inner[kFewRows][kFewInner];
    const int64_t n_outer = TRANSPOSED ? a.kept.cols : a.outs, n_inner = TRANSPOSED ? a.outs : a.kept.cols;
    const int64_t i0 = static_cast<int64_t>(blockIdx.y) * kFewOuter, j0 = static_cast<int64_t>(blockIdx.x) * kFewInner;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const auto value = [&](int64_t t, int64_t c) {
        return __fmul_rn(static_cast<float>(a.kept.codes[t * a.kept.pitch + c]), scale_value(a.kept.scales[scale_at(a.kept, t, c / 32)]));
    };
    const auto gradient = [&](int64_t t, int64_t o) { return load_value<GY>(a.dy, t * a.ld_dy + o); };
    float sum[8][8];
#pragma unroll
    for (int p = 0; p < 8; ++p)
#pragma unroll
        for (int q = 0; q < 8; ++q) sum[p][q] = 0.0f;
    wait_for_primary();
    for (int64_t t0 = 0; t0 < a.kept.rows; t0 += kFewRows) {
        const int rows = static_cast<int>(min(a.kept.rows - t0, static_cast<int64_t>(kFewRows)));
        if (t0 > 0) __syncthreads();
        static_assert(kFewThreads == kFewInner, "a thread fetches one inner index of every row");
        const int64_t j = j0 + threadIdx.x;
#pragma unroll 8
        for (int t = 0; t < rows; ++t) {
            float x = 0.0f;
            if (j < n_inner) x = TRANSPOSED ? gradient(t0 + t, j) : value(t0 + t, j);
            inner[t][threadIdx.x] = x;
        }
#pragma unroll 4
        for (int e = threadIdx.x; e < rows * kFewOuter; e += kFewThreads) {
            const int t = e / kFewOuter, i = e % kFewOuter;
            float x = 0.0f;
            if (i0 + i < n_outer) x = TRANSPOSED ? value(t0 + t, i0 + i) : gradient(t0 + t, i0 + i);
            outer[t][i] = x;
        }
        __syncthreads();
        for (int t = 0; t < rows; ++t) {
            const float4 x0 = *reinterpret_cast<const float4 *>(&inner[t][4 * lane]), x1 = *reinterpret_cast<const float4 *>(&inner[t][128 + 4 * lane]);
            const float4 y0 = *reinterpret_cast<const float4 *>(&outer[t][8 * warp]), y1 = *reinterpret_cast<const float4 *>(&outer[t][8 * warp + 4]);
            const float x[8] = {x0.x, x0.y, x0.z, x0.w, x1.x, x1.y, x1.z, x1.w}, y[8] = {y0.x, y0.y, y0.z, y0.w, y1.x, y1.y, y1.z, y1.w};
#pragma unroll
            for (int p = 0; p < 8; ++p)
#pragma unroll
                for (int q = 0; q < 8; ++q) sum[p][q] = __fmaf_rn(y[p], x[q], sum[p][q]);
        }
    }
    // Columns 4 lane .. + 3 of each half of the 256, four rows of them at a time: what
    // they are added to is loaded ahead of the stores.  Whole tiles without branches.
    const int64_t ld = TRANSPOSED ? a.stride_c : a.stride_o;
    const auto results = [&](auto whole) {
#pragma unroll
        for (int p0 = 0; p0 < 8; p0 += 4) {
            float before[8][4];
            if (a.accumulate) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int64_t i = i0 + 8 * warp + p0 + e / 2, j = j0 + e % 2 * 128 + 4 * lane, at = i * ld + j;
                    const int left = whole.value ? 4 : i < n_outer ? static_cast<int>(min(n_inner - j, int64_t{4})) : 0;
                    load_four<GW>(a.dw, at, whole.value, left, before[e]);
                }
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int p = p0 + e / 2, half = e % 2;
                const int64_t i = i0 + 8 * warp + p, j = j0 + half * 128 + 4 * lane, at = i * ld + j;
                const int left = whole.value ? 4 : i < n_outer ? static_cast<int>(min(n_inner - j, int64_t{4})) : 0;
                float v[4] = {sum[p][4 * half], sum[p][4 * half + 1], sum[p][4 * half + 2], sum[p][4 * half + 3]};
                if (a.accumulate) {
#pragma unroll
                    for (int q = 0; q < 4; ++q) v[q] = __fadd_rn(v[q], before[e][q]);
                }
                if constexpr (whole.value) {
                    if constexpr (GW::kBytes == 2)
                        *reinterpret_cast<uint2 *>(static_cast<unsigned short *>(a.dw) + at) = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]));
                    else
                        *reinterpret_cast<float4 *>(static_cast<float *>(a.dw) + at) = make_float4(v[0], v[1], v[2], v[3]);
                } else {
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        if (q < left) store_value<GW>(a.dw, at + q, v[q]);
                }
            }
        }
    };
    if (vector && i0 + kFewOuter <= n_outer && j0 + kFewInner <= n_inner)
        results(std::true_type());
    else
        results(std::false_type());
}

}  // namespace star
