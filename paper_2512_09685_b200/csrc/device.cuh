// Device helpers shared by the operators of a worker's step (sm_100a).
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "kernels.cuh"

namespace star {

// 2^x, 2 ulp; -inf gives 0, NaN stays NaN.
__device__ __forceinline__ float exp2_fast(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

constexpr float kLog2e = 1.44269504088896340736f;
// Element i of a buffer of type G (GradF32 or GradBF16), widened.
template <typename G> __device__ __forceinline__ float load_value(const void *base, int64_t i)
{
    if constexpr (G::kBytes == 2)
        return __uint_as_float(static_cast<uint32_t>(static_cast<const unsigned short *>(base)[i]) << 16);
    else
        return static_cast<const float *>(base)[i];
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

template <typename G> __device__ __forceinline__ void store_value(void *base, int64_t i, float x)
{
    if constexpr (G::kBytes == 2)
        static_cast<unsigned short *>(base)[i] = static_cast<unsigned short>(pack_bf16(x, 0.0f));
    else
        static_cast<float *>(base)[i] = x;
}

// Two binary32 values worked on by one instruction.
using Pair = unsigned long long;
__device__ __forceinline__ Pair make_pair(float lo, float hi)
{
    Pair r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void split_pair(Pair p, float *lo, float *hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(*lo), "=f"(*hi) : "l"(p)); }
__device__ __forceinline__ Pair pair_add(Pair a, Pair b)
{
    Pair r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ Pair pair_mul(Pair a, Pair b)
{
    Pair r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ Pair pair_fma(Pair a, Pair b, Pair c)
{
    Pair r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}

__device__ __forceinline__ Pair pair_of(float x) { return make_pair(x, x); }
__device__ __forceinline__ Pair pair_exp2(Pair p)
{
    float lo, hi;
    split_pair(p, &lo, &hi);
    return make_pair(exp2_fast(lo), exp2_fast(hi));
}
// 1 / x, 1 ulp; 0 for an infinite x.
__device__ __forceinline__ float reciprocal_fast(float x)
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ Pair pair_reciprocal(Pair p)
{
    float lo, hi;
    split_pair(p, &lo, &hi);
    return make_pair(reciprocal_fast(lo), reciprocal_fast(hi));
}

// ---------------------------------------------------------------------------
// Shared memory, clusters, and launches that follow one another.
// ---------------------------------------------------------------------------
__device__ __forceinline__ uint32_t smem_address(const void *p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }
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
__device__ __forceinline__ uint32_t cluster_size()
{
    uint32_t r;
    asm("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(r));
    return r;
}

// ---------------------------------------------------------------------------
// Barriers in shared memory.  Every wait ends: after `tries` attempts it sets a
// flag that star_check_waits reads and reports failure, upon which the kernel takes
// up no further work, waits for its copies and matrix instructions in flight
// (kWaitTries attempts at most, whatever `tries` is) and ends without a valid result.
// ---------------------------------------------------------------------------
// An attempt takes 20 ns or more, and the hardware may hold it for longer, so this
// many end after a third of a second at the earliest; waits for memory take
// microseconds.  Attempts are counted, not time: a kernel that is taken off the
// device for a while is not late when it comes back.
constexpr int kWaitTries = 1 << 24;
static __device__ int g_wait_expired;        // one of each source file that includes this

__device__ __forceinline__ void barrier_init(uint32_t bar, uint32_t count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" :: "r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void barrier_expect(uint32_t bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" :: "r"(bar), "r"(bytes) : "memory");
}
// `bar` is a barrier of any block of the cluster.
__device__ __forceinline__ void barrier_arrive(uint32_t bar)
{
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" :: "r"(bar) : "memory");
}
__device__ __forceinline__ bool barrier_try(uint32_t bar, uint32_t parity)
{
    uint32_t done;
    asm volatile("{\n\t.reg .pred p;\n\t"
                 "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
                 "selp.u32 %0, 1, 0, p;\n\t}" : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    return done != 0;
}
__device__ __forceinline__ bool barrier_wait(uint32_t bar, uint32_t parity, int tries)
{
    for (int left = tries; left > 0; --left)
        if (barrier_try(bar, parity)) return true;
    atomicExch(&g_wait_expired, 1);
    return false;
}

__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 :: "r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}

// A kernel launched as a programmatic dependent may start before the kernel in
// front of it in the stream is done; wait_for_primary() returns once that one is
// complete and its writes are visible.  launch_dependents() lets it start.
__device__ __forceinline__ void wait_for_primary() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void launch_dependents() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// Reads and clears this source file's flag, after the work on `stream`.
static inline cudaError_t take_expired(cudaStream_t stream, int *expired)
{
    const int none = 0;
    cudaError_t e = cudaMemcpyFromSymbolAsync(expired, g_wait_expired, sizeof *expired, 0, cudaMemcpyDeviceToHost, stream);
    if (e == cudaSuccess) e = cudaStreamSynchronize(stream);
    if (e == cudaSuccess && *expired) e = cudaMemcpyToSymbolAsync(g_wait_expired, &none, sizeof none, 0, cudaMemcpyHostToDevice, stream);
    if (e == cudaSuccess) e = cudaStreamSynchronize(stream);
    return e;
}

}  // namespace star
