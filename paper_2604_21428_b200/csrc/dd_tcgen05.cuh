// Tensor cores, tensor memory, the TMA engine and the bounded waits of the kernels that use them: the
// instructions behind the products of the learner's operators.
#pragma once

#include <cuda.h>

#include <cuda_bf16.h>

#include "dd_merge_tma.cuh"

namespace ddm {

constexpr unsigned kSpinLimit = 1u << 30;         // attempts and nanoseconds of a bounded wait
constexpr unsigned long long kWaitNs = 1000000000ull;
constexpr int kChunkBytes = 64 * 128;             // one TMA box: 64 rows of 64 bf16

// ---- tcgen05 ----------------------------------------------------------------------------------

__device__ __forceinline__ bool elect_one()
{
    unsigned p;
    asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(p));
    return p != 0;
}

__device__ __forceinline__ void tma_load_2d(unsigned dst, const CUtensorMap *map, int x, int y, unsigned bar)
{
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 :: "r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}

__device__ __forceinline__ void umma_bf16(unsigned d, unsigned long long a, unsigned long long b, unsigned idesc, unsigned accumulate)
{
    asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
                 " tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}"
                 :: "r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}

// Arrives on `bar` once every tcgen05.mma this thread has issued so far is complete.
__device__ __forceinline__ void umma_commit(unsigned bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" :: "r"(bar) : "memory");
}

// The same for a pair: products of both SMs, `bar` in every CTA of `mask`.
__device__ __forceinline__ void umma_commit_pair(unsigned bar, unsigned short mask)
{
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                 :: "r"(bar), "h"(mask) : "memory");
}

__device__ __forceinline__ void umma_bf16_pair(unsigned d, unsigned long long a, unsigned long long b, unsigned idesc, unsigned accumulate)
{
    asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
                 " tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}"
                 :: "r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}

// A copy into this CTA that reports to a barrier (a cluster address) of either CTA of the pair.
__device__ __forceinline__ void tma_load_2d_pair(unsigned dst, const CUtensorMap *map, int x, int y, unsigned bar)
{
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 :: "r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}

// This CTA's shared-memory address as the cluster address of the same place in CTA `rank`.
__device__ __forceinline__ unsigned cluster_addr(unsigned addr, unsigned rank)
{
    unsigned r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}

// Four floats at `addr` (a shared-memory address of this CTA) in the CTA of rank `rank`.
__device__ __forceinline__ float4 ld_cluster4(unsigned addr, unsigned rank)
{
    float4 x;
    asm volatile("{\n .reg .b32 r;\n mapa.shared::cluster.u32 r, %4, %5;\n ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [r];\n}"
                 : "=f"(x.x), "=f"(x.y), "=f"(x.z), "=f"(x.w) : "r"(addr), "r"(rank) : "memory");
    return x;
}

// Relaxed: what it reports is that tensor memory has been read into registers, which the wait on
// those loads has ensured.  A release would hold the warp until its stores to global memory are
// acknowledged: 2-5k cycles a tile.
__device__ __forceinline__ void mbar_arrive_cluster(unsigned bar)
{
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" :: "r"(bar) : "memory");
}

__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// The same without ordering memory, for the end of a kernel: a release would wait for the results to be
// acknowledged, which the end of the launch does anyway.
__device__ __forceinline__ void cluster_sync_relaxed()
{
    asm volatile("barrier.cluster.arrive.relaxed.aligned;\n barrier.cluster.wait.aligned;" ::: "memory");
}

__device__ __forceinline__ void tmem_ld32(unsigned addr, unsigned (&r)[32])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
        "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
          "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
          "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(addr));
}

__device__ __forceinline__ void tmem_ld16(unsigned addr, unsigned (&r)[16])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
                   "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(addr));
}

__device__ __forceinline__ void tmem_ld_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// Shared-memory operand descriptor, 128-byte swizzle.  Chunks are 64 rows of 128 bytes.
//   K contiguous: rows are M (N); groups of 8 rows follow every 1024 bytes, chunks continue them.
//   M (N) contiguous: rows are K, groups of 8 every 1024 bytes; the next 64 M (N) are one chunk on.
__device__ __forceinline__ unsigned long long umma_desc(unsigned addr, bool mn)
{
    const unsigned long long lead = mn ? kChunkBytes / 16 : 1, stride = 1024 / 16;
    return ((unsigned long long)(addr >> 4) & 0x3fff) | (lead << 16) | (stride << 32) | (1ull << 46) | (2ull << 61);
}

// Bounded wait of a pipeline role.  No suspend hint: with one (4 us) a role woke up to 3 us after its
// phase had completed.  The limit is on time, a second, looked at every 256 attempts.
__device__ __forceinline__ bool gemm_wait(unsigned bar, unsigned parity, volatile int *abort)
{
    unsigned long long start = 0;
    for (unsigned spins = 0; spins < kSpinLimit; ++spins) {
        unsigned ok;
        asm volatile("{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}"
                     : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
        if (ok) return true;
        if (*abort) return false;
        if ((spins & 255) == 255) {
            unsigned long long now;
            asm volatile("mov.u64 %0, %globaltimer;" : "=l"(now));
            if (!start) start = now;
            else if (now - start > kWaitNs) break;
        }
    }
    *abort = 1;
    return false;
}

__device__ __forceinline__ unsigned pack2(float lo, float hi)
{
    const __nv_bfloat162 b = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const unsigned *>(&b);
}

// 2^x to 2 ulp, 0 below the normal range.
__device__ __forceinline__ float exp2_fast(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

}  // namespace ddm
