// PTX wrappers of the tensor-core kernels: mbarriers with bounded waits, TMA, tensor memory, commits, shared-memory descriptors.
#pragma once

#include <cuda.h>

#include "sat_internal.h"

#define TC_WAIT_LIMIT (1u << 22)

__device__ __forceinline__ uint32_t smem_u32(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void mbar_init(uint64_t *bar, uint32_t count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(bar)), "r"(count));
}
__device__ __forceinline__ void mbar_expect_tx(uint64_t *bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_u32(bar)), "r"(bytes) : "memory");
}
// bounded wait: returns false (and raises *dead) when the limit is hit or another thread already gave up.
// SLEEP_NS > 0 backs off between polls: a spinning warp otherwise takes issue slots from the warps doing the work
// (the epilogue shares its schedulers with the waiting converter warps).
template <int SLEEP_NS = 0>
__device__ __forceinline__ bool mbar_wait(uint64_t *bar, uint32_t parity, volatile int *dead, int *status)
{
    const uint32_t addr = smem_u32(bar);
    for (uint32_t it = 0; it < TC_WAIT_LIMIT; ++it) {
        uint32_t ok;
        asm volatile(
            "{\n\t"
            ".reg .pred p;\n\t"
            "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t"
            "}"
            : "=r"(ok)
            : "r"(addr), "r"(parity)
            : "memory");
        if (ok) return true;
        if (*dead) return false;
        if (SLEEP_NS > 0) __nanosleep(SLEEP_NS);
    }
    *dead = 1;
    atomicOr(status, 1);
    return false;
}
// For a thread that gave up: the loads that are still on their way into a ring of `slots` stages land before the shared memory goes to somebody else.  `issued`
// of them went to the slots in turn, each a phase of its slot's barrier; 100 ns at least a look, 2 ms at least a slot.
__device__ __forceinline__ void mbar_settle(uint64_t *bars, uint32_t slots, uint32_t issued)
{
    for (uint32_t i = issued > slots ? issued - slots : 0u; i < issued; ++i)
        for (uint32_t it = 0; it < 20000u; ++it) {
            uint32_t ok;
            asm volatile(
                "{\n\t"
                ".reg .pred p;\n\t"
                "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
                "selp.u32 %0, 1, 0, p;\n\t"
                "}"
                : "=r"(ok)
                : "r"(smem_u32(bars + i % slots)), "r"((i / slots) & 1u)
                : "memory");
            if (ok) break;
            __nanosleep(100);
        }
}
// whole-warp wait: lane 0 polls, then every lane observes the completed phase itself (one immediate try_wait each), so
// that a waiting warp issues one poll per round instead of 32
__device__ __forceinline__ bool mbar_wait_warp(uint64_t *bar, uint32_t parity, volatile int *dead, int *status, int lane)
{
    int ok = 1;
    if (lane == 0) ok = mbar_wait<64>(bar, parity, dead, status) ? 1 : 0;
    ok = __shfl_sync(0xffffffffu, ok, 0);
    if (!ok) return false;
    return mbar_wait(bar, parity, dead, status);
}
// every lane waits; the result is that of the whole warp
__device__ __forceinline__ bool mbar_wait_all(uint64_t *bar, uint32_t parity, volatile int *dead, int *status)
{
    return __all_sync(0xffffffffu, mbar_wait(bar, parity, dead, status));
}
__device__ __forceinline__ void tma_prefetch(const CUtensorMap *map) { asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory"); }
__device__ __forceinline__ void tma_load_2d(void *smem_dst, const CUtensorMap *map, uint64_t *bar, int32_t x, int32_t y)
{
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];" ::"r"(
                     smem_u32(smem_dst)),
                 "l"((uint64_t)map), "r"(smem_u32(bar)), "r"(x), "r"(y)
                 : "memory");
}
__device__ __forceinline__ void tma_store_2d(const CUtensorMap *map, const void *smem_src, int32_t x, int32_t y)
{
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];" ::"l"((uint64_t)map), "r"(smem_u32(smem_src)),
                 "r"(x), "r"(y)
                 : "memory");
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}
// waits until at most `N` of this thread's bulk stores still read their shared-memory source
template <int N>
__device__ __forceinline__ void tma_store_wait_read()
{
    asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ void tma_store_wait_all() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
__device__ __forceinline__ bool elect_one()
{
    uint32_t p;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
    return p != 0;
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// One warp; GROUP = 2: one warp of each CTA of the pair, which get the same columns
template <int GROUP>
__device__ __forceinline__ void tc_alloc(uint32_t *base, uint32_t cols)
{
    if (GROUP == 2) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(base)), "r"(cols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(base)), "r"(cols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
}
template <int GROUP>
__device__ __forceinline__ void tc_dealloc(uint32_t base, uint32_t cols)
{
    if (GROUP == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(base), "r"(cols) : "memory");
    else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(base), "r"(cols) : "memory");
}
__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
}
// arrives on the barrier once this thread's MMAs so far have completed; GROUP = 2: on that of both CTAs of the pair
template <int GROUP>
__device__ __forceinline__ void tc_commit(uint64_t *bar)
{
    if (GROUP == 2)
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(smem_u32(bar)),
                     "h"((uint16_t)3)
                     : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
// D (+)= A B.  USE_A: what becomes of the A tile in the tensor core's operand collector -- 1: it stays, 2: it is taken from there for
// the last time.  (The two products with A hi read it from shared memory once: 1.3 % of a 179250 x 512 x 512 contraction.)
#define TC_MMA_ASM(G, KIND, COLLECTOR)                                                                 \
    asm volatile(                                                                                      \
        "{\n\t"                                                                                        \
        ".reg .pred p;\n\t"                                                                            \
        "setp.ne.b32 p, %4, 0;\n\t"                                                                    \
        "tcgen05.mma.cta_group::" G ".kind::" KIND COLLECTOR " [%0], %1, %2, %3, p;\n\t"                   \
        "}" ::"r"(tmem_d),                                                                             \
        "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)                                            \
        : "memory")
template <int USE_A, int GROUP>
__device__ __forceinline__ void tc_mma(uint32_t tmem_d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate)
{
    if (GROUP == 2) {
        if (USE_A == 1) TC_MMA_ASM("2", "tf32", ".collector::a::fill");
        else if (USE_A == 2) TC_MMA_ASM("2", "tf32", ".collector::a::lastuse");
        else TC_MMA_ASM("2", "tf32", "");
    } else {
        if (USE_A == 1) TC_MMA_ASM("1", "tf32", ".collector::a::fill");
        else if (USE_A == 2) TC_MMA_ASM("1", "tf32", ".collector::a::lastuse");
        else TC_MMA_ASM("1", "tf32", "");
    }
}
// the same with 16-bit operands; USE_A = 3: it is taken from there and stays
template <int USE_A, int GROUP>
__device__ __forceinline__ void tc_mma_f16(uint32_t tmem_d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate)
{
    if (GROUP == 2) {
        if (USE_A == 1) TC_MMA_ASM("2", "f16", ".collector::a::fill");
        else if (USE_A == 2) TC_MMA_ASM("2", "f16", ".collector::a::lastuse");
        else if (USE_A == 3) TC_MMA_ASM("2", "f16", ".collector::a::use");
        else TC_MMA_ASM("2", "f16", "");
    } else {
        if (USE_A == 1) TC_MMA_ASM("1", "f16", ".collector::a::fill");
        else if (USE_A == 2) TC_MMA_ASM("1", "f16", ".collector::a::lastuse");
        else if (USE_A == 3) TC_MMA_ASM("1", "f16", ".collector::a::use");
        else TC_MMA_ASM("1", "f16", "");
    }
}
__device__ __forceinline__ void tc_ld32(uint32_t taddr, uint32_t *r)
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, "
        "%19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
          "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
          "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr)
        : "memory");
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}

// shared-memory matrix descriptor: start address, leading / stride byte offsets (16-byte units), sm_100 version, swizzle mode
__device__ __forceinline__ uint64_t make_desc(uint32_t saddr, uint32_t lbo_bytes, uint32_t sbo_bytes, uint32_t layout_type)
{
    uint64_t d = 0;
    d |= (uint64_t)((saddr >> 4) & 0x3FFFu);
    d |= (uint64_t)((lbo_bytes >> 4) & 0x3FFFu) << 16;
    d |= (uint64_t)((sbo_bytes >> 4) & 0x3FFFu) << 32;
    d |= (uint64_t)1 << 46;
    d |= (uint64_t)layout_type << 61;
    return d;
}
__device__ __forceinline__ void mbar_arrive(uint64_t *bar)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
}
// A warp's arrival on a barrier that the MMA issuer waits for.  CTAS = 1: every lane arrives.  2: lane 0 does, on the barrier at the same
// place in CTA 0 of the pair, without a scope, that is at CTA scope.  An assumption rests on that: that shared-memory writes in front of
// the proxy fence and TMEM reads in front of their wait are done for the pair's MMAs when the arrival is seen.  The memory model does not
// say so across two CTAs; it is the customary form of arriving at the other CTA of a pair, and
// tests/test_gpu_edges.py compares pair launches with single CTAs bit by bit.  (With .release.cluster the arrival also waits for
// everything else the SM has in flight, 1.4 us: a 179250 x 512 x 512 contraction took 490 us instead of 370; waits that acquire at
// cluster scope, which would be half of it, cost 0.3-0.5 % of an epoch.)
template <int CTAS>
__device__ __forceinline__ void mbar_arrive_warp(uint64_t *bar, int lane)
{
    if (CTAS == 1) {
        mbar_arrive(bar);
        return;
    }
    __syncwarp();
    if (lane == 0)
        asm volatile(
            "{\n\t"
            ".reg .b32 a;\n\t"
            "mapa.shared::cluster.u32 a, %0, 0;\n\t"
            "mbarrier.arrive.shared::cluster.b64 _, [a];\n\t"
            "}" ::"r"(smem_u32(bar))
            : "memory");
}
// lane 0's arrival on the same barriers with single CTAs too
template <int CTAS>
__device__ __forceinline__ void mbar_arrive_lane0(uint64_t *bar, int lane)
{
    __syncwarp();
    if (CTAS == 2) mbar_arrive_warp<CTAS>(bar, lane);
    else if (lane == 0) mbar_arrive(bar);
}
// make generic-proxy shared-memory writes visible to the tensor-core (async) proxy
__device__ __forceinline__ void fence_async_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// 2-D tensor map: `inner` contiguous elements per row, `outer` rows `ld_bytes` apart (sat_gemm_tc.cu)
sat_status sat_tensor_map(sat_ctx *ctx, CUtensorMap *map, CUtensorMapDataType type, const void *base, int64_t inner, int64_t outer, int64_t ld_bytes,
                          int box_inner, int box_outer, CUtensorMapSwizzle swz);
