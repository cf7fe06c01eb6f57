// What the kernels that use the tensor cores share: mbarriers with bounded waits, TMA loads, tcgen05 descriptors,
// instructions and tensor-memory reads, and the host side's tensor maps.
#pragma once

#include "lgc_internal.cuh"

namespace lgc {

constexpr long long kWaitCycles = 2000000000ll;   // a wait on an mbarrier gives up after about a second

__device__ __forceinline__ uint32_t smem_addr(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_init_fence() { asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory"); }
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t bar)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
// Polls the barrier; gives up when the limit is reached or another role has given up (then *failed is set).
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, volatile int *failed)
{
    long long begin = 0;
    for (;;) {
        uint32_t done;
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(done)
            : "r"(bar), "r"(parity)
            : "memory");
        if (done) return true;
        const long long now = clock64();
        if (begin == 0) begin = now;
        if (*failed) return false;
        if (now - begin > kWaitCycles) break;
    }
    *failed = 1;
    return false;
}
// After a wait that ran out: copies of this CTA may still be on their way into its shared memory.  Gives them a millisecond
// (a copy takes microseconds) before the CTA ends.
__device__ __forceinline__ void let_copies_land(volatile int *failed)
{
    if (!*failed) return;
    for (const long long begin = clock64(); clock64() - begin < kWaitCycles / 1000;) {}
}

// bar_wait for a whole warp that stays together: every lane polls, and the result is the same for all.  The warps that
// issue tensor-core work run this way: their descriptors and addresses then are uniform values, which the instructions
// want; from a branch that one thread takes alone each of them costs a move (0.2 us per stage of four MMAs).
__device__ __forceinline__ bool bar_wait_together(uint32_t bar, uint32_t parity, volatile int *failed)
{
    long long begin = 0;
    for (;;) {
        uint32_t done;
        asm volatile(
            "{\n\t.reg .pred p, q;\n\t.reg .u32 n;\n\t"
            "mov.u32 n, 0;\n\t"
            "POLL:\n\t"
            "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
            "@p bra DONE;\n\t"
            "add.u32 n, n, 1;\n\t"
            "setp.lt.u32 q, n, 256;\n\t"
            "@q bra POLL;\n\t"
            "DONE:\n\t"
            "selp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(done)
            : "r"(bar), "r"(parity)
            : "memory");
        if (__all_sync(0xffffffffu, done)) return true;
        const long long now = clock64();
        if (begin == 0) begin = now;
        if (__any_sync(0xffffffffu, *failed || now - begin > kWaitCycles)) break;
    }
    *failed = 1;
    return false;
}
// One lane of a warp that is together, always the same.
__device__ __forceinline__ bool elect_one()
{
    uint32_t e;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(e));
    return e != 0;
}

// ---- pairs of CTAs (clusters of two) ---------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// The address, in CTA `rank` of the cluster, of what lies at `addr` in this one.
__device__ __forceinline__ uint32_t cluster_addr(uint32_t addr, uint32_t rank)
{
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
// What the arrival publishes is this CTA's own shared memory and tensor memory, for the tensor cores: CTA scope is enough
// (after async_proxy_fence or tc_fence_before).  Cluster scope would make every arrival drain the thread's writes and every
// wait drop the L1 cache: 0.4 us per stage of the weight gradient.
__device__ __forceinline__ void bar_arrive_cluster(uint32_t cluster_bar)
{
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(cluster_bar) : "memory");
}
// A TMA load into this CTA's shared memory that completes at a barrier of either CTA of the pair (a cluster address).
__device__ __forceinline__ void tma_load_pair(uint32_t dst, const CUtensorMap *map, uint32_t cluster_bar, int c0, int c1)
{
    asm volatile(
        "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
        ::"r"(dst), "l"(map), "r"(cluster_bar), "r"(c0), "r"(c1)
        : "memory");
}
// tcgen05 for the pair: tensor memory is allocated in both CTAs, one thread of CTA 0 issues, and completion arrives at the
// same barrier of both.
__device__ __forceinline__ void tc_alloc_pair(uint32_t *where, uint32_t cols)
{
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(where)), "r"(cols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tc_free_pair(uint32_t tmem, uint32_t cols)
{
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(cols) : "memory");
}
__device__ __forceinline__ void tc_commit_pair(uint32_t bar)
{
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((uint16_t)3)
                 : "memory");
}

// Shared memory that threads have written becomes visible to the tensor cores and the TMA.
__device__ __forceinline__ void async_proxy_fence() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// `bytes` contiguous bytes: a multiple of 16, from and to 16-byte boundaries
__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar)
                 : "memory");
}
// Four bytes, asynchronously, by this thread; with `bytes` below four only those are read and the rest becomes zero.
__device__ __forceinline__ void word_load(uint32_t dst, const void *src, uint32_t bytes = 4)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap *map, uint32_t bar, int c0, int c1)
{
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
        ::"r"(dst), "l"(map), "r"(bar), "r"(c0), "r"(c1)
        : "memory");
}

// Shared-memory matrix descriptors, 128-byte swizzle.  K-major: rows of 128 bytes along K, groups of eight rows 1024
// bytes apart.  MN-major: rows of 128 bytes along M or N, one per k; groups of eight k 1024 bytes apart, the next 128
// bytes of M or N `piece` bytes on.
__device__ __forceinline__ uint64_t tc_desc(uint32_t addr, uint32_t piece)
{
    return (uint64_t)((addr & 0x3ffffu) >> 4) | (uint64_t)(piece >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 |
           (uint64_t)2 << 61;
}
__device__ __forceinline__ uint64_t tc_desc_k(uint32_t addr) { return tc_desc(addr, 16); }
// No swizzle, for tcgen05.cp of 32 rows of 16 bytes: groups of eight rows 128 bytes apart.
__device__ __forceinline__ uint64_t tc_desc_copy(uint32_t addr)
{
    return (uint64_t)((addr & 0x3ffffu) >> 4) | (uint64_t)(16 >> 4) << 16 | (uint64_t)(128 >> 4) << 32 | (uint64_t)1 << 46;
}

__device__ __forceinline__ void tc_alloc(uint32_t *where, uint32_t cols)
{
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(where)), "r"(cols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tc_free(uint32_t tmem, uint32_t cols)
{
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(cols) : "memory");
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// Makes the mbarrier complete once every tcgen05 operation issued so far by this thread has finished.
__device__ __forceinline__ void tc_commit(uint32_t bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// 32 columns of this warp's quarter of tensor memory (row = lane); complete after tc_read_wait.
__device__ __forceinline__ void tc_read32(uint32_t taddr, uint32_t (&r)[32])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
          "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
          "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tc_read_wait(uint32_t (&r)[32])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < 32; ++i) asm volatile("" : "+r"(r[i]));      // the values are used after the wait, not before
}
// 16 columns, complete.
__device__ __forceinline__ void tc_read16(uint32_t taddr, uint32_t (&r)[16])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr)
        : "memory");
}

// ---- host: tensor maps ------------------------------------------------------------------------------------------
// A matrix of `rows` rows of `cols` elements, `ld` elements apart; boxes of box_cols x box_rows.  What lies outside reads as zero.
cudaError_t make_matrix_map(CUtensorMap *m, CUtensorMapDataType type, int elem_bytes, const void *base, int64_t cols, int64_t rows,
                            int64_t ld, int box_cols, int box_rows, CUtensorMapSwizzle swizzle);

}  // namespace lgc
