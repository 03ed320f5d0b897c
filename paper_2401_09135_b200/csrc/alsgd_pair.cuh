// Instructions for two blocks of a cluster that work on one tile: copies that report to the first block's barriers, matrix
// products over both blocks' shared and tensor memory.  One function per instruction; what one block does alone is in
// alsgd_tc.cuh.
#pragma once
#include "alsgd_tc.cuh"

namespace alsgd_tc {

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
// The same place in the shared memory of the cluster's block `rank`.
__device__ __forceinline__ uint32_t at_rank(uint32_t addr, uint32_t rank) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// A wait of one of two blocks.  What it waits for in vain the other block works with too: the first issues the products over both
// blocks' shared memory, and either copies half of an operand.  So the other block is marked as well, and first: whoever sees this
// block's mark may go on to hand over a tile.
__device__ __forceinline__ void wait_pair(uint32_t bar, uint32_t parity, volatile uint32_t* dead, uint32_t code, uint32_t tries = kWaitTries) {
    wait(bar, parity, dead, code, tries, [dead] {
        asm volatile("st.relaxed.cluster.shared::cluster.u32 [%0], %1;" ::"r"(at_rank(smem_u32(const_cast<const uint32_t*>(dead)), cluster_rank() ^ 1)), "r"(1) : "memory");
        asm volatile("fence.acq_rel.cluster;" ::: "memory");
    });
}
// `bar` as at_rank gives it.  What it announces is tensor memory that has been read (the reads have completed, a
// tc_fence_before behind them): ordering wider than the block's own would wait for every store in flight, most of a microsecond.
__device__ __forceinline__ void bar_arrive_cluster(uint32_t bar, uint32_t times) {
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0], %1;" ::"r"(bar), "r"(times) : "memory");
}
__device__ __forceinline__ void tma_load2_pair(uint32_t dst, const CUtensorMap* m, uint32_t bar, int x, int y) {
    asm volatile(
        "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
        ::"r"(dst), "l"(m), "r"(bar), "r"(x), "r"(y) : "memory");
}
__device__ __forceinline__ void tma_load3_pair(uint32_t dst, const CUtensorMap* m, uint32_t bar, int x, int y, int z) {
    asm volatile(
        "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
        ::"r"(dst), "l"(m), "r"(bar), "r"(x), "r"(y), "r"(z) : "memory");
}
// Every store of the thread has been written.
__device__ __forceinline__ void tma_store_wait() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }

__device__ __forceinline__ void tmem_alloc_pair(uint32_t smem_dst, uint32_t columns) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_dst), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
}
__device__ __forceinline__ void tmem_free_pair(uint32_t addr, uint32_t columns) {
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(columns));
}
// bf16 x bf16 -> fp32, M = 256: 128 rows in either block, half of the columns of B from either block.
__host__ __device__ constexpr uint32_t mma_desc_pair(uint32_t n, bool a_m_major, bool b_n_major) {
    return (1u << 4) | (1u << 7) | (1u << 10) | ((a_m_major ? 1u : 0u) << 15) | ((b_n_major ? 1u : 0u) << 16) | ((n >> 3) << 17) |
           ((256u >> 4) << 24);
}
// Shared-memory operands without a swizzle, in groups of 8 x 16 bytes, each 128 bytes in a row: 8 rows of the operand with 8
// of K each, or 8 of K with 8 rows each (mma_desc_pair's a_m_major).  Bytes to the next 8 of K, to the next 8 rows.
__device__ __forceinline__ uint64_t desc_plain(uint32_t addr, uint32_t k_step, uint32_t row_step) {
    return (uint64_t)((addr >> 4) & 0x3FFF) | ((uint64_t)(k_step >> 4) << 16) | ((uint64_t)(row_step >> 4) << 32) | (1ull << 46);
}
// D (+)= A B; issued by one thread of the first block.
__device__ __forceinline__ void mma_ss_pair(uint32_t d, uint64_t a, uint64_t b, uint32_t desc, bool accumulate) {
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}\n"
        ::"r"(d), "l"(a), "l"(b), "r"(desc), "r"((uint32_t)accumulate) : "memory");
}
// Arrives on both blocks' barriers at this place when every product issued so far by this thread has completed.
__device__ __forceinline__ void mma_commit_pair(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                 ::"r"(bar), "h"((uint16_t)3) : "memory");
}

}  // namespace alsgd_tc
