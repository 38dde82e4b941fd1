// One or two blocks (a cluster, kPair) that work on a tile of a matrix product as one: tcgen05 instructions over both blocks' tensor memory
// and shared memory are issued by the first.
#pragma once
#include "eoq_epilogue.cuh"

namespace eoq {

// the barrier at the same place of every block receives one arrival when the MMAs issued so far are done
template <bool kPair>
__device__ __forceinline__ void commit_both(uint32_t bar, uint32_t leader)
{
    if constexpr (kPair)
        asm volatile(
            "{\n\t.reg .pred q;\n\t"
            "setp.ne.b32 q, %1, 0;\n\t"
            "@q tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %2;\n\t}"
            ::"r"(bar), "r"(leader), "h"((uint16_t)3) : "memory");
    else
        ptx::mma_commit(bar, leader);
}
// An arrival at the first block's barrier, in the default scope: whatever it announces lies in this block's own SM, where this SM's half of the MMA
// reads or writes it, and is done by then.  Operands (full_bar) are written to shared memory and fenced towards the asynchronous proxy; tensor memory
// (moved_bar) has been read and written, both waited for, with the fence of tcgen05 in front of the arrival and behind the first block's wait.  No data passes
// between the blocks' threads themselves.  In the scope of the cluster, which waits for more than that, the weight gradient from 8-bit inputs took 288 us for the operands (269 with
// one warp passing a barrier of the block on) and 147 for tensor memory, instead of 135: 1024 to 4096 channels, 16,384 rows.
template <bool kPair>
__device__ __forceinline__ void arrive_first(uint32_t bar)
{
    if constexpr (kPair)
        asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(ptx::cluster_addr(bar, 0)) : "memory");
    else
        ptx::mbar_arrive(bar);
}
// wait_bar for a barrier that threads of both blocks arrive at, in the scope of the cluster
template <bool kPair>
__device__ __forceinline__ bool wait_both(uint32_t bar, uint32_t parity, const RoleCtx &c)
{
    if constexpr (!kPair) {
        return wait_bar(bar, parity, c);
    } else {
        for (uint32_t i = 0; i < kSpinLimit; ++i) {
            uint32_t done;
            asm volatile(
                "{\n\t.reg .pred p;\n\t"
                "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
                "selp.u32 %0, 1, 0, p;\n\t}"
                : "=r"(done)
                : "r"(bar), "r"(parity)
                : "memory");
            if (done) return true;
            if (*c.abort_flag) return false;
        }
        *c.abort_flag = 1u;
        atomicOr(&c.dev->status, EOQ_DEV_TIMEOUT);
        return false;
    }
}
template <bool kPair>
__device__ __forceinline__ void tmem_take(uint32_t result, uint32_t columns)
{
    if constexpr (kPair) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(result), "r"(columns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
        ptx::tmem_alloc(result, columns);
        ptx::tmem_relinquish();
    }
}
template <bool kPair>
__device__ __forceinline__ void tmem_return(uint32_t base, uint32_t columns)
{
    if constexpr (kPair) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(base), "r"(columns) : "memory");
    else ptx::tmem_dealloc(base, columns);
}

}  // namespace eoq
