// tc_pair.cuh -- two-CTA tcgen05 (cta_group::2): loads, products and tensor memory of a CTA pair.
#pragma once

#include "tc_common.cuh"

namespace resbm {
namespace tc {

// ---- CTA pairs (cta_group::2): the two CTAs of a cluster of 2 work on one 256-row tile -------------
// tma_load_2d whose bytes complete on an mbarrier of either CTA of the pair (`bar` from map_shared)
__device__ __forceinline__ void tma_load_2d_pair(uint32_t dst, const CUtensorMap *m, int32_t x, int32_t y, uint32_t bar)
{
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2"
        " [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(m)), "r"(x), "r"(y), "r"(bar)
        : "memory");
}

// D (+)= A * B over both CTAs, issued by one thread of the even CTA: A's rows 0..127 and the first half
// of B's columns from its own shared memory, the rest from the odd CTA's (the same offsets); each CTA's
// TMEM receives its own 128 rows of D.
__device__ __forceinline__ void mma_bf16_pair(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc,
                                              bool accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
        "l"(a_desc), "l"(b_desc), "r"(idesc), "r"((uint32_t)accumulate)
        : "memory");
}

// Arrive on the mbarrier at the same offset in the CTAs of `mask` (3: both, 1: the even one) when every
// pair MMA issued so far has completed.
__device__ __forceinline__ void mma_commit_pair(uint32_t bar, uint16_t mask = 3)
{
    asm volatile(
        "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar),
        "h"(mask)
        : "memory");
}

// tmem_alloc / tmem_dealloc of a pair: executed by one warp of each of the two CTAs
__device__ __forceinline__ void tmem_alloc_pair(uint32_t dst, uint32_t ncols)
{
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(dst), "r"(ncols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_dealloc_pair(uint32_t taddr, uint32_t ncols)
{
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(taddr), "r"(ncols) : "memory");
}

}  // namespace tc
}  // namespace resbm
