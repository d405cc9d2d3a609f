// Instructions of the microscaled linear layer beside those of sm100.cuh: block-scaled MMAs, untiled
// copies, wide reads of another CTA's shared memory.
#pragma once

#include "sm100.cuh"

namespace mpq {
namespace sm100 {

// ---- block-scaled MMA (kind::mxf4) -------------------------------------------------------------
// D[tmem] (+)= (A x scales)[smem] * (B x scales)[smem]^T for E2M1 operands, 64 elements of K, an E8M0
// scale for each 32 of them, in tensor memory at sfa and sfb; issued by one thread.
__device__ __forceinline__ void mma_mxf4(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc,
                                         uint32_t idesc, uint32_t sfa, uint32_t sfb,
                                         uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], "
        "p;\n\t}" ::"r"(d_tmem),
        "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate)
        : "memory");
}

// The CTA-pair form, as mma_f16_pair's: A is M = 256 rows, 128 in each CTA; B is N rows, N/2 in each; each
// CTA's tensor memory holds the scales of its own rows of A at sfa and of all rows of B at sfb.
__device__ __forceinline__ void mma_mxf4_pair(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc,
                                              uint32_t idesc, uint32_t sfa, uint32_t sfb,
                                              uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], "
        "p;\n\t}" ::"r"(d_tmem),
        "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate)
        : "memory");
}

// Instruction descriptor, kind::mxf4: A and B E2M1, E8M0 scales, both K-major; the scales of this
// K = 64 are bytes sf, sf + 1 (sf 0 or 2) of the 4-byte words in tensor memory.
__host__ __device__ constexpr uint32_t idesc_mxf4(int M, int N, int sf)
{
    return ((uint32_t)sf << 4)            // B's scale bytes
           | (1u << 7)                    // A format: E2M1
           | (1u << 10)                   // B format: E2M1
           | ((uint32_t)(N >> 3) << 17)   // N / 8
           | (1u << 23)                   // scales: E8M0
           | ((uint32_t)(M >> 4) << 24)   // M / 16
           | ((uint32_t)sf << 29);        // A's scale bytes
}

// `bytes` (a multiple of 16) of global memory into shared memory at dst, both 16-byte aligned,
// counted on `bar`.
__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, uint32_t bytes,
                                          uint64_t *bar)
{
    asm volatile(
        "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
        ::"r"(dst), "l"(__cvta_generic_to_global(src)), "r"(bytes), "r"(smem_u32(bar))
        : "memory");
}

// ---- another CTA's shared memory ---------------------------------------------------------------
__device__ __forceinline__ float4 ld_dsmem_f32x4(const float *local, uint32_t rank)
{
    uint32_t remote;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(smem_u32(local)),
                 "r"(rank));
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                 : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(remote) : "memory");
    return v;
}

}  // namespace sm100
}  // namespace mpq
