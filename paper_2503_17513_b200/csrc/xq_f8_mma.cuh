// tcgen05 pieces of the block-scaled E4M3 products (kind::mxf8f6f4): descriptors, scale copies, the instruction itself.
#pragma once

#include "xq_ptx.cuh"

namespace xqf8 {

// Instruction descriptor: E4M3 operands (format 0 at bits 7-9 and 10-12), both K-major; N >> 3 at bits 17-22; E8M0 scales
// (bit 23); M >> 4 at bits 24-28; the byte of each scale word that the instruction uses at bits 4-5 (B) and 29-30 (A).  One
// instruction covers 32 codes and has one scale per row of either operand: the four instructions of a 128-code block name the
// same byte, the four blocks of a scale word name bytes 0 to 3.
__device__ __forceinline__ uint32_t idesc(int m, int n, uint32_t byte) {
  return ((uint32_t)(n >> 3) << 17) | (1u << 23) | ((uint32_t)(m >> 4) << 24) | (byte << 4) | (byte << 29);
}
// Scale words in shared memory: 32 rows of 16 bytes (the words of rows r, r + 32, r + 64, r + 96), no swizzle, 8-row groups 128
// bytes apart; tcgen05.cp broadcasts the block to the four lane quarters of tensor memory (four columns).
__device__ __forceinline__ uint64_t sf_desc(uint32_t smem_addr) {
  return (uint64_t)((smem_addr & 0x3FFFFu) >> 4) | ((uint64_t)(128 >> 4) << 32) | (1ull << 46);
}
template <int CG>
__device__ __forceinline__ void sf_copy(uint32_t taddr, uint64_t sdesc) {
  if (CG == 1)
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(sdesc) : "memory");
  else
    asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(sdesc) : "memory");
}
template <int CG>
__device__ __forceinline__ void mma(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t id, uint32_t accumulate, uint32_t sfa_tmem,
                                    uint32_t sfb_tmem) {
  if (CG == 1)
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.block32 [%0], %1, %2, %3, [%5], [%6], p;\n\t}" ::"r"(d_tmem),
        "l"(adesc), "l"(bdesc), "r"(id), "r"(accumulate), "r"(sfa_tmem), "r"(sfb_tmem)
        : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.block32 [%0], %1, %2, %3, [%5], [%6], p;\n\t}" ::"r"(d_tmem),
        "l"(adesc), "l"(bdesc), "r"(id), "r"(accumulate), "r"(sfa_tmem), "r"(sfb_tmem)
        : "memory");
}

// One thread of a converged warp (the same one each time).  The loops that feed the tensor core run in such a thread from
// beginning to end: branched on inside the loop, or picked by lane number, the operands of every tcgen05 instruction are
// moved to uniform registers by code that provides for 32 threads, which costs more issue time than the MMAs take.
__device__ __forceinline__ bool elect_one() {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "elect.sync _|p, 0xffffffff;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok));
  return ok != 0;
}

// ---- thread-block clusters ---------------------------------------------------------------------------
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }
__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
// address of the same shared-memory location in CTA `rank` of the cluster
__device__ __forceinline__ uint32_t map_to(uint32_t smem_addr, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem_addr), "r"(rank));
  return r;
}
__device__ __forceinline__ void st_cluster(uint32_t addr, uint4 v) {
  asm volatile("st.shared::cluster.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

}  // namespace xqf8
