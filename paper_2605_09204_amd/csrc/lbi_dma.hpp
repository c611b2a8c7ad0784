// Tiles that are loaded from memory straight into LDS (buffer_load_dwordx4 ... lds), shared by the
// products of Phase 1 and of the projections.
#ifndef LBI_DMA_HPP
#define LBI_DMA_HPP

#include "lbi_device.hpp"

namespace lbi {
namespace {

// LDS tile layout: 128 rows of 64 bf16 (eight 16-byte chunks), two rows per
// 256-byte line, chunk q of row R at line R / 2, slot ((R & 1) 8 + q) ^ (R / 2 & 7).
// The 16 lanes that a b128 access serves together then touch 16 distinct
// slots (all 64 banks) both when they read one chunk of 16 consecutive rows
// (an MFMA operand) and when they write the 8 chunks of 2 consecutive rows.
__device__ __forceinline__ int lds_off(int row, int q)
{
    return (row >> 1) * 128 + ((((row & 1) << 3) + q) ^ ((row >> 1) & 7)) * 8;
}

typedef int i4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ i4 dma_rsrc(const void *base, uint32_t bytes)
{
    // (the values are wave-uniform; the scalar registers an asm operand of
    // class "s" needs are made explicit)
    const uint64_t x = (uint64_t)(uintptr_t)base;
    i4 v;
    v[0] = __builtin_amdgcn_readfirstlane((int)(uint32_t)x);
    v[1] = __builtin_amdgcn_readfirstlane((int)((uint32_t)(x >> 32) & 0xFFFFu));
    v[2] = __builtin_amdgcn_readfirstlane((int)bytes);
    v[3] = kBufferWord3;
    return v;
}
// 16 bytes per lane from rs at voff + soff into LDS at lds + 16 lane; M0 (the
// LDS destination, one wait state after writing it) is saved and restored in
// the asm
__device__ __forceinline__ void dma_b128(uint32_t lds, i4 rs, int voff, int soff)
{
    uint32_t keep;
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\t"
                 "buffer_load_dwordx4 %2, %3, %4 offen lds\n\ts_mov_b32 m0, %0"
                 : "=&s"(keep)
                 : "s"(lds), "v"(voff), "s"(rs), "s"(soff)
                 : "memory");
}
// all of this wave's loads but the N most recent, and its LDS operations, done;
// then the workgroup barrier (the waits are the compiler's own, so it counts
// them when it places its LDS waits)
template <int N> __device__ __forceinline__ void dma_barrier()
{
    __builtin_amdgcn_s_waitcnt((N & 15) | (((N >> 4) & 3) << 14) | (7 << 4));
    __builtin_amdgcn_s_barrier();
}

}  // namespace
}  // namespace lbi

#endif  // LBI_DMA_HPP
