// Copies from global memory straight into LDS and the waits for them, shared by
// the GEMM tiles and the paged attention.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace qm {

namespace qg {

// s_waitcnt vmcnt(N) with expcnt and lgkmcnt left free (gfx9 encoding:
// vmcnt[3:0] in bits 3:0 and vmcnt[5:4] in bits 15:14).
template <int N>
__device__ __forceinline__ void vm_wait() {
  static_assert(N >= 0 && N <= 63, "vmcnt is 6 bits");
  __builtin_amdgcn_s_waitcnt((N & 0xF) | ((N >> 4) << 14) | (0x7 << 4) | (0xF << 8));
}

// 16 bytes per lane from global memory straight into LDS: lane l of the
// wavefront writes lds_dst + 16 l (lds_dst is wavefront-uniform and goes
// to M0).  Issued as inline asm so that the compiler's wait-count tracking
// does not see it: with an LDS DMA pending, that tracking would wait for
// every outstanding load (vmcnt 0) before the next use of any loaded
// register.  The hardware still counts it in vmcnt; the kernel waits for it
// explicitly (vm_wait), and every later wait the compiler computes stays
// conservative.  The s_nop is the wait state gfx9 needs between a scalar write
// of M0 and an LDS DMA, which the assembler does not add inside inline asm:
// without it the DMA may take the previous M0 (1 KiB of a tile lands on the piece
// before).
__device__ __forceinline__ uint32_t lds_address(const void* p) {
  return static_cast<uint32_t>(reinterpret_cast<size_t>((const void __attribute__((address_space(3)))*)p));
}
template <bool NT = false>
__device__ __forceinline__ void lds_dma16(const void* src, const void* lds_dst) {
  if constexpr (NT)
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off nt" : : "v"(src), "s"(lds_address(lds_dst))
                 : "memory", "m0");
  else
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(src), "s"(lds_address(lds_dst))
                 : "memory", "m0");
}
// The same from a wavefront-uniform address and a byte offset per lane.
__device__ __forceinline__ void lds_dma16(const void* src, uint32_t offset, const void* lds_dst) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(offset), "s"(src),
               "s"(lds_address(lds_dst)) : "memory", "m0");
}
// 4 bytes per lane, lane l to lds_dst + 4 l.
template <bool NT = false>
__device__ __forceinline__ void lds_dma4(const void* src, const void* lds_dst) {
  if constexpr (NT)
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off nt" : : "v"(src), "s"(lds_address(lds_dst))
                 : "memory", "m0");
  else
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" : : "v"(src), "s"(lds_address(lds_dst))
                 : "memory", "m0");
}

}  // namespace qg

}  // namespace qm
