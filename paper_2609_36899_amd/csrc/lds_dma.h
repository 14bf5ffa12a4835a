// Loads into LDS that the compiler does not see, for rings whose stage is chosen at run time: of
// the builtins' loads it takes every LDS read to want the bytes, and waits for all of them.
// Callers wait with wait_vmem, for loads that may be in flight at the end of the kernel too.
// They write no register.  A vector instruction that wrote one of the scalar operands has to be
// five wait states behind, which the compiler does not see to either: hence the s_nop.
#pragma once

#include "hip_common.h"

namespace pdec {

// A buffer's first address and the bytes from there on; reads behind them bring zeros.
struct DmaBuffer {
  u32x4 words;
};
__device__ __forceinline__ DmaBuffer dma_buffer(const void* base, uint32_t bytes) {
  const uint64_t b = (uint64_t)base;
  return {u32x4{(uint32_t)b, (uint32_t)(b >> 32) & 0xFFFFu, bytes, 0x00020000u}};
}
__device__ __forceinline__ void dma16_unseen(const DmaBuffer& src, int voff, int soff,
                                             uint32_t lds) {
  asm volatile(
      "s_mov_b32 m0, %3\n\ts_nop 4\n\tbuffer_load_dwordx4 %0, %1, %2 offen lds" ::"v"(voff),
      "s"(src.words), "s"(soff), "s"(lds)
      : "memory", "m0");
}
// Four bytes per active lane, lane i's at lds + 4 i.
__device__ __forceinline__ void dma4_unseen(const DmaBuffer& src, int voff, uint32_t lds) {
  asm volatile(
      "s_mov_b32 m0, %2\n\ts_nop 4\n\tbuffer_load_dword %0, %1, 0 offen lds" ::"v"(voff),
      "s"(src.words), "s"(lds)
      : "memory", "m0");
}

}  // namespace pdec
