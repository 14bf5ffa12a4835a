// Loads into LDS that the compiler does not see, for rings whose stage is chosen at run time: of
// the builtins' loads it takes every LDS read to want the bytes, and waits for all of them.
// Callers wait with wait_vmem, for loads that may be in flight at the end of the kernel too.
// They write no register.  A vector instruction that wrote one of the scalar operands has to be
// five wait states behind, which the compiler does not see to either: hence the s_nop.
#pragma once

#include "hip_common.h"

#include <type_traits>

namespace pdec {

// A buffer's first address and the bytes from there on; reads behind them bring zeros.
struct DmaBuffer {
  u32x4 words;
};
__device__ __forceinline__ DmaBuffer dma_buffer(const void* base, uint32_t bytes) {
  const uint64_t b = (uint64_t)base;
  return {u32x4{(uint32_t)b, (uint32_t)(b >> 32) & 0xFFFFu, bytes, 0x00020000u}};
}
// Sixteen bytes a lane, from voff + soff + FROM, lane i's to lds + TO + 16 i.  (The instruction's
// own offset counts for both places.)  ONCE: for bytes that no one else reads soon.
template <int FROM, int TO, bool ONCE = false>
__device__ __forceinline__ void dma16_unseen(const DmaBuffer& src, int voff, int soff,
                                             uint32_t lds) {
  static_assert(FROM >= 0 && FROM < 4096, "the instruction's offset");
  if constexpr (ONCE)
    asm volatile(
        "s_add_u32 m0, %3, %4\n\ts_nop 4\n\tbuffer_load_dwordx4 %0, %1, %2 offen offset:%5 nt lds" ::
            "v"(voff),
        "s"(src.words), "s"(soff), "s"(lds), "n"(TO - FROM), "n"(FROM)
        : "memory", "m0", "scc");
  else asm volatile(
      "s_add_u32 m0, %3, %4\n\ts_nop 4\n\tbuffer_load_dwordx4 %0, %1, %2 offen offset:%5 lds" ::"v"(
          voff),
      "s"(src.words), "s"(soff), "s"(lds), "n"(TO - FROM), "n"(FROM)
      : "memory", "m0", "scc");
}
// f(0) to f(N - 1), each a constant of its own type.
template <int N, typename F>
__device__ __forceinline__ void each(F&& f) {
  if constexpr (N > 0) {
    each<N - 1>(f);
    f(std::integral_constant<int, N - 1>{});
  }
}
// Four bytes per active lane, lane i's at lds + 4 i.
__device__ __forceinline__ void dma4_unseen(const DmaBuffer& src, int voff, uint32_t lds) {
  asm volatile(
      "s_mov_b32 m0, %2\n\ts_nop 4\n\tbuffer_load_dword %0, %1, 0 offen lds" ::"v"(voff),
      "s"(src.words), "s"(lds)
      : "memory", "m0");
}

}  // namespace pdec
