// Sums, extremes and scans over a wave of 64 lanes, all active, without LDS: DPP moves
// within the rows of 16 lanes and gfx950's cross-row swaps.  A step of __shfl is an LDS
// permute, whose latency a short kernel waits for a dozen times in a row.
#pragma once

#include "hip_common.h"

namespace pdec {

template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, CTRL, 0xf, 0xf, false);
}
template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
  return __uint_as_float(dpp<CTRL>(__float_as_uint(v)));
}
template <int CTRL>
__device__ __forceinline__ int dpp(int v) {
  return (int)dpp<CTRL>((uint32_t)v);
}
template <int CTRL>
__device__ __forceinline__ uint64_t dpp(uint64_t v) {
  return (uint64_t)dpp<CTRL>((uint32_t)(v >> 32)) << 32 | dpp<CTRL>((uint32_t)v);
}

// f over all lanes, the same in every lane: within a row by rotations of 8, 4, 2 and 1
// lanes, then over the rows (each swap of a value with itself leaves both operands).
__device__ __forceinline__ void swap_rows(uint32_t v, int which, uint32_t& a, uint32_t& b) {
  const auto r = which == 16 ? __builtin_amdgcn_permlane16_swap(v, v, false, false)
                             : __builtin_amdgcn_permlane32_swap(v, v, false, false);
  a = r[0];
  b = r[1];
}
template <typename T, typename F>
__device__ __forceinline__ T wave_all(T v, F&& f) {
  v = f(v, dpp<0x128>(v));
  v = f(v, dpp<0x124>(v));
  v = f(v, dpp<0x122>(v));
  v = f(v, dpp<0x121>(v));
#pragma unroll
  for (int which = 16; which <= 32; which += 16) {
    uint32_t a[2], b[2];
    if constexpr (sizeof(T) == 8) {
      swap_rows((uint32_t)v, which, a[0], b[0]);
      swap_rows((uint32_t)(v >> 32), which, a[1], b[1]);
      v = f((T)a[1] << 32 | a[0], (T)b[1] << 32 | b[0]);
    } else {
      swap_rows(__builtin_bit_cast(uint32_t, v), which, a[0], b[0]);
      v = f(__builtin_bit_cast(T, a[0]), __builtin_bit_cast(T, b[0]));
    }
  }
  return v;
}
template <typename T>
__device__ __forceinline__ T wave_add(T v) {
  return wave_all(v, [](T a, T b) { return a + b; });
}
__device__ __forceinline__ float wave_top(float v) {  // a NaN is passed over
  return wave_all(v, [](float a, float b) { return fmaxf(a, b); });
}

// Sum of the lanes up to and with this one, of int or uint64_t: shifts within the rows,
// then row ends added to the rows behind them.
template <int CTRL, int ROWS, typename T>
__device__ __forceinline__ T dpp_or_zero(T v) {
  if constexpr (sizeof(T) == 8) {
    const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)v, CTRL, ROWS, 0xf, false);
    const uint32_t hi =
        __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(v >> 32), CTRL, ROWS, 0xf, false);
    return (T)hi << 32 | lo;
  } else {
    return (T)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, false);
  }
}
template <typename T>
__device__ __forceinline__ T wave_prefix(T v) {
  v += dpp_or_zero<0x111, 0xf>(v);  // row_shr:1, 2, 4, 8
  v += dpp_or_zero<0x112, 0xf>(v);
  v += dpp_or_zero<0x114, 0xf>(v);
  v += dpp_or_zero<0x118, 0xf>(v);
  v += dpp_or_zero<0x142, 0xa>(v);  // row_bcast:15 to rows 1 and 3
  v += dpp_or_zero<0x143, 0xc>(v);  // row_bcast:31 to rows 2 and 3
  return v;
}
// A lane's value, the same lane in all of them.
__device__ __forceinline__ int lane_of(int v, int lane) { return __builtin_amdgcn_readlane(v, lane); }
__device__ __forceinline__ uint64_t lane_of(uint64_t v, int lane) {
  return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(v >> 32), lane) << 32 |
         (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, lane);
}

}  // namespace pdec
