// Rows of a call that belong to sequences: what the appends and the reading of pages as rows
// share.  Row r is of the sequence b with row_start[b] <= r < row_start[b + 1].
#pragma once

#include "hip_common.h"

namespace pdec {

typedef uint16_t u16x4_any __attribute__((ext_vector_type(4), aligned(2)));

// Four consecutive elements at element alignment.
__device__ __forceinline__ f32x4 read4(const float* p) { return *(const f32x4_any*)p; }
__device__ __forceinline__ f32x4 read4(const uint16_t* p) {
  const u16x4_any v = *(const u16x4_any*)p;
  return f32x4{bf16_to_f32(v.x), bf16_to_f32(v.y), bf16_to_f32(v.z), bf16_to_f32(v.w)};
}
__device__ __forceinline__ float read1(const float* p) { return *p; }
__device__ __forceinline__ float read1(const uint16_t* p) { return bf16_to_f32(*p); }

// The smallest power of two s, 2^-100 to 2^100, with amax <= 448 s (448 = 1.75 * 2^8).
__device__ __forceinline__ float scale_for(float amax) {
  const uint32_t b = __float_as_uint(amax);
  const int e = (int)(b >> 23) - 127 - 8 + ((b & 0x7FFFFFu) > 0x600000u);
  return __uint_as_float((uint32_t)(min(max(amax > 0.f ? e : -100, -100), 100) + 127) << 23);
}
// One over a power of two of that range.
__device__ __forceinline__ float inverse_pow2(float s) {
  return __uint_as_float((254u << 23) - __float_as_uint(s));
}

// The sequence that holds row r, or -1, by every wave for itself: 64 sequences at a time,
// from where r lies if all have as many rows.  r is the same over the wave.
__device__ __forceinline__ int find_seq(const int32_t* row_start, int n_seqs, int n_rows, int r) {
  const int lane = threadIdx.x & 63, chunks = (n_seqs + 63) / 64;
  int c = (int)((int64_t)r * n_seqs / n_rows) / 64;
  for (int i = 0; i < chunks; ++i) {
    const int b = c * 64 + lane;
    const bool in = b < n_seqs && row_start[b] <= r && r < row_start[b + 1];
    const uint64_t hit = __ballot(in);
    if (hit) return c * 64 + __builtin_ctzll(hit);
    c = c + 1 < chunks ? c + 1 : 0;
  }
  return -1;
}

}  // namespace pdec
