// What the kernels of the attention over latent pages share: units of work, and the first
// product's operands.
#pragma once

#include "hip_common.h"
#include "kernels.h"
#include "lds_dma.h"
#include "stretch.h"

namespace pdec {

constexpr int kRope = kLatentRope;
// A row's reference maximum moves only where its scores outgrow it by this many powers of
// two: the weights are then up to 2^16 instead of 1, no less exact, and the accumulators are
// rescaled a few times a row instead of at most tiles.  The sums of n keys overflow where values
// exceed 2^112 / n.
constexpr float kSlack = 16.f;

typedef short s16x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef int s32x2 __attribute__((ext_vector_type(2)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
#define PDEC_LDS __attribute__((address_space(3)))

__device__ __forceinline__ int clamp_len(const LatentAttnArgs& a, int b) {
  return min(max(a.lens[b], 0), a.max_len);
}
// Rows of unit u, its first row within the sequence, and the keys that any of them sees.
__device__ __forceinline__ int unit_row0(const LatentAttnArgs& a, int u) {
  return u % a.blocks_per_seq * a.block_rows;
}
__device__ __forceinline__ int unit_rows(const LatentAttnArgs& a, int row0) {
  return min(a.block_rows, a.n_q * a.n_heads - row0);
}
__device__ __forceinline__ int unit_keys(const LatentAttnArgs& a, int u) {
  const int row0 = unit_row0(a, u);
  const int j = (row0 + unit_rows(a, row0) - 1) / a.n_heads;  // its last token
  return max(clamp_len(a, u / a.blocks_per_seq) - a.n_q + j + 1, 0);
}
template <int TILE>
__device__ __forceinline__ int unit_tiles(const LatentAttnArgs& a, int u) {
  return (unit_keys(a, u) + TILE - 1) / TILE;
}

// A piece of a unit costs as much as some tiles before its first one and after its last (its
// queries, its first pages' way, its output): the units are laid end to end with so many ahead of
// each, so that a group with two pieces has less of them.  us without / with: 128 heads over 64 x
// 1K to 8K bf16 154 / 131, 32 heads x 4 tokens over 8 x 64K to 128K E4M3 230 / 214, 16 heads over
// 64 x 1K to 8K E4M3 54 / 50; with half as many 135, 224 and 53.
template <int TILE>
__device__ __forceinline__ int unit_head(const LatentAttnArgs& a) {
  return a.unit_groups ? 0 : TILE == 64 ? 6 : 8;
}
template <int TILE>
__device__ __forceinline__ int unit_size(const LatentAttnArgs& a, int u) {
  const int n = unit_tiles<TILE>(a, u);
  return n > 0 ? n + unit_head<TILE>(a) : 0;
}

// Eight codes (code i in byte i of the two dwords) to bf16, exactly.
__device__ __forceinline__ bf16x8 decode8(u32x2 w) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w.x, 1.f, false);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w.x, 1.f, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w.y, 1.f, false);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w.y, 1.f, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// a and b as two E4M3 numbers each, times `scale` (a power of two): what is nearest, and what is
// nearest to the rest.  Into half `which` / 2 of the dwords hi and lo.
__device__ __forceinline__ void split(float a, float b, float scale, int which, int& hi, int& lo) {
  s16x2 h = __builtin_bit_cast(s16x2, hi), l = __builtin_bit_cast(s16x2, lo);
  f32x2 near;
  if (which) {
    h = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(h, a, b, scale, true);
    near = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(__builtin_bit_cast(int, h), scale, true);
    l = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(l, a - near[0], b - near[1], scale, true);
  } else {
    h = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(h, a, b, scale, false);
    near = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(__builtin_bit_cast(int, h), scale, false);
    l = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(l, a - near[0], b - near[1], scale, false);
  }
  hi = __builtin_bit_cast(int, h);
  lo = __builtin_bit_cast(int, l);
}
// c + a b over 128 E4M3 codes a row and a column, each lane's part of b times 2^(b_exp - 127).
__device__ __forceinline__ f32x4 mx_mfma(i32x8 a, i32x8 b, f32x4 c, int b_exp) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 0, 0, 0, 127, 0, b_exp);
}

// A query's latent part as the sum of two E4M3 numbers, 2^q_exp times each: four bits and what
// they leave of bf16's eight, so exact but below 2^-10 of the row's largest element, where at
// most 2^-17 of that is lost.  Two products of twice the rate, and the codes enter them as they
// are.  NaN and infinities become NaN.  LW: windows of 128 elements.  A lane's elements of a
// window: 32 from 32 q4 on, its two chunks of 16 exchanged for odd q4, as the keys' are.
template <int LW>
__device__ __forceinline__ void read_query(const uint16_t* row, int q4, bf16x8 (&x)[4 * LW]) {
#pragma unroll
  for (int i = 0; i < 4 * LW; ++i)
    x[i] = *(const bf16x8*)(row + (i >> 2) * 128 + q4 * 32 + (((i & 3) * 8) ^ (q4 & 1) << 4));
}
// Returns the exponent as the product takes it.
template <int LW>
__device__ __forceinline__ int split_query(const bf16x8 (&x)[4 * LW], i32x8 (&qh)[LW],
                                           i32x8 (&ql)[LW]) {
  float top = 0.f;
#pragma unroll
  for (int i = 0; i < 4 * LW; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf((float)x[i][e]));
  top = max_over_key_groups(top);
  const int q_exp = min(max((int)(__float_as_uint(top) >> 23), 1), 254) - 127 - 7;
  const float scale = __uint_as_float((uint32_t)min(max(q_exp + 127, 1), 254) << 23);
#pragma unroll
  for (int i = 0; i < 4 * LW; ++i) {
    int hi[2] = {0, 0}, lo[2] = {0, 0};
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
      const float v0 = (float)x[i][e], v1 = (float)x[i][e + 1];
      const float s0 = v0 + v0 * 0.f, s1 = v1 + v1 * 0.f;
      split(s0, s1, scale, e & 2, hi[e >> 2], lo[e >> 2]);
    }
    qh[i >> 2][(i & 3) * 2] = hi[0], qh[i >> 2][(i & 3) * 2 + 1] = hi[1];
    ql[i >> 2][(i & 3) * 2] = lo[0], ql[i >> 2][(i & 3) * 2 + 1] = lo[1];
  }
  return min(max(q_exp + 127, 1), 254);
}

// Where in a window (128 bytes each of eight keys) the 16 bytes `c` of key `key` lie.  LDS reads
// 256 bytes a cycle if the sixteen lanes that it serves at once, of eight keys and two
// neighbouring chunks, differ in their place in 256 bytes: 4.0 cycles a read of a wave so, 8.0
// with every second place unused.
template <bool FP8>
__device__ __forceinline__ int spot(int key, int c) {
  if constexpr (FP8) return (key & 7) * 128 + ((c ^ (key & 7) ^ (key >> 1 & 4)) << 4);
  else
    return (key >> 1 & 3) * 256 + ((((key & 1) << 3 | c) ^ ((key & 6) | (key >> 3 & 1) * 9)) << 4);
}
// What lane l of a load brings of a window of group g: the 16 bytes for place 16 l.
template <bool FP8, int ROW>
__device__ __forceinline__ int window_offset(int l, int g) {
  if constexpr (FP8) {
    return (l >> 3) * ROW + (((l & 7) ^ (l >> 3) ^ ((g & 1) << 2)) << 4);
  } else {
    const int hc = (l & 15) ^ ((l >> 4) * 2 | (g & 1) * 9);
    return ((l >> 4) * 2 + (hc >> 3)) * ROW + ((hc & 7) << 4);
  }
}

// The lane, worked out anew each time: places that follow from it, kept over a loop, would cost
// registers that the products need, and loads of spilled ones would wait for the tiles in flight.
__device__ __forceinline__ int lane_now() {
  int l;
  asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(l));
  return l;
}

}  // namespace pdec
