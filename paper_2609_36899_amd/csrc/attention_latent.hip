// Attention of one or several query tokens per sequence over latent pages, with the sequence
// lengths on the device: keys and values are one shared vector a token (the absorbed form).
//
//   out[b][j][h] = softmax(scale * q[b][j][h] . (c | k)^T) c  over positions
//   0 .. lens[b] - n_q + j of sequence b, c a token's latent of R elements, k its rotary key.
//
// Rows.  A sequence's query rows (tokens x heads, all of which read the same keys) go in
// blocks of up to 128, a unit each; a tile of 32 or 64 keys comes into LDS once for the block.
// Per key 2 (2 R + 64) operations a row stand against (R + 64) 2 bytes (bf16), R + 132 (E4M3):
// at R = 512 HBM bounds blocks of up to some 64 rows (E4M3) or 115 (bf16), the matrix units
// more.
//
// Work split.  The units' tiles laid end to end are cut into n_groups equal stretches, one for
// each work group, found from the lengths on the device (stretch.h).  The piece of unit u in
// group w leaves its softmax partial in slot w + u; the merge pass joins a unit's pieces.  A
// unit that one group covers whole is written out at once, and where there are many units, or
// none can be long, each has a group of its own.
//
// One tile.  S^T = K Q^T with the waves along rows and keys, then the weights P go through LDS
// and every wave multiplies all of the block's P by its eighth of the latent's width: O^T =
// C^T P^T.  So O takes 16 registers a row tile instead of 128, and each latent is read from
// LDS once in the second product, transposed by the read itself (ds_read_tr).  The tiles come
// by LDS-DMA into a ring of stages, 16-byte chunk n of a key's row in place n ^ (key & 7) of
// its 128 bytes, so that eight lanes reading the same chunk of eight keys meet all banks.
#include "hip_common.h"
#include "kernels.h"
#include "stretch.h"

#include <algorithm>
#include <type_traits>

namespace pdec {

namespace {

constexpr int kThreads = 512, kWaves = kThreads / 64, kRope = kLatentRope;
constexpr int kLoaders = 4;  // waves that bring the tiles, one on each SIMD
// A row's reference maximum moves only where its scores outgrow it by this many powers of
// two: the weights are then up to 2^16 instead of 1, no less exact, and the accumulators are
// rescaled a few times a row instead of at most tiles.
constexpr float kSlack = 16.f;

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef int s32x2 __attribute__((ext_vector_type(2)));
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

// Eight codes (code i in byte i of the two dwords) to bf16, exactly.
__device__ __forceinline__ bf16x8 decode8(u32x2 w) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w.x, 1.f, false);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w.x, 1.f, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w.y, 1.f, false);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w.y, 1.f, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

template <int R, int RT, bool FP8>
struct Form {
  static constexpr int kRow = FP8 ? R + 2 * kRope : (R + kRope) * 2;  // a key's bytes
  // What LDS holds beside the weights: four stages of 32 wide rows, or three of 64.
  static constexpr int kTile = latent_tile(FP8, R), kStages = kTile == 32 ? 4 : 3;
  static constexpr int kStage = kTile * kRow;
  static constexpr int kRows = 16 * RT;
  // Waves along rows, a tile of 16 each, and along keys in the first product; key tiles of a wave.
  static constexpr int WR = RT;
  static constexpr int WK = kTile / 16 < kWaves / WR ? kTile / 16 : kWaves / WR;
  static constexpr int KTW = kTile / 16 / WK;
  // LDS offsets.
  static constexpr int kP = kStages * kStage;             // weights [kRows][kTile] bf16
  static constexpr int kScale = kP + kRows * kTile * 2;   // [kStages][kTile]
  static constexpr int kTop = kScale + (FP8 ? kStages * kTile * 4 : 0);  // [WK][kRows]
  static constexpr int kAlpha = kTop + WK * kRows * 4;    // [kRows]
  static constexpr int kLim = kAlpha + kRows * 4;         // [kRows]: keys that a row sees
  static constexpr int kFlag = kLim + kRows * 4;          // [WR], then the bad keys' mask
  static constexpr int kBytes = kFlag + 48;
  static_assert(kBytes <= 160 * 1024 - 64 && kRow % 128 == 0 && kStage % 128 == 0, "LDS layout");
};

template <int R, int RT, bool FP8>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2))) void
latent_attn_kernel(LatentAttnArgs a, const int32_t* __restrict__ table) {
  typedef Form<R, RT, FP8> F;
  constexpr int TILE = F::kTile, NST = F::kStages, ROW = F::kRow, WR = F::WR, WK = F::WK;
  constexpr int KTW = F::KTW, PPT = TILE / kPage;
  constexpr int KC = (R + kRope) / 32, LC = R / 32;  // k-steps of QK^T; of the latent part
  constexpr int DT = R / 16 / kWaves;                // 16-wide tiles of a wave's part of R
  constexpr int CPR = ROW / 16;                      // chunks of a row
  constexpr int KPW = TILE / kLoaders;               // keys that a loading wave brings
  constexpr int NV = 8 * CPR / 64;                   // loads of eight keys
  constexpr int NL = NV * (KPW / 8) + (FP8 ? 1 : 0);  // a wave's loads of a tile
  static_assert(8 * CPR % 64 == 0 && KPW % 8 == 0 && (!FP8 || KPW == kPage), "whole loads");
  __shared__ __attribute__((aligned(128))) uint8_t lds[F::kBytes];
  __shared__ int red[kWaves];
  __shared__ int found[2];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int c16 = lane & 15, q4 = lane >> 4;
  const int rw = wave % WR, kw = wave / WR;
  const bool active = kw < WK;  // in the first product
  const int w = blockIdx.x;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(PDEC_LDS uint8_t*)lds;

  int at = 0, end, u = w, first = 0;
  if (a.unit_groups) {
    end = unit_tiles<TILE>(a, u);
    if (end == 0) {
      const int row0 = unit_row0(a, u), rows = unit_rows(a, row0);
      uint16_t* o = (uint16_t*)a.out +
                    ((int64_t)(u / a.blocks_per_seq) * a.n_q * a.n_heads + row0) * R;
      for (int i = threadIdx.x; i < rows * (R / 8); i += kThreads)
        *(u32x4*)(o + i * 8) = u32x4{0, 0, 0, 0};
      return;
    }
  } else {
    const Stretch mine = stretch_of<kThreads>(a.n_units, a.n_groups, a.min_tiles, w, red, found,
                                              [&](int v) { return unit_tiles<TILE>(a, v); });
    at = w * mine.per;
    if (at >= mine.total) return;
    end = min(at + mine.per, mine.total);
    u = __builtin_amdgcn_readfirstlane(mine.unit);
    first = __builtin_amdgcn_readfirstlane(mine.first);
    at = __builtin_amdgcn_readfirstlane(at);
    end = __builtin_amdgcn_readfirstlane(end);
  }

  // The order of a tile's keys in the second product.  The transposing read of bf16 gives a
  // lane four keys, which must differ in their place in the 128 bytes (two chunks of a key
  // side by side are exchanged by the key's lowest bit): every other key of eight.  So slot
  // 8 g + i is key 8 g + 2 i for i < 4, 8 g + 2 (i - 4) + 1 behind.  Of E4M3 codes it gives
  // eight keys, in order.
  auto key_of = [](int slot) { return FP8 ? slot : (slot & ~7) | ((slot & 3) << 1) | (slot >> 2 & 1); };
  auto slot_of = [](int key) { return FP8 ? key : (key & ~7) | ((key >> 1) & 3) | ((key & 1) << 2); };
  // Where row `row`'s weight of slot `slot` lies (a multiple of four): chunks exchanged by the
  // row, as the keys' are.
  auto p_at = [](int row, int slot) {
    const int byte = slot * 2, c = byte >> 4;
    if constexpr (TILE == 64) return F::kP + row * 128 + ((c ^ (row & 7)) << 4) + (byte & 15);
    else
      return F::kP + (row >> 1) * 128 + ((((row & 1) << 2) | (c ^ (row >> 1 & 3))) << 4) + (byte & 15);
  };

  // The lane, as a value that the compiler takes for new each time: places worked out from it
  // and kept over the loop would cost registers that the products need, and loads of spilled
  // ones would wait for the tiles in flight.
  auto lane_now = [&] {
    int l = lane;
    asm volatile("" : "+v"(l));
    return l;
  };

  for (; at < end; ++u) {
    const int tiles = unit_tiles<TILE>(a, u);
    if (first + tiles <= at) {  // empty unit
      first += tiles;
      continue;
    }
    const int b = u / a.blocks_per_seq, row0 = unit_row0(a, u), rows = unit_rows(a, row0);
    const int base_lim = clamp_len(a, b) - a.n_q + 1;  // keys that token 0 sees
    const int kv_lim = max(base_lim + (row0 + rows - 1) / a.n_heads, 0);
    const int min_lim = max(base_lim + row0 / a.n_heads, 0);  // keys that every row sees
    const int n_pages = (kv_lim + kPage - 1) / kPage;
    const int p_begin = at - first, p_end = min(tiles, end - first);
    const int64_t q_row0 = (int64_t)b * a.n_q * a.n_heads + row0;
    const int32_t* bt = table + (int64_t)b * a.bt_stride;

    // The pages of a tile: the one that this wave brings (-1: none), and which of them there are.
    struct Spot {
      int page, ok;
    };
    auto look = [&](int t) {
      Spot s = {-1, 0};
#pragma unroll
      for (int i = 0; i < PPT; ++i) {
        const int n = t * PPT + i;
        int page = t < p_end && n < n_pages ? bt[n] : -1;
        if (page < 0 || page >= a.n_pages) page = -1;
        if (page >= 0) s.ok |= 1 << i;
        if (i == wave * PPT / kLoaders) s.page = page;
      }
      return s;
    };
    // A page that is not there is a buffer without bytes: its loads bring nothing, and count.
    auto issue = [&](const Spot& s, int st) {
      if (wave >= kLoaders) return;
      const bool on = s.page >= 0;
      const int64_t page = on ? s.page : 0;
      constexpr int kPart = KPW * ROW;  // this wave's part of the tile
      DmaBuffer src = dma_buffer(
          (const uint8_t*)a.pages + page * (kPage * ROW) + (KPW < kPage ? (wave & 1) * kPart : 0),
          on ? kPart : 0);
      uint32_t to = lds0 + st * F::kStage + wave * kPart;
      dma_ready(src, to);
      // Eight keys' chunks in LDS order, each from its place in the page.
      const int l = lane_now();
      int voff[NV];
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int n = i * 64 + l, key = n / CPR, c = n % CPR;
        voff[i] = key * ROW + ((c ^ key) << 4);
      }
#pragma unroll
      for (int h = 0; h < KPW / 8; ++h)
#pragma unroll
        for (int i = 0; i < NV; ++i)
          dma16_unseen(src, voff[i], h * 8 * ROW, to + (h * NV + i) * 1024);
      if constexpr (FP8) {
        DmaBuffer sc = dma_buffer(a.scales + page * kPage, on ? kPage * 4 : 0);
        uint32_t to = lds0 + F::kScale + (st * TILE + wave * kPage) * 4;
        dma_ready(sc, to);
        if (lane < kPage) dma4_unseen(sc, lane * 4, to);
      }
    };

    wait_vmem<0>();
    __syncthreads();  // the piece before is done with LDS
    Spot next = look(p_begin);
    uint32_t ok = 0;  // four bits a stage
    auto push = [&](int t, int st) {
      issue(next, st);
      ok = (ok & ~(15u << (4 * st))) | (uint32_t)next.ok << (4 * st);
      next = look(t + 1);
    };
    push(p_begin, 0);
    bf16x8 qf[KC];
    int row_lim;  // keys that this lane's row sees
    {
      const int row = min(rw * 16 + c16, rows - 1);  // rows past the block's repeat its last
      row_lim = base_lim + (row0 + row) / a.n_heads;
      if (kw == 0 && q4 == 0) *(int*)(lds + F::kLim + (rw * 16 + c16) * 4) = row_lim;
      const uint16_t* src = (const uint16_t*)a.q + (q_row0 + row) * (R + kRope);
#pragma unroll
      for (int c = 0; c < KC; ++c) {
        const int dim = FP8 && c < LC ? (c >> 1) * 64 + q4 * 16 + (c & 1) * 8 : c * 32 + q4 * 8;
        qf[c] = *(const bf16x8*)(src + dim);
      }
    }
    // Here the queries are waited for, and the first tile with them; the others' loads follow.
#pragma unroll
    for (int c = 0; c < KC; ++c) asm volatile("" : "+v"(qf[c]));
#pragma unroll
    for (int i = 1; i < NST - 1; ++i) push(p_begin + i, i);

    float m = -INFINITY, l = 0.f;  // a reference for the row's scores; this lane's part of its sum
    f32x4 acc[RT][DT];
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
      for (int d = 0; d < DT; ++d) acc[t][d] = f32x4{0.f, 0.f, 0.f, 0.f};

    int st = 0;
    for (int p = p_begin; p < p_end; ++p) {
      wait_vmem<(NST - 2) * NL>();
      wg_barrier();  // this tile is here, and the one before has been used
      push(p + NST - 1, st == 0 ? NST - 1 : st - 1);
      const uint8_t* tile = lds + st * F::kStage;
      const int key0 = p * TILE, here = ok >> (4 * st) & 15;
      // Keys that some row does not see, or that are not there.
      const bool cut = key0 + TILE > min_lim || here != (1 << PPT) - 1;
      auto there = [&](int key) { return key0 + key < kv_lim && (here >> (key / kPage) & 1); };
      uint64_t bad = 0;  // keys that only some rows see and that are not finite
      if (cut) {
        uint32_t* odd_keys = (uint32_t*)(lds + F::kFlag + 32);
        if (threadIdx.x < 2) odd_keys[threadIdx.x] = 0;
        __syncthreads();
        // 0 times what a key without data holds may be NaN: it becomes 0.
        constexpr int CL = (FP8 ? R : 2 * R) / 16;  // chunks of a latent
        for (int i = threadIdx.x; i < TILE * CL; i += kThreads) {
          const int key = i / CL;
          u32x4* at = (u32x4*)(lds + st * F::kStage + key * ROW + i % CL * 16);
          if (!there(key)) {
            *at = u32x4{0, 0, 0, 0};
          } else if (key0 + key >= min_lim) {
            bool odd = false;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const uint32_t x = (*at)[e];
              if constexpr (FP8) {
#pragma unroll
                for (int s = 0; s < 32; s += 8) odd |= (x >> s & 0x7F) == 0x7F;
              } else {
                odd |= (x & 0x7F80) == 0x7F80 || (x >> 16 & 0x7F80) == 0x7F80;
              }
            }
            if (odd) atomicOr(&odd_keys[key >> 5], 1u << (key & 31));
          }
        }
        __syncthreads();
        bad = (uint64_t)odd_keys[1] << 32 | odd_keys[0];
      }

      const int l1 = lane_now(), row_l = l1 & 15, q_l = l1 >> 4;
      const int key_a = KTW * kw * 16 + key_of(row_l);  // this lane's key in the first product
      const int k_base = key_a * ROW + ((q_l ^ (key_a & 7)) << 4);
      const uint8_t* at0 = tile + k_base;
      const uint8_t* at1 = tile + (k_base ^ 64);
      // Scores of key tile k of this wave against its rows: key slot 4 q4 + e of column c16.  Of
      // E4M3 pages the latent part is scaled, by the tokens' scales vs, before the rotary part.
      // The reads of a few steps are under way while those before are multiplied, and no more:
      // they would take the registers that O lies in.
      auto scores = [&](int k, f32x4 vs) {
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
        const uint8_t* k0 = at0 + k * 16 * ROW;
        const uint8_t* k1 = at1 + k * 16 * ROW;
        if constexpr (FP8) {
          constexpr int G = 2, N = LC / 2;
          u32x4 x[2][G];
          bf16x8 r[2];
          auto read = [&](int g) {
#pragma unroll
            for (int i = 0; i < G; ++i)
              x[g & 1][i] = *(const u32x4*)((i & 1 ? k1 : k0) + (g * G + i) / 2 * 128);
          };
          read(0);
#pragma unroll
          for (int g = 0; g < N / G; ++g) {
            if (g + 1 < N / G) {
              read(g + 1);
            } else {
              r[0] = *(const bf16x8*)(k0 + R);
              r[1] = *(const bf16x8*)(k1 + R);
            }
#pragma unroll
            for (int i = 0; i < G; ++i) {
              const u32x4 y = x[g & 1][i];
              o = __builtin_amdgcn_mfma_f32_16x16x32_bf16(decode8(u32x2{y.x, y.y}), qf[2 * (g * G + i)],
                                                          o, 0, 0, 0);
              o = __builtin_amdgcn_mfma_f32_16x16x32_bf16(decode8(u32x2{y.z, y.w}),
                                                          qf[2 * (g * G + i) + 1], o, 0, 0, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
          }
          o *= vs;
#pragma unroll
          for (int c = 0; c < 2; ++c)
            o = __builtin_amdgcn_mfma_f32_16x16x32_bf16(r[c], qf[LC + c], o, 0, 0, 0);
        } else {
          constexpr int G = KC % 3 == 0 ? 3 : 2;
          static_assert(KC % G == 0, "whole groups");
          bf16x8 x[2][G];
          auto read = [&](int g) {
#pragma unroll
            for (int i = 0; i < G; ++i) {
              const int c = g * G + i;
              x[g & 1][i] = *(const bf16x8*)((c & 1 ? k1 : k0) + (c >> 1) * 128);
            }
          };
          read(0);
#pragma unroll
          for (int g = 0; g < KC / G; ++g) {
            if (g + 1 < KC / G) read(g + 1);
#pragma unroll
            for (int i = 0; i < G; ++i)
              o = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[g & 1][i], qf[g * G + i], o, 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
          }
        }
        return o;
      };
      auto token_scales = [&](int k) {
        return FP8 ? *(const f32x4*)(lds + F::kScale + (st * TILE + (kw * KTW + k) * 16 + 4 * q_l) * 4)
                   : f32x4{1.f, 1.f, 1.f, 1.f};
      };
      // Where a row does not see a key the score is -inf, and the scale, which may be anything, 0.
      auto mask = [&](int k, f32x4& x, f32x4& vs) {
        if (!cut) return;
        const int page = kw * KTW + k;
        int lim = here >> page & 1 ? row_lim - key0 - page * kPage : 0;
        asm volatile("" : "+v"(lim));  // compared here, not ahead of the branch
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (key_of(4 * q_l + e) >= lim) {
            x[e] = -INFINITY;
            vs[e] = 0.f;
          }
      };
      // The weights of key tile k, into LDS; returns their sum.  They enter the second product
      // in bf16, each off by at most half a step (2^-8); the normaliser is the fp32 sum of the
      // weights as they were rounded, so that what the rounding does to a row's large weights
      // cancels.  A token's latent scale goes with its weight: exact for powers of two, another
      // half step for scales that are none.
      auto weigh = [&](int k, f32x4 x, f32x4 vs) {
        const float base = m == -INFINITY ? 0.f : m;
        u32x2 pw;
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 4; e += 2) {
          f32x2 y = {__builtin_amdgcn_exp2f(__builtin_fmaf(x[e], a.scale_log2, -base)),
                     __builtin_amdgcn_exp2f(__builtin_fmaf(x[e + 1], a.scale_log2, -base))};
          uint32_t bits = __builtin_bit_cast(uint32_t, __builtin_convertvector(y, bf16x2));
          y = f32x2{__uint_as_float(bits << 16), __uint_as_float(bits & 0xFFFF0000u)};
          sum += y[0] + y[1];
          if constexpr (FP8) {
            y[0] *= vs[e];
            y[1] *= vs[e + 1];
            bits = __builtin_bit_cast(uint32_t, __builtin_convertvector(y, bf16x2));
          }
          pw[e / 2] = bits;
        }
        *(u32x2*)(lds + p_at(rw * 16 + row_l, (kw * KTW + k) * 16 + 4 * q_l)) = pw;
        return sum;
      };
      // The row's reference follows a top that outgrows it; O is rescaled behind the barrier.
      int moved = 0;
      auto follow = [&](float top) {
        const float now = top * a.scale_log2;
        const bool need = now > m + kSlack, begun = m > -INFINITY;
        const float alpha = need && begun ? __builtin_amdgcn_exp2f(m - now) : 1.f;
        if (need) m = now;
        l *= alpha;
        moved = __any(need && begun);
        if (moved && kw == 0 && q_l == 0) *(float*)(lds + F::kAlpha + (rw * 16 + row_l) * 4) = alpha;
      };
      if constexpr (WK == 1) {
        // The weights at the reference as it was; where that was too low (a piece's first tile,
        // and hardly ever again) all over again.
        float sum;
        for (;;) {
          float top = -INFINITY;
          sum = 0.f;
#pragma unroll 1  // unrolled, its places in LDS spill
          for (int k = 0; k < KTW; ++k) {
            f32x4 vs = token_scales(k), x = scores(k, vs);
            mask(k, x, vs);
            top = fmaxf(fmaxf(fmaxf(top, x[0]), fmaxf(x[1], x[2])), x[3]);
            sum += weigh(k, x, vs);
            __builtin_amdgcn_sched_barrier(0);
          }
          if (!__any(top * a.scale_log2 > m + kSlack)) break;
          follow(max_over_key_groups(top));
        }
        l += sum;
      } else {
        f32x4 x[KTW], vs[KTW];
        float* tops = (float*)(lds + F::kTop);
        if (active) {
          float top = -INFINITY;
#pragma unroll
          for (int k = 0; k < KTW; ++k) {
            vs[k] = token_scales(k);
            x[k] = scores(k, vs[k]);
            mask(k, x[k], vs[k]);
            top = fmaxf(fmaxf(fmaxf(top, x[k][0]), fmaxf(x[k][1], x[k][2])), x[k][3]);
          }
          top = max_over_key_groups(top);
          if (q_l == 0) tops[kw * F::kRows + rw * 16 + row_l] = top;
        }
        wg_barrier();
        if (active) {
          float top = -INFINITY;  // over the waves that share the rows
#pragma unroll
          for (int k = 0; k < WK; ++k) top = max2(top, tops[k * F::kRows + rw * 16 + row_l]);
          follow(top);
#pragma unroll
          for (int k = 0; k < KTW; ++k) l += weigh(k, x[k], vs[k]);
        }
      }
      if (kw == 0 && l1 == 0) *(int*)(lds + F::kFlag + rw * 4) = moved;
      wg_barrier();

      int any = 0;
#pragma unroll
      for (int i = 0; i < WR; ++i) any |= *(const int*)(lds + F::kFlag + i * 4);
      if (__builtin_amdgcn_readfirstlane(any)) {
        const int c16 = lane_now() & 15;
#pragma unroll
        for (int t = 0; t < RT; ++t) {
          // Not written where a wave's own rows did not move.
          const int mine = *(const int*)(lds + F::kFlag + t * 4);
          const float f = *(const float*)(lds + F::kAlpha + (t * 16 + c16) * 4);
          const float alpha = mine ? f : 1.f;
#pragma unroll
          for (int d = 0; d < DT; ++d) acc[t][d] *= alpha;
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      if (bad) {  // uniform
        const int l3 = lane_now(), c16 = l3 & 15, q4 = l3 >> 4;
        // Keys that some rows do not see and that are not finite: a weight of 0 would leave
        // NaN of them.  They are added here for the rows that see them, and are 0 behind.
        for (uint64_t rest = bad; rest; rest &= rest - 1) {
          const int key = __builtin_ctzll(rest), slot = slot_of(key);
          f32x4 v[DT];
#pragma unroll
          for (int d = 0; d < DT; ++d) {
            const int dim = wave * (R / kWaves) + d * 16 + 4 * q4;
            if constexpr (FP8) {
              const uint32_t x = *(const uint32_t*)(tile + key * ROW + ((dim >> 4 ^ (key & 7)) << 4) +
                                                    (dim & 15));
              const bf16x8 y = decode8(u32x2{x, 0});
              v[d] = f32x4{(float)y[0], (float)y[1], (float)y[2], (float)y[3]};
            } else {
              const u32x2 x = *(const u32x2*)(tile + key * ROW + ((dim >> 3 ^ (key & 7)) << 4) +
                                              (dim & 7) * 2);
              v[d] = f32x4{__uint_as_float(x.x << 16), __uint_as_float(x.x & 0xFFFF0000u),
                           __uint_as_float(x.y << 16), __uint_as_float(x.y & 0xFFFF0000u)};
            }
          }
#pragma unroll
          for (int t = 0; t < RT; ++t) {
            const int row = t * 16 + c16;
            const float w =
                bf16_to_f32(*(const uint16_t*)(lds + p_at(row, slot & ~3) + (slot & 3) * 2));
            if (key0 + key < *(const int*)(lds + F::kLim + row * 4))
#pragma unroll
              for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[t][d][e] = __builtin_fmaf(w, v[d][e], acc[t][d][e]);
            __builtin_amdgcn_sched_barrier(0);
          }
        }
        __syncthreads();
        for (int i = threadIdx.x; i < TILE * CPR; i += kThreads)
          if (bad >> (i / CPR) & 1) *(u32x4*)(lds + st * F::kStage + i * 16) = u32x4{0, 0, 0, 0};
        __syncthreads();
      }
      // The lane's key in a block of 32 keys, and its place among the wave's dims.
      const int l2 = lane_now(), row_2 = l2 & 15, q_2 = l2 >> 4;
      const int v_key = 8 * q_2 + (FP8 ? row_2 >> 1 : 2 * (row_2 >> 2));
      const int v_chunk = FP8 ? wave * DT : wave * DT * 2 + ((row_2 & 3) >> 1);
      const int v_base = v_key * ROW + ((v_chunk ^ (v_key & 7)) << 4) + ((row_2 & 1) << 3);
#pragma unroll
      for (int kb = 0; kb < TILE / 32; ++kb) {
        bf16x8 v[DT];
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          if constexpr (FP8) {
            const uint8_t* from = tile + ((v_base ^ (d << 4)) + kb * 32 * ROW);
            v[d] = decode8(__builtin_bit_cast(
                u32x2, __builtin_amdgcn_ds_read_tr8_b64_v2i32((PDEC_LDS s32x2*)from)));
          } else {
            const uint8_t* from = tile + ((v_base ^ (d << 5)) + kb * 32 * ROW);
            const uint8_t* odd = tile + ((v_base ^ 16 ^ (d << 5)) + (kb * 32 + 1) * ROW);
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((PDEC_LDS s16x4*)from);
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((PDEC_LDS s16x4*)odd);
            v[d] = __builtin_bit_cast(
                bf16x8, s16x8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]});
          }
        }
#pragma unroll
        for (int t = 0; t < RT; ++t) {
          const bf16x8 pf = *(const bf16x8*)(lds + p_at(t * 16 + row_2, kb * 32 + q_2 * 8));
#pragma unroll
          for (int d = 0; d < DT; ++d)
            acc[t][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[d], pf, acc[t][d], 0, 0, 0);
        }
      }
      st = st + 1 == NST ? 0 : st + 1;
    }

    // The rows' sums and maxima meet every wave's part of the output.
    wg_barrier();
    float* sums = (float*)(lds + F::kTop);
    float* tops = (float*)(lds + F::kAlpha);
    if (active) {
      const int row = rw * 16 + c16;
      const float sum = sum_over_key_groups(l);
      if (q4 == 0) {
        sums[kw * F::kRows + row] = sum;
        if (kw == 0) tops[row] = m;
      }
    }
    wg_barrier();
    const bool whole = p_begin == 0 && p_end == tiles;
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      const int row = t * 16 + c16;
      if (row >= rows) continue;
      float sum = 0.f;
#pragma unroll
      for (int k = 0; k < WK; ++k) sum += sums[k * F::kRows + row];
      if (whole) {
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        uint16_t* o = (uint16_t*)a.out + (q_row0 + row) * R + wave * (R / kWaves) + 4 * q4;
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          const f32x2 lo = {acc[t][d][0] * inv, acc[t][d][1] * inv};
          const f32x2 hi = {acc[t][d][2] * inv, acc[t][d][3] * inv};
          *(u32x2*)(o + d * 16) =
              u32x2{__builtin_bit_cast(uint32_t, __builtin_convertvector(lo, bf16x2)),
                    __builtin_bit_cast(uint32_t, __builtin_convertvector(hi, bf16x2))};
        }
      } else {
        const int64_t pr = ((int64_t)w + u) * F::kRows + row;
        if (wave == 0 && q4 == 0) *(float2*)(a.part_ml + pr * 2) = float2{tops[row], sum};
        float* o = a.part_acc + pr * R + wave * (R / kWaves) + 4 * q4;
#pragma unroll
        for (int d = 0; d < DT; ++d) *(f32x4*)(o + d * 16) = acc[t][d];
      }
    }
    at = first + p_end;
    first += tiles;
  }
  wait_vmem<0>();  // no LDS write may still be in flight when the group ends
}

// Merges the pieces of each unit, and writes zeros for the rows of a unit that sees no key.
// A work group per row of a unit: R / 4 lanes a piece, the others' pieces side by side, then
// the results in order.
template <int R, int TILE>
__global__ __launch_bounds__(512) void latent_merge_kernel(LatentAttnArgs a, int rows_per_unit) {
  constexpr int L = R / 4, S = 512 / L;  // lanes of a piece, pieces at once
  __shared__ int red[2][8];
  __shared__ float sh[S - 1][6][L];
  const int u = blockIdx.x, row0 = unit_row0(a, u), row = blockIdx.y;
  if (row >= unit_rows(a, row0)) return;
  int all = 0, before = 0;
  for (int v = threadIdx.x; v < a.n_units; v += 512) {
    const int n = unit_tiles<TILE>(a, v);
    all += n;
    before += v < u ? n : 0;
  }
  all = wave_add(all);
  before = wave_add(before);
  if ((threadIdx.x & 63) == 0) {
    red[0][threadIdx.x >> 6] = all;
    red[1][threadIdx.x >> 6] = before;
  }
  __syncthreads();
  int total = 0, first = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    total += red[0][i];
    first += red[1][i];
  }
  const int per = max((total + a.n_groups - 1) / a.n_groups, a.min_tiles);
  const int tiles = unit_tiles<TILE>(a, u), w0 = first / per;
  const int w1 = tiles > 0 ? (first + tiles - 1) / per : w0 - 1;
  if (tiles > 0 && w0 == w1) return;
  const int lane = threadIdx.x % L, part = threadIdx.x / L;
  float m = -INFINITY, l = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  auto join = [&](float mi, float li, f32x4 oi) {
    const float mn = fmaxf(m, mi), mu = mn == -INFINITY ? 0.f : mn;
    const float so = exp2f(m - mu), si = exp2f(mi - mu);
    l = l * so + li * si;
    o = o * so + oi * si;
    m = mn;
  };
  for (int w = w0 + part; w <= w1; w += 8 * S) {
    float2 ml[8];
    f32x4 x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int64_t pr = ((int64_t)min(w + i * S, w1) + u) * rows_per_unit + row;
      ml[i] = *(const float2*)(a.part_ml + pr * 2);
      x[i] = *(const f32x4*)(a.part_acc + pr * R + lane * 4);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (w + i * S <= w1) join(ml[i].x, ml[i].y, x[i]);
  }
  if (part > 0) {
    float(*d)[L] = sh[part - 1];
    d[0][lane] = m;
    d[1][lane] = l;
#pragma unroll
    for (int e = 0; e < 4; ++e) d[2 + e][lane] = o[e];
  }
  __syncthreads();
  if (part > 0) return;
#pragma unroll
  for (int i = 0; i < S - 1; ++i) {
    const float(*d)[L] = sh[i];
    join(d[0][lane], d[1][lane], f32x4{d[2][lane], d[3][lane], d[4][lane], d[5][lane]});
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  const f32x2 lo = {o[0] * inv, o[1] * inv}, hi = {o[2] * inv, o[3] * inv};
  *(u32x2*)((uint16_t*)a.out +
            ((int64_t)(u / a.blocks_per_seq) * a.n_q * a.n_heads + row0 + row) * R + lane * 4) =
      u32x2{__builtin_bit_cast(uint32_t, __builtin_convertvector(lo, bf16x2)),
            __builtin_bit_cast(uint32_t, __builtin_convertvector(hi, bf16x2))};
}

}  // namespace

hipError_t launch_latent_attention(int fp8, int latent, int row_tiles, const LatentAttnArgs& a,
                                   hipStream_t stream) {
  const dim3 grid(a.unit_groups ? a.n_units : a.n_groups);
#define PDEC_LATENT(R_, FP8_)                                                                    \
  do {                                                                                           \
    if (row_tiles == 1)                                                                          \
      latent_attn_kernel<R_, 1, FP8_><<<grid, kThreads, 0, stream>>>(a, a.block_table);          \
    else if (row_tiles == 2)                                                                     \
      latent_attn_kernel<R_, 2, FP8_><<<grid, kThreads, 0, stream>>>(a, a.block_table);          \
    else if (row_tiles == 4)                                                                     \
      latent_attn_kernel<R_, 4, FP8_><<<grid, kThreads, 0, stream>>>(a, a.block_table);          \
    else                                                                                         \
      latent_attn_kernel<R_, 8, FP8_><<<grid, kThreads, 0, stream>>>(a, a.block_table);          \
    hipError_t e = hipGetLastError();                                                            \
    if (e != hipSuccess || a.unit_groups) return e;                                              \
    const dim3 mgrid(a.n_units, std::min(a.block_rows, a.n_q * a.n_heads));                      \
    latent_merge_kernel<R_, latent_tile(FP8_, R_)><<<mgrid, 512, 0, stream>>>(a, 16 * row_tiles); \
  } while (0)
  if (latent == 512) {
    if (fp8) PDEC_LATENT(512, true);
    else PDEC_LATENT(512, false);
  } else {
    if (fp8) PDEC_LATENT(256, true);
    else PDEC_LATENT(256, false);
  }
#undef PDEC_LATENT
  return hipGetLastError();
}

}  // namespace pdec
