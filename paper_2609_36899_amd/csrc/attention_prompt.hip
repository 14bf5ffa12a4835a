// Attention of prompts over keys and values expanded from latents: for each head keys of DIM
// elements beside the rotary key that all heads share, and values of DIM.
//
//   out[i][h] = softmax(scale * (q[i][h][:DIM] . k[j][h] + q[i][h][DIM:] . rope_keys[j])) v[j][h]
//   over the keys j of i's sequence up to i's own: the last of its n_keys belong to its n_rows.
//
// Bound by the matrix units: 2 (2 DIM + 64) operations a pair of row and key.  A work group of
// four waves takes a block of 128 rows of one head, 32 a wave, over tiles of 32 keys that come
// into LDS by DMA, a ring of three; two groups a unit fill each other's gaps.  S^T = K Q^T, with
// the keys of a tile dealt to two MFMA tiles, even and odd ones, so that a lane's eight weights
// are the operand P of O^T = V^T P^T as they are, against V transposed by the LDS read
// (ds_read_tr).  LDS holds windows of 128 bytes of eight keys, laid so that the reads meet all
// banks; nothing is spilled, since a reload in the loop waits for the tiles on their way (284 us
// with spills, 139 without).
//
// Work split.  Per head the blocks' tiles laid end to end are cut into n_groups equal stretches
// (stretch.h), found from the sequences' starts on the device.  A stretch's first piece, where
// its block began before, and its last, where it goes on behind, leave partials; the merge pass
// joins each block that was cut.  Where there are enough blocks each has a group of its own.
//
// 20 heads over 4096 tokens, D = 128: 132 us (0.81 PFLOP/s) by a group a block, 141 by equal
// stretches, of which the merge 15; there each head more costs 5 us (1.07 PFLOP/s, where a large
// matrix product reaches 1.33), the beginnings, partials and merge some 50.  Tried without gain:
// the next tile's first product beside this one's weights in each wave, heads gathered by die,
// the loads one by one between the products.
#include "hip_common.h"
#include "kernels.h"
#include "lds_dma.h"
#include "stretch.h"

#include <algorithm>

namespace pdec {

namespace {

constexpr int kRope = kLatentRope;
constexpr float kSlack = 16.f;  // as of the attention over latents

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
#define PDEC_LDS __attribute__((address_space(3)))

// A sequence's rows and keys; starts are not trusted.  Where the rows' descend anywhere the call
// does nothing: sequences that share rows may be of more tiles in all than 32 bits count, and then
// no place among them means anything.
struct Seq {
  int q0, nq, k0, nk;
};
__device__ __forceinline__ Seq seq_of(const LatentPromptArgs& a, int b) {
  Seq s;
  s.q0 = min(max(a.q_start[b], 0), a.n_rows);
  s.nq = min(max(a.q_start[b + 1], s.q0), a.n_rows) - s.q0;
  s.k0 = min(max(a.k_start[b], 0), a.n_keys);
  s.nk = min(max(a.k_start[b + 1], s.k0), a.n_keys) - s.k0;
  return s;
}
// Whether they descend: each wave notes it of the sequences that stretch_of shows it, in a place of
// its own, whose barriers pass it on to descends().
__device__ __forceinline__ void note_descent(const LatentPromptArgs& a, int b, int* down) {
  if (a.q_start[b] > a.q_start[b + 1]) down[threadIdx.x >> 6] = 1;
}
template <int T>
__device__ __forceinline__ bool descends(const int* down) {
  int any = 0;
#pragma unroll
  for (int w = 0; w < T / 64; ++w) any |= down[w];
  return any;
}
// Tiles of block blk: those of the keys that its last row sees, at least one.
template <int ROWS, int TILE>
__device__ __forceinline__ int block_tiles(const Seq& s, int blk) {
  const int keys = s.nk - s.nq + min((blk + 1) * ROWS, s.nq);
  return max((keys + TILE - 1) / TILE, 1);
}
// The same and what a piece of a block costs beside its tiles (its queries, the first tiles' way,
// its output), in tiles, which equal stretches count ahead of each block's.  us at 0 / 2 / 4 / 12: 16
// heads over 4096 120 / 117 / 113 / 119, over 2048 53.5 / 52.8 / 50.7 / 51.2, four over 8192 115 / 113 /
// 111 / 112, 20 heads, 200 behind 20K, 102 / 101 / 100 / 99, 32 heads over five turns of 100 to 700
// 253 / 248 / 249 / 252.
constexpr int kHead = 4;
// That of the blocks before blk: of each whole block ROWS / TILE more than of the one before.
template <int ROWS, int TILE>
__device__ __forceinline__ int size_before(const Seq& s, int blk) {
  constexpr int K = ROWS / TILE;
  static_assert(K * TILE == ROWS && K % 2 == 0 && (TILE & (TILE - 1)) == 0, "whole tiles a block");
  const int full = s.nq / ROWS, n = min(blk, full);
  const int base = (s.nk - s.nq + TILE - 1) & -TILE, first = base / TILE;  // rounded up
  const int ones = min(max(-first / K, 0), n);  // blocks that no key is seen of
  // Modulo 2^32, where terms of a sequence with more rows than keys may be large.
  const uint32_t live = n - ones;
  const int sum = (int)(kHead * (uint32_t)blk + ones + live * (uint32_t)first +
                        K / 2 * live * (uint32_t)(n + ones + 1));
  return blk > full ? sum + block_tiles<ROWS, TILE>(s, full) : sum;
}
template <int ROWS, int TILE>
__device__ __forceinline__ int seq_size(const Seq& s) {
  return size_before<ROWS, TILE>(s, (s.nq + ROWS - 1) / ROWS);
}
// The block that tile `at` of a sequence's lies in.
template <int ROWS, int TILE>
__device__ __forceinline__ int block_of(const Seq& s, int at) {
  int lo = 0, hi = (s.nq + ROWS - 1) / ROWS;  // size_before(lo) <= at < size_before(hi)
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (size_before<ROWS, TILE>(s, mid) <= at) lo = mid;
    else hi = mid;
  }
  return lo;
}

constexpr int kWaves = 4, kThreads = 64 * kWaves, kRows = 32 * kWaves, kTile = 32, kStages = 3;

template <int DIM>
__global__ __launch_bounds__(kThreads, 2) void prompt_attn_kernel(LatentPromptArgs a) {
  constexpr int KC = (DIM + kRope) / 32, DT = DIM / 16;  // steps of the first product, tiles of dims
  // A tile in LDS, by groups of eight keys (a wave brings one): K, rotary, V, each of windows of
  // 128 bytes of the eight.
  constexpr int WIN = DIM / 64, GK = WIN * 1024, K = 4 * GK, ROPE = 4 * 1024;
  constexpr int STAGE = 2 * K + ROPE, NL = 2 * WIN + 1;
  __shared__ __attribute__((aligned(256))) uint8_t lds[kStages * STAGE];
  __shared__ __attribute__((aligned(16))) uint8_t weights[kWaves][32 * 64];
  __shared__ int red[kWaves];
  __shared__ int found[2];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = blockIdx.x;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(PDEC_LDS uint8_t*)lds;
  // With a group for each block the blocks' order is turned round, so that the long ones of a
  // prompt begin first (and of several prompts the last one's).
  const int w = a.block_groups ? gridDim.y - 1 - blockIdx.y : blockIdx.y;
  __shared__ int down[kWaves];
  if ((threadIdx.x & 63) == 0) down[wave] = 0;
  const Stretch mine = stretch_of<kThreads>(
      a.n_seqs, gridDim.y, a.block_groups ? 1 : a.min_tiles, w, red, found, [&](int b) {
        note_descent(a, b, down);
        const Seq s = seq_of(a, b);
        return a.block_groups ? (s.nq + kRows - 1) / kRows : seq_size<kRows, kTile>(s);
      });
  if (descends<kThreads>(down)) return;
  int at = w * mine.per;
  if (at >= mine.total) return;
  int end = min(at + mine.per, mine.total), first = mine.first;
  int b = mine.unit;
  Seq s = seq_of(a, b);
  int blk;
  if (a.block_groups) {
    blk = at - first;
    at = first = 0;
    end = block_tiles<kRows, kTile>(s, blk);
  } else {
    blk = block_of<kRows, kTile>(s, at - first);
    first += size_before<kRows, kTile>(s, blk);
  }

  // The lane's number, made where it is used: what is computed from threadIdx.x ahead of the
  // loop is kept in registers over it.
  auto lane_now = [] {
    int l;
    asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(l));
    return l;
  };
  // Where in a window of eight keys the 16 bytes `c` of key `key` lie: the sixteen lanes that an
  // LDS read serves at once, of eight even (or odd) keys and two neighbouring chunks, differ in
  // their place in 256 bytes, as do those of a transposing read.
  auto spot = [](int key, int c) {
    return (key >> 1 & 3) * 256 + ((((key & 1) << 3 | c) ^ ((key & 6) | (key >> 3 & 1) * 9)) << 4);
  };
  const int k_row = (int)a.k_stride * 2, v_row = (int)a.v_stride * 2, r_row = (int)a.r_stride * 2;
  int k_off, v_off, r_off;  // of what a lane brings of a window: its 16 bytes of eight keys' 128
  {
    const int l = lane_now(), hc = (l & 15) ^ ((l >> 4) * 2 | (wave & 1) * 9);
    const int key = wave * 8 + (l >> 4) * 2 + (hc >> 3), in = (hc & 7) << 4;
    k_off = key * k_row + in;
    v_off = key * v_row + in;
    r_off = key * r_row + in;
  }
  const int l0 = lane_now(), c16 = l0 & 15, q4 = l0 >> 4;
  // Where in a stage the lane reads keys' chunks (key_of even: 8 (c16 / 4) + 2 (c16 % 4); steps
  // of the first product two to a window, ^ 64) and, transposed, values.
  const int k_at = (c16 >> 2) * GK + spot(8 * (c16 >> 2) + 2 * (c16 & 3), q4);
  const int r_at = K + (c16 >> 2) * 1024 + spot(8 * (c16 >> 2) + 2 * (c16 & 3), q4);
  const int v_at = K + ROPE + q4 * GK + spot(8 * q4 + 2 * (c16 >> 2), (c16 & 3) >> 1) + ((c16 & 1) << 3);
  const bf16x8 ones = __builtin_bit_cast(
      bf16x8, u16x8{0x3F80, 0x3F80, 0x3F80, 0x3F80, 0x3F80, 0x3F80, 0x3F80, 0x3F80});

  for (; at < end; ++blk) {
    if (blk * kRows >= s.nq) {
      if (++b >= a.n_seqs) break;
      s = seq_of(a, b);
      blk = -1;
      continue;
    }
    const int tiles = block_tiles<kRows, kTile>(s, blk);
    const int body = first + (a.block_groups ? 0 : kHead);  // where its tiles begin
    first = body + tiles;
    const int p_begin = max(at - body, 0), p_end = min(tiles, end - body);
    at = min(first, end);
    if (p_end <= p_begin) continue;  // no tile of it
    const int base_lim = s.nk - s.nq + 1;  // keys that row 0 of the sequence sees
    const int row0 = blk * kRows + wave * 32;
    const int min_lim = base_lim + row0;   // keys that every row of the wave sees

    // The tile to be brought next: its place, and the keys from there on.
    uint64_t k_next, v_next, r_next;
    int t_next = p_begin, n_next = s.nk - p_begin * kTile;
    {
      const int64_t k = (int64_t)s.k0 + p_begin * kTile;
      k_next = (uint64_t)(a.k + k * a.k_stride + h * a.k_head);
      v_next = (uint64_t)(a.v + k * a.v_stride + h * a.v_head);
      r_next = (uint64_t)(a.rope_keys + k * a.r_stride);
    }
    auto issue = [&](int st) {  // loads of the tiles behind the piece bring nothing, and count
      int kn = 31 * k_row + DIM * 2, vn = 31 * v_row + DIM * 2, rn = 31 * r_row + kRope * 2;
      if (t_next >= p_end || n_next < kTile) {
        const int n = t_next < p_end ? n_next : 0;
        kn = n > 0 ? (n - 1) * k_row + DIM * 2 : 0;
        vn = n > 0 ? (n - 1) * v_row + DIM * 2 : 0;
        rn = n > 0 ? (n - 1) * r_row + kRope * 2 : 0;
      }
      const DmaBuffer kb = dma_buffer((const void*)k_next, kn);
      const DmaBuffer vb = dma_buffer((const void*)v_next, vn);
      const DmaBuffer rb = dma_buffer((const void*)r_next, rn);
      const uint32_t to = lds0 + st * STAGE + wave * GK;
      each<WIN>([&](auto i) { dma16_unseen<i * 128, i * 1024>(kb, k_off, 0, to); });
      dma16_unseen<0, K>(rb, r_off, 0, lds0 + st * STAGE + wave * 1024);
      each<WIN>([&](auto i) { dma16_unseen<i * 128, K + ROPE + i * 1024>(vb, v_off, 0, to); });
      ++t_next;
      n_next -= kTile;
      k_next += (int64_t)kTile * k_row;
      v_next += (int64_t)kTile * v_row;
      r_next += (int64_t)kTile * r_row;
    };

    wait_vmem<0>();
    __syncthreads();  // the piece before is done with LDS
    issue(0);
    bf16x8 qf[2][KC];
    int row_lim[2];
    {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int row = min(row0 + t * 16 + c16, s.nq - 1);  // rows past the last repeat it
        row_lim[t] = base_lim + row;
        const uint16_t* src = a.q + ((int64_t)s.q0 + row) * a.q_stride + h * a.q_head;
#pragma unroll
        for (int c = 0; c < KC; ++c) qf[t][c] = *(const bf16x8*)(src + c * 32 + q4 * 8);
      }
    }
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int c = 0; c < KC; ++c) asm volatile("" : "+v"(qf[t][c]));
#pragma unroll
    for (int i = 1; i < kStages - 1; ++i) issue(i);

    float m[2] = {-INFINITY, -INFINITY};
    f32x4 acc[2][DT], sum[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      sum[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int d = 0; d < DT; ++d) acc[t][d] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    int st = 0;
#pragma unroll 1
    for (int p = p_begin; p < p_end; ++p) {
      wait_vmem<(kStages - 2) * NL>();
      wg_barrier();  // this tile is here, and the one before has been used
      issue(st == 0 ? kStages - 1 : st - 1);
      const uint8_t* kt = lds + st * STAGE;
      const uint8_t* vt = kt + K + ROPE;
      st = st + 1 == kStages ? 0 : st + 1;
      const int key0 = p * kTile;
      if (key0 >= min_lim + 31 || row0 >= s.nq) continue;  // nothing that a row of the wave sees
      const bool cut = key0 + kTile > min_lim;

      // Score e of key tile k of this lane belongs to key 8 q4 + 2 e + k.
      f32x4 sc[2][2];
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int k = 0; k < 2; ++k) sc[t][k] = f32x4{0.f, 0.f, 0.f, 0.f};
      {
        constexpr int N = 2 * KC, D = 6;  // reads; of them under way
        bf16x8 x[D];
        auto read = [&](int n) {  // step n / 2 of key tile n % 2
          const int c = n >> 1, flip = (c & 1) << 6 ^ (n & 1) << 7;
          x[n % D] = *(const bf16x8*)(kt + (c < 2 * WIN ? (k_at ^ flip) + (c >> 1) * 1024 : r_at ^ flip));
        };
#pragma unroll
        for (int n = 0; n < D; ++n) read(n);
#pragma unroll
        for (int n = 0; n < N; ++n) {
#pragma unroll
          for (int t = 0; t < 2; ++t)
            sc[t][n & 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[n % D], qf[t][n >> 1],
                                                                   sc[t][n & 1], 0, 0, 0);
          if (n + D < N) read(n + D);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      // The values, transposed: even and odd keys of eight, as the weights are.
      bf16x8 v[DT];
      {
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          const uint8_t* even = kt + (d >> 2) * 1024 + (v_at ^ (d & 3) << 5);
          const uint8_t* odd = kt + (d >> 2) * 1024 + (v_at ^ ((d & 3) << 5 | 128));
          const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((PDEC_LDS s16x4*)even);
          const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((PDEC_LDS s16x4*)odd);
          v[d] = __builtin_bit_cast(
              bf16x8, s16x8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]});
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      if (cut)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          int lim = row_lim[t] - key0 - 8 * q4;
          asm volatile("" : "+v"(lim));  // compared here, not ahead of the branch
#pragma unroll
          for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (2 * e + k >= lim) sc[t][k][e] = -INFINITY;
        }
      float now[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        float top = max2(max2(sc[t][0][0], sc[t][0][1]), max2(sc[t][0][2], sc[t][0][3]));
        top = max2(top, max2(max2(sc[t][1][0], sc[t][1][1]), max2(sc[t][1][2], sc[t][1][3])));
        now[t] = max_over_key_groups(top) * a.scale_log2;
      }
      if (__any(!(now[0] <= m[0] + kSlack) || !(now[1] <= m[1] + kSlack))) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const bool need = now[t] > m[t] + kSlack;
          const float to = need ? now[t] : m[t];
          const float alpha = need ? __builtin_amdgcn_exp2f(m[t] - to) : 1.f;
          m[t] = to;
          sum[t] *= alpha;
#pragma unroll
          for (int d = 0; d < DT; ++d) acc[t][d] *= alpha;
        }
      }
      // The weights enter the second product in bf16, each off by at most half a step (2^-8);
      // the normaliser sums them as they were rounded.
      bf16x8 pf[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const float base = m[t] == -INFINITY ? 0.f : m[t];
        uint32_t pw[4];
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
          const f32x2 x = {
              __builtin_amdgcn_exp2f(__builtin_fmaf(sc[t][e >> 2][e & 3], a.scale_log2, -base)),
              __builtin_amdgcn_exp2f(__builtin_fmaf(sc[t][e >> 2][(e & 3) + 1], a.scale_log2, -base))};
          pw[e / 2] = __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2));
        }
        pf[t] = __builtin_bit_cast(bf16x8, u32x4{pw[0], pw[1], pw[2], pw[3]});
        sum[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pf[t], sum[t], 0, 0, 0);
      }
      // 0 times what a row does not see is 0, unless something there is infinite or NaN: such
      // tiles are summed key by key, of the rows that see them alone, and their values made 0.
      if (cut) {
        f32x4 z = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int d = 0; d < DT; ++d)
          z = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[d], bf16x8{}, z, 0, 0, 0);
        if (__any(z[0] + z[1] + z[2] + z[3] != 0.f)) {
          uint8_t* mine = weights[wave];
#pragma unroll
          for (int t = 0; t < 2; ++t)
            *(bf16x8*)(mine + (t * 16 + c16) * 64 + q4 * 16) = pf[t];
#pragma unroll 1
          for (int key = 0; key < kTile; ++key) {
            const int l1 = lane_now(), c16 = l1 & 15, q4 = l1 >> 4;
            const uint8_t* from = mine + c16 * 64 + (key >> 3) * 16 + ((key & 1) * 4 + (key >> 1 & 3)) * 2;
            const float w0 = bf16_to_f32(*(const uint16_t*)from);
            const float w1 = bf16_to_f32(*(const uint16_t*)(from + 16 * 64));
            const bool s0 = key0 + key < row_lim[0], s1 = key0 + key < row_lim[1];
#pragma unroll
            for (int d = 0; d < DT; ++d) {
              const u32x2 x = *(const u32x2*)(vt + (key >> 3) * GK + (d >> 2) * 1024 +
                                              spot(key, (d & 3) * 2 + (q4 >> 1)) + (q4 & 1) * 8);
              const f32x4 y = {__uint_as_float(x.x << 16), __uint_as_float(x.x & 0xFFFF0000u),
                               __uint_as_float(x.y << 16), __uint_as_float(x.y & 0xFFFF0000u)};
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                if (s0) acc[0][d][i] = __builtin_fmaf(w0, y[i], acc[0][d][i]);
                if (s1) acc[1][d][i] = __builtin_fmaf(w1, y[i], acc[1][d][i]);
              }
              __builtin_amdgcn_sched_barrier(0);
            }
          }
#pragma unroll
          for (int d = 0; d < DT; ++d) v[d] = bf16x8{};
        }
      }
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int t = 0; t < 2; ++t)
          acc[t][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[d], pf[t], acc[t][d], 0, 0, 0);
    }

    const bool whole = p_begin == 0 && p_end == tiles;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int row = row0 + t * 16 + c16;
      if (row >= s.nq) continue;
      const float l = sum[t][0];
      if (whole) {
        const float inv = l == 0.f ? 0.f : 1.f / l;
        uint16_t* o = a.out + (((int64_t)s.q0 + row) * a.n_heads + h) * DIM + 4 * q4;
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          const f32x2 lo = {acc[t][d][0] * inv, acc[t][d][1] * inv};
          const f32x2 hi = {acc[t][d][2] * inv, acc[t][d][3] * inv};
          *(u32x2*)(o + d * 16) =
              u32x2{__builtin_bit_cast(uint32_t, __builtin_convertvector(lo, bf16x2)),
                    __builtin_bit_cast(uint32_t, __builtin_convertvector(hi, bf16x2))};
        }
      } else {
        // The group's first piece, or the one that begins in it and goes on.
        const int64_t pr = (((int64_t)w * 2 + (body + p_begin != w * mine.per)) * a.n_heads + h) * kRows +
                           row - blk * kRows;
        if (q4 == 0) *(float2*)(a.part_ml + pr * 2) = float2{m[t], l};
        float* o = a.part_acc + pr * DIM + 4 * q4;
#pragma unroll
        for (int d = 0; d < DT; ++d) *(f32x4*)(o + d * 16) = acc[t][d];
      }
    }
  }
  wait_vmem<0>();  // no LDS write may still be in flight when the group ends
}

// Merges the block that ends in stretch w and began before it, if there is one: its pieces are
// the first of w and of the stretches before, and where it began the last.  A group per
// (stretch, head, 32 rows): DIM / 4 lanes a row.
template <int DIM>
__global__ __launch_bounds__(512) void prompt_merge_kernel(LatentPromptArgs a, int n_groups) {
  constexpr int L = DIM / 4, RB = 512 / L;  // rows at once
  __shared__ int red[8];
  __shared__ int found[2];
  const int w = blockIdx.z, h = blockIdx.x;
  __shared__ int down[8];
  if ((threadIdx.x & 63) == 0) down[threadIdx.x >> 6] = 0;
  const Stretch mine = stretch_of<512>(a.n_seqs, n_groups, a.min_tiles, w, red, found, [&](int b) {
    note_descent(a, b, down);
    return seq_size<kRows, kTile>(seq_of(a, b));
  });
  if (descends<512>(down)) return;
  const int at = w * mine.per;
  if (at >= mine.total) return;
  const int end = min(at + mine.per, mine.total);
  const Seq s = seq_of(a, mine.unit);
  const int blk = block_of<kRows, kTile>(s, at - mine.first);
  const int body = mine.first + size_before<kRows, kTile>(s, blk) + kHead;
  const int tiles = block_tiles<kRows, kTile>(s, blk);
  if (blk * kRows >= s.nq || body >= at || body + tiles > end) return;
  const int lane = threadIdx.x % L, w0 = body / mine.per;
  const int row_end = min(kRows, s.nq - blk * kRows);
  for (int row = blockIdx.y * RB + threadIdx.x / L; row < row_end; row += gridDim.y * RB) {
    float m = -INFINITY, l = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    for (int v = w0; v <= w; v += 8) {
      float2 ml[8];
      f32x4 x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (v + i <= w) {
          const int g = v + i;
          const int64_t pr =
              (((int64_t)g * 2 + (g == w0 && body != w0 * mine.per)) * a.n_heads + h) * kRows + row;
          ml[i] = *(const float2*)(a.part_ml + pr * 2);
          x[i] = *(const f32x4*)(a.part_acc + pr * DIM + lane * 4);
        }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (v + i > w) continue;
        const float mn = fmaxf(m, ml[i].x), mu = mn == -INFINITY ? 0.f : mn;
        const float so = exp2f(m - mu), si = exp2f(ml[i].x - mu);
        l = l * so + ml[i].y * si;
        o = o * so + x[i] * si;
        m = mn;
      }
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const f32x2 lo = {o[0] * inv, o[1] * inv}, hi = {o[2] * inv, o[3] * inv};
    *(u32x2*)(a.out + (((int64_t)s.q0 + blk * kRows + row) * a.n_heads + h) * DIM + lane * 4) =
        u32x2{__builtin_bit_cast(uint32_t, __builtin_convertvector(lo, bf16x2)),
              __builtin_bit_cast(uint32_t, __builtin_convertvector(hi, bf16x2))};
  }
}

}  // namespace

hipError_t launch_latent_prompt(int dim, int n_groups, const LatentPromptArgs& a,
                                hipStream_t stream) {
  const dim3 grid(a.n_heads, n_groups);
#define PDEC_PROMPT(D_)                                                                 \
  do {                                                                                  \
    prompt_attn_kernel<D_><<<grid, kThreads, 0, stream>>>(a);                           \
    hipError_t e = hipGetLastError();                                                   \
    if (e != hipSuccess || a.block_groups || n_groups == 1) return e;                   \
    const dim3 mgrid(a.n_heads, 2, n_groups);                                           \
    prompt_merge_kernel<D_><<<mgrid, 512, 0, stream>>>(a, n_groups);                    \
  } while (0)
  if (dim == 128) PDEC_PROMPT(128);
  else PDEC_PROMPT(64);
#undef PDEC_PROMPT
  return hipGetLastError();
}

}  // namespace pdec
