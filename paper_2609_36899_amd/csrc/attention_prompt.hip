// Attention of prompts over keys and values expanded from latents: for each head keys of DIM
// elements beside the rotary key that all heads share, and values of DIM.
//
//   out[i][h] = softmax(scale * (q[i][h][:DIM] . k[j][h] + q[i][h][DIM:] . rope_keys[j])) v[j][h]
//   over the keys j of i's sequence up to i's own: the last of its n_keys belong to its n_rows.
//
// Bound by the matrix units: 2 (2 DIM + 64) operations a pair of row and key.  A work group
// takes a block of rows of one head, 32 a wave, over tiles of keys that come into LDS by DMA,
// a ring of three.  S^T = K Q^T, with the keys of a block of 32 dealt to two MFMA tiles, even
// and odd ones, so that a lane's eight weights are the operand P of O^T = V^T P^T as they are,
// against V transposed by the LDS read (ds_read_tr).  Each 16-byte chunk n of a row lies in
// place n ^ f of its 128 bytes, f from the key: eight lanes that read eight keys' chunk n, and
// the sixteen of a transposing read (four keys, two chunks), meet different banks.
//
// Work split.  Per head the blocks' tiles laid end to end are cut into n_groups equal stretches
// (stretch.h), found from the sequences' starts on the device.  A stretch's first piece, where
// its block began before, and its last, where it goes on behind, leave partials; the merge pass
// joins each block that was cut.  Where there are enough blocks each has a group of its own.
#include "hip_common.h"
#include "kernels.h"
#include "stretch.h"

#include <algorithm>

namespace pdec {

namespace {

constexpr int kRope = kLatentRope;
constexpr float kSlack = 16.f;  // powers of two that scores may outgrow a row's reference by

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
#define PDEC_LDS __attribute__((address_space(3)))

// A sequence's rows and keys; starts are not trusted.
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
// Tiles of block blk: those of the keys that its last row sees, at least one.
template <int ROWS, int TILE>
__device__ __forceinline__ int block_tiles(const Seq& s, int blk) {
  const int keys = s.nk - s.nq + min((blk + 1) * ROWS, s.nq);
  return max((keys + TILE - 1) / TILE, 1);
}
template <int ROWS, int TILE>
__device__ __forceinline__ int seq_tiles(const Seq& s) {
  int n = 0;
  for (int blk = 0; blk * ROWS < s.nq; ++blk) n += block_tiles<ROWS, TILE>(s, blk);
  return n;
}

template <int DIM, int WAVES>
struct PromptForm {
  static constexpr int kRows = 32 * WAVES, kTile = WAVES == 8 ? 64 : 32, kStages = 3;
  static constexpr int kK = kTile * DIM * 2, kR = kTile * kRope * 2;  // bytes of K, and V; of rotary
  static constexpr int kStage = 2 * kK + kR;
};

template <int DIM, int WAVES>
__global__ __launch_bounds__(64 * WAVES) __attribute__((amdgpu_waves_per_eu(2))) void
prompt_attn_kernel(LatentPromptArgs a) {
  typedef PromptForm<DIM, WAVES> F;
  constexpr int TILE = F::kTile, NST = F::kStages, ROWS = F::kRows, THREADS = 64 * WAVES;
  constexpr int KN = DIM / 32, KC = KN + 2, DT = DIM / 16, KT = TILE / 16;
  constexpr int NK = F::kK / 1024 / WAVES, NR = F::kR / 1024 / WAVES, NL = 2 * NK + NR;
  static_assert(NK * 1024 * WAVES == F::kK && NR * 1024 * WAVES == F::kR, "whole loads");
  __shared__ __attribute__((aligned(128))) uint8_t lds[NST * F::kStage];
  __shared__ int red[WAVES];
  __shared__ int found[2];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int c16 = lane & 15, q4 = lane >> 4, h = blockIdx.x;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(PDEC_LDS uint8_t*)lds;
  // With a group for each block the blocks' order is turned round, so that the long ones begin
  // first.
  const int w = a.block_groups ? gridDim.y - 1 - blockIdx.y : blockIdx.y;
  const Stretch mine = stretch_of<THREADS>(
      a.n_seqs, gridDim.y, a.block_groups ? 1 : a.min_tiles, w, red, found, [&](int b) {
        const Seq s = seq_of(a, b);
        return a.block_groups ? (s.nq + ROWS - 1) / ROWS : seq_tiles<ROWS, TILE>(s);
      });
  int at = w * mine.per;
  if (at >= mine.total) return;
  int end = min(at + mine.per, mine.total), first = mine.first, blk = 0;
  int b = min(max(mine.unit, 0), a.n_seqs - 1);  // whatever the starts hold
  Seq s = seq_of(a, b);
  if (a.block_groups) {
    blk = at - first;
    at = first = 0;
    end = block_tiles<ROWS, TILE>(s, blk);
  }

  auto f_of = [](int key) { return (key & 6) | (key >> 3 & 1); };  // the key's place in 128 bytes
  int k_off[NK], v_off[NK], r_off[NR];
  const int k_row = (int)a.k_stride * 2, v_row = (int)a.v_stride * 2, r_row = (int)a.r_stride * 2;
#pragma unroll
  for (int i = 0; i < NK; ++i) {
    const int n = (wave * NK + i) * 64 + lane, key = n / (DIM / 8), c = n % (DIM / 8) ^ f_of(key);
    k_off[i] = key * k_row + c * 16;
    v_off[i] = key * v_row + c * 16;
  }
#pragma unroll
  for (int i = 0; i < NR; ++i) {
    const int n = (wave * NR + i) * 64 + lane, key = n / 8;
    r_off[i] = key * r_row + ((n % 8) ^ f_of(key)) * 16;
  }
  const int key_a = 8 * (c16 >> 2) + 2 * (c16 & 3);  // this lane's even key of a block of 32
  const int k_sw = (q4 ^ f_of(key_a)) << 4;
  const int v_key = 8 * q4 + 2 * (c16 >> 2);
  const int v_base = v_key * (DIM * 2) + ((((c16 & 3) >> 1) ^ f_of(v_key)) << 4) + ((c16 & 1) << 3);
  const bf16x8 ones = __builtin_bit_cast(
      bf16x8, u16x8{0x3F80, 0x3F80, 0x3F80, 0x3F80, 0x3F80, 0x3F80, 0x3F80, 0x3F80});

  for (; at < end; ++blk) {
    if (blk * ROWS >= s.nq) {
      if (++b >= a.n_seqs) break;
      s = seq_of(a, b);
      blk = -1;
      continue;
    }
    const int tiles = block_tiles<ROWS, TILE>(s, blk);
    if (first + tiles <= at) {
      first += tiles;
      continue;
    }
    const int p_begin = max(at - first, 0), p_end = min(tiles, end - first);
    const int base_lim = s.nk - s.nq + 1;  // keys that row 0 of the sequence sees
    const int row0 = blk * ROWS + wave * 32;
    const int min_lim = base_lim + row0;   // keys that every row of the wave sees

    auto issue = [&](int t, int st) {
      const int key0 = t * TILE, n = t < p_end ? min(s.nk - key0, TILE) : 0;
      const int64_t k = (int64_t)s.k0 + (n > 0 ? key0 : 0);
      const uint32_t to = lds0 + st * F::kStage;
      const DmaBuffer kb = dma_buffer(a.k + k * a.k_stride + h * a.k_head,
                                n > 0 ? (n - 1) * k_row + DIM * 2 : 0);
      const DmaBuffer vb = dma_buffer(a.v + k * a.v_stride + h * a.v_head,
                                n > 0 ? (n - 1) * v_row + DIM * 2 : 0);
      const DmaBuffer rb = dma_buffer(a.rope_keys + k * a.r_stride,
                                n > 0 ? (n - 1) * r_row + kRope * 2 : 0);
#pragma unroll
      for (int i = 0; i < NK; ++i) dma16_unseen(kb, k_off[i], 0, to + (wave * NK + i) * 1024);
#pragma unroll
      for (int i = 0; i < NR; ++i)
        dma16_unseen(rb, r_off[i], 0, to + F::kK + (wave * NR + i) * 1024);
#pragma unroll
      for (int i = 0; i < NK; ++i)
        dma16_unseen(vb, v_off[i], 0, to + F::kK + F::kR + (wave * NK + i) * 1024);
    };

    wait_vmem<0>();
    __syncthreads();  // the piece before is done with LDS
    issue(p_begin, 0);
    bf16x8 qf[2][KC];
    int row_lim[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int row = min(row0 + t * 16 + c16, s.nq - 1);  // rows past the last repeat it
      row_lim[t] = base_lim + row;
      const uint16_t* src = a.q + ((int64_t)s.q0 + row) * a.q_stride + h * a.q_head;
#pragma unroll
      for (int c = 0; c < KC; ++c) qf[t][c] = *(const bf16x8*)(src + c * 32 + q4 * 8);
    }
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int c = 0; c < KC; ++c) asm volatile("" : "+v"(qf[t][c]));
#pragma unroll
    for (int i = 1; i < NST - 1; ++i) issue(p_begin + i, i);

    float m[2] = {-INFINITY, -INFINITY};
    f32x4 acc[2][DT], sum[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      sum[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int d = 0; d < DT; ++d) acc[t][d] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    int st = 0;
    for (int p = p_begin; p < p_end; ++p) {
      wait_vmem<(NST - 2) * NL>();
      wg_barrier();  // this tile is here, and the one before has been used
      issue(p + NST - 1, st == 0 ? NST - 1 : st - 1);
      const uint8_t* kt = lds + st * F::kStage;
      const uint8_t* rt = kt + F::kK;
      const uint8_t* vt = rt + F::kR;
      st = st + 1 == NST ? 0 : st + 1;
      const int key0 = p * TILE;
      if (key0 >= min_lim + 31 || row0 >= s.nq) continue;  // nothing that a row of the wave sees
      const bool cut = key0 + TILE > min_lim;

      // Score e of key tile k of this lane belongs to key 32 (k / 2) + 8 q4 + 2 e + k % 2.
      f32x4 sc[2][KT];
#pragma unroll
      for (int k = 0; k < KT; ++k) {
        const int key = (k >> 1) * 32 + key_a + (k & 1);
#pragma unroll
        for (int t = 0; t < 2; ++t) sc[t][k] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < KC; ++c) {
          const uint8_t* row = c < KN ? kt + key * (DIM * 2) + (c >> 1) * 128 : rt + key * (kRope * 2);
          const bf16x8 x = *(const bf16x8*)(row + (k_sw ^ (c & 1) << 6));
#pragma unroll
          for (int t = 0; t < 2; ++t)
            sc[t][k] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, qf[t][c], sc[t][k], 0, 0, 0);
        }
      }
      uint32_t pw[2][KT][2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        float top = -INFINITY;
#pragma unroll
        for (int k = 0; k < KT; ++k)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if (cut && key0 + (k >> 1) * 32 + 8 * q4 + 2 * e + (k & 1) >= row_lim[t])
              sc[t][k][e] = -INFINITY;
            top = fmaxf(top, sc[t][k][e]);
          }
        const float now = max_over_key_groups(top) * a.scale_log2;
        const bool need = now > m[t] + kSlack;
        if (__any(need)) {
          const float to = need ? now : m[t];
          const float alpha = need ? __builtin_amdgcn_exp2f(m[t] - to) : 1.f;
          m[t] = to;
          sum[t] *= alpha;
#pragma unroll
          for (int d = 0; d < DT; ++d) acc[t][d] *= alpha;
        }
        // The weights enter the second product in bf16, each off by at most half a step (2^-8);
        // the normaliser sums them as they were rounded.
        const float base = m[t] == -INFINITY ? 0.f : m[t];
#pragma unroll
        for (int k = 0; k < KT; ++k)
#pragma unroll
          for (int e = 0; e < 4; e += 2) {
            const f32x2 x = {
                __builtin_amdgcn_exp2f(__builtin_fmaf(sc[t][k][e], a.scale_log2, -base)),
                __builtin_amdgcn_exp2f(__builtin_fmaf(sc[t][k][e + 1], a.scale_log2, -base))};
            pw[t][k][e / 2] = __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2));
          }
      }
#pragma unroll
      for (int kb = 0; kb < TILE / 32; ++kb) {
        bf16x8 pf[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          pf[t] = __builtin_bit_cast(bf16x8, u32x4{pw[t][2 * kb][0], pw[t][2 * kb][1],
                                                   pw[t][2 * kb + 1][0], pw[t][2 * kb + 1][1]});
          sum[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pf[t], sum[t], 0, 0, 0);
        }
        auto value = [&](int d) {
          const int at = (v_base ^ ((d & 3) << 5)) + (d >> 2) * 128 + kb * 32 * DIM * 2;
          const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((PDEC_LDS s16x4*)(vt + at));
          const s16x4 hi =
              __builtin_amdgcn_ds_read_tr16_b64_v4i16((PDEC_LDS s16x4*)(vt + at + DIM * 2));
          return __builtin_bit_cast(
              bf16x8, s16x8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]});
        };
        // 0 times what a row does not see is 0, unless something there is infinite or NaN:
        // such blocks of 32 keys are summed key by key, of the rows that see them alone.
        bool finite = true;
        if (cut) {
          f32x4 z = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int d = 0; d < DT; ++d)
            z = __builtin_amdgcn_mfma_f32_16x16x32_bf16(value(d), bf16x8{}, z, 0, 0, 0);
          finite = !__any(z[0] + z[1] + z[2] + z[3] != 0.f);
        }
        if (finite) {
#pragma unroll
          for (int d = 0; d < DT; ++d) {
            const bf16x8 v = value(d);
#pragma unroll
            for (int t = 0; t < 2; ++t)
              acc[t][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, pf[t], acc[t][d], 0, 0, 0);
          }
        } else {
          for (int g = 0; g < 4; ++g)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const int key = kb * 32 + 8 * g + 2 * (e & 3) + (e >> 2);
              float pv[2];
#pragma unroll
              for (int t = 0; t < 2; ++t) {
                const uint32_t pair = pw[t][2 * kb + (e >> 2)][(e & 3) / 2];
                pv[t] = __shfl(__uint_as_float(e & 1 ? pair & 0xFFFF0000u : pair << 16), g * 16 + c16, 64);
              }
#pragma unroll
              for (int d = 0; d < DT; ++d) {
                const int dim = d * 16 + 4 * q4;
                const u32x2 x = *(const u32x2*)(vt + key * (DIM * 2) + ((dim >> 3 ^ f_of(key)) << 4) +
                                                (dim & 7) * 2);
                const f32x4 v = {__uint_as_float(x.x << 16), __uint_as_float(x.x & 0xFFFF0000u),
                                 __uint_as_float(x.y << 16), __uint_as_float(x.y & 0xFFFF0000u)};
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                  for (int i = 0; i < 4; ++i)
                    acc[t][d][i] = key0 + key < row_lim[t]
                                       ? __builtin_fmaf(pv[t], v[i], acc[t][d][i])
                                       : acc[t][d][i];
              }
            }
        }
      }
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
        const int64_t pr = (((int64_t)w * 2 + (first + p_begin != w * mine.per)) * a.n_heads + h) * ROWS +
                           row - blk * ROWS;
        if (q4 == 0) *(float2*)(a.part_ml + pr * 2) = float2{m[t], l};
        float* o = a.part_acc + pr * DIM + 4 * q4;
#pragma unroll
        for (int d = 0; d < DT; ++d) *(f32x4*)(o + d * 16) = acc[t][d];
      }
    }
    at = first + p_end;
    first += tiles;
  }
  wait_vmem<0>();  // no LDS write may still be in flight when the group ends
}

// Merges the block that ends in stretch w and began before it, if there is one: its pieces are
// the first of w and of the stretches before, and where it began the last.  A group per
// (stretch, head, 32 rows): DIM / 4 lanes a row.
template <int DIM, int WAVES>
__global__ __launch_bounds__(512) void prompt_merge_kernel(LatentPromptArgs a, int n_groups) {
  constexpr int ROWS = 32 * WAVES, TILE = PromptForm<DIM, WAVES>::kTile;
  constexpr int L = DIM / 4, RB = 512 / L;  // rows at once
  __shared__ int red[8];
  __shared__ int found[2];
  const int w = blockIdx.y, h = blockIdx.x;
  const Stretch mine = stretch_of<512>(a.n_seqs, n_groups, a.min_tiles, w, red, found, [&](int b) {
    return seq_tiles<ROWS, TILE>(seq_of(a, b));
  });
  const int at = w * mine.per;
  if (at >= mine.total) return;
  const int end = min(at + mine.per, mine.total);
  const Seq s = seq_of(a, min(max(mine.unit, 0), a.n_seqs - 1));
  int blk = 0, first = mine.first, tiles = 0;
  for (; blk * ROWS < s.nq; ++blk) {
    tiles = block_tiles<ROWS, TILE>(s, blk);
    if (first + tiles > at) break;
    first += tiles;
  }
  if (blk * ROWS >= s.nq || first < 0 || first >= at || first + tiles > end) return;
  const int row = blockIdx.z * RB + threadIdx.x / L, lane = threadIdx.x % L;
  if (blk * ROWS + row >= s.nq || row >= ROWS) return;
  const int w0 = first / mine.per;
  float m = -INFINITY, l = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int v = w0; v <= w; v += 8) {
    float2 ml[8];
    f32x4 x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int g = min(v + i, w);
      const int64_t pr =
          (((int64_t)g * 2 + (g == w0 && first != w0 * mine.per)) * a.n_heads + h) * ROWS + row;
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
  *(u32x2*)(a.out + (((int64_t)s.q0 + blk * ROWS + row) * a.n_heads + h) * DIM + lane * 4) =
      u32x2{__builtin_bit_cast(uint32_t, __builtin_convertvector(lo, bf16x2)),
            __builtin_bit_cast(uint32_t, __builtin_convertvector(hi, bf16x2))};
}

}  // namespace

hipError_t launch_latent_prompt(int dim, int waves, int n_groups, const LatentPromptArgs& a,
                                hipStream_t stream) {
  const dim3 grid(a.n_heads, n_groups);
#define PDEC_PROMPT(D_, W_)                                                                   \
  do {                                                                                        \
    prompt_attn_kernel<D_, W_><<<grid, 64 * W_, 0, stream>>>(a);                              \
    hipError_t e = hipGetLastError();                                                         \
    if (e != hipSuccess || a.block_groups || n_groups == 1) return e;                         \
    const dim3 mgrid(a.n_heads, n_groups, 32 * W_ * D_ / 4 / 512);                            \
    prompt_merge_kernel<D_, W_><<<mgrid, 512, 0, stream>>>(a, n_groups);                      \
  } while (0)
  if (dim == 128) {
    if (waves == 8) PDEC_PROMPT(128, 8);
    else PDEC_PROMPT(128, 4);
  } else {
    if (waves == 8) PDEC_PROMPT(64, 8);
    else PDEC_PROMPT(64, 4);
  }
#undef PDEC_PROMPT
  return hipGetLastError();
}

}  // namespace pdec
