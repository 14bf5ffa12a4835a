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
// more.  Units of at most 16 rows are attention_latent_few.hip's.
//
// Work split.  The units' tiles laid end to end are cut into n_groups equal stretches, one for
// each work group, found from the lengths on the device (stretch.h).  The piece of unit u in
// group w leaves its softmax partial in slot w + u; the merge pass joins a unit's pieces.  A
// unit that one group covers whole is written out at once, and where there are many units, or
// none can be long, each has a group of its own.
//
// One step.  S^T = K Q^T of tile p, a wave a row tile, whose weights P go through LDS; beside
// it the second product of tile p - 1, by every wave for its eighth of the latent's width: O^T =
// C^T P^T.  So O takes 16 registers a row tile instead of 128, and each latent is read from LDS
// once in the second product, transposed by the read itself (ds_read_tr).  Neither product of a
// step needs the other's: half the waves take one first, half the other, and one barrier a step
// serves both.  E4M3 codes enter the first product as they are, against queries split in two;
// the second takes them decoded to bf16.
//
// The tiles come by LDS-DMA into a ring of three stages, by the four waves that wait at the
// barrier otherwise (all eight: 189 against 182 us).  Nothing is spilled in the loop: a reload
// would wait, as loads return in order, for the tile on its way (128 heads 584 us with spills,
// 192 without).  128 heads over 64 x 1K to 8K bf16 124 us (0.71 PFLOP/s; of it the pieces'
// beginnings and ends 18 and the merge 20), 32 heads x 4 tokens over 8 x 64K to 128K E4M3 220
// (0.97).  Tried without gain: loads one by one between the products (142), weights read two or
// three tiles ahead, a higher priority for either half of the waves.
#include "latent_attn.h"

#include <algorithm>
#include <type_traits>

namespace pdec {

namespace {

constexpr int kThreads = 512, kWaves = kThreads / 64;

template <int R, int RT, bool FP8>
struct Form {
  static constexpr int kRow = FP8 ? R + 2 * kRope : (R + kRope) * 2;  // a key's bytes
  static constexpr int kTile = latent_tile(FP8, R);
  // Two tiles are in use, the others on their way.  More stages do not fit beside the weights.
  static constexpr int kStages = 3;
  static constexpr int kStage = kTile * kRow;
  static constexpr int kRows = 16 * RT;
  // LDS offsets.
  static constexpr int kWeights = kRows * kTile * 2;          // [kRows][kTile] bf16
  static constexpr int kP = kStages * kStage;                 // [2]
  static constexpr int kScale = kP + 2 * kWeights;            // [kStages][kTile]
  static constexpr int kAlpha = kScale + (FP8 ? kStages * kTile * 4 : 0);  // [2][kRows]
  static constexpr int kLim = kAlpha + 2 * kRows * 4;         // [kRows]: keys that a row sees
  static constexpr int kFlag = kLim + kRows * 4;              // [2][8] bytes: rows whose O moves
  static constexpr int kIds = kFlag + 16;                     // [64]
  static constexpr int kBytes = kIds + 256;
  static_assert(kBytes <= 160 * 1024 - 64 && kRow % 128 == 0 && kStage % 256 == 0, "LDS layout");
};

template <int R, int RT, bool FP8>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2))) void
latent_attn_kernel(LatentAttnArgs a) {
  typedef Form<R, RT, FP8> F;
  constexpr int TILE = F::kTile, NST = F::kStages, ROW = F::kRow, PPT = TILE / kPage;
  constexpr int NB = TILE / 32;                      // blocks of 32 keys
  constexpr int DT = R / 16 / kWaves, DW = R / kWaves;  // 16-wide tiles of a wave's part of R
  constexpr int WIN = ROW / 128, LW = (FP8 ? R : 2 * R) / 128;  // a row's windows; its latent's
  constexpr int GROUP = 8 * ROW;                     // bytes of eight keys
  // Loads of a wave: the windows of eight keys, or where a tile is four such groups half of them.
  constexpr int NW = TILE == 64 ? WIN : (WIN + 1) / 2;
  __shared__ __attribute__((aligned(256))) uint8_t lds[F::kBytes];
  __shared__ int red[kWaves];
  __shared__ int found[2];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), w = blockIdx.x;
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
                                              [&](int v) { return unit_size<TILE>(a, v); });
    at = w * mine.per;
    if (at >= mine.total) return;
    end = min(at + mine.per, mine.total);
    u = __builtin_amdgcn_readfirstlane(mine.unit);
    first = __builtin_amdgcn_readfirstlane(mine.first);
    at = __builtin_amdgcn_readfirstlane(at);
    end = __builtin_amdgcn_readfirstlane(end);
  }

  // Key numbers.  Score e of key tile t (of two) of a block of 32 keys belongs in lane (c, q) to
  // key_of(q, t, e), and the eight of a lane side by side are what the second product takes:
  // of bf16 pages t = 0 the four even keys of eight and t = 1 the odd ones, since a transposing
  // read brings four keys, which must differ in their place by more than one; of E4M3 pages,
  // where it brings eight, in order.
  auto key_of = [](int q, int t, int e) { return FP8 ? 8 * q + 4 * t + e : 8 * q + 2 * e + t; };
  // The position of a key's weight within its block, and where row `row`'s weights of block
  // `blk` lie: chunk c of 16 bytes, exchanged by the row.
  auto p_at = [](int row, int c) {
    if constexpr (TILE == 64) return row * 128 + ((c ^ (row & 7)) << 4);
    else return (row >> 1) * 128 + ((((row & 1) << 2) | (c ^ (row >> 1 & 3))) << 4);
  };

  for (; at < end; ++u) {
    const int tiles = unit_tiles<TILE>(a, u), size = unit_size<TILE>(a, u);
    const int body = first + size - tiles;  // where its tiles begin
    first += size;
    const int p_begin = max(at - body, 0), p_end = min(tiles, end - body);
    at = min(max(first, at), end);
    if (p_end <= p_begin) continue;  // an empty unit, or no tile of it
    const int b = u / a.blocks_per_seq, row0 = unit_row0(a, u), rows = unit_rows(a, row0);
    const int base_lim = clamp_len(a, b) - a.n_q + 1;  // keys that token 0 sees
    const int kv_lim = max(base_lim + (row0 + rows - 1) / a.n_heads, 0);
    const int min_lim = max(base_lim + row0 / a.n_heads, 0);  // keys that every row sees
    const int n_pages = (kv_lim + kPage - 1) / kPage;
    const int64_t q_row0 = (int64_t)b * a.n_q * a.n_heads + row0;

    // The ids of 64 pages from page0 on, in LDS (each wave puts the same there), and which of
    // them there are.
    int page0 = p_begin * PPT;
    uint64_t there;
    auto look = [&] {
      const int l = lane_now(), n = page0 + l;
      const int id = n < n_pages ? a.block_table[(int64_t)b * a.bt_stride + n] : -1;
      there = __ballot(id >= 0 && id < a.n_pages);
      *(int*)(lds + F::kIds + l * 4) = id;
    };
    // Which pages of the tiles in the stages are there, four bits a stage.
    uint32_t ok = 0;
    // A wave brings the windows of a group of eight keys, 128 bytes of each key a load.  A page
    // that is not there is not brought.
    auto push = [&](int t, int st) {
      if (t >= p_end) {
        ok &= ~(15u << (4 * st));
        return;
      }
      int i = t * PPT - page0;
      if (i >= 64) {
        page0 += 64;
        i -= 64;
        look();
      }
      ok = (ok & ~(15u << (4 * st))) | ((uint32_t)(there >> i) & ((1 << PPT) - 1)) << (4 * st);
      if ((wave < kWaves / 2) != (RT == 8)) return;
      const int l = lane_now();
#pragma unroll
      for (int h = 0; h < TILE / 32; ++h) {
        const int g = (wave & 3) + h * 4;
        if (!(there >> (i + (g >> 1)) & 1)) continue;
        const int64_t p =
            __builtin_amdgcn_readfirstlane(*(const int*)(lds + F::kIds + (i + (g >> 1)) * 4));
        const DmaBuffer src = dma_buffer((const uint8_t*)a.pages + p * (kPage * ROW), 2 * GROUP);
        const int voff = window_offset<FP8, ROW>(l, g);
        const uint32_t to = lds0 + st * F::kStage + g * GROUP;
        // A sequence's pages that one unit reads do not stay in the caches: from HBM 128 heads over
        // 64 x 1K to 8K bf16 130 us, then 127, 32 heads x 4 tokens over 8 x 64K to 128K E4M3 232 and
        // 225.  Forks share pages: 32 heads, bf16, so / kept there, eight forks each of eight
        // prompts of 4K 79 / 65, with 1K to 8K of their own behind 1K 103 / 109, 64 that share
        // nothing 84 / 90; E4M3 63 / 62, 73 / 74, 62 / 65; 128 heads alike within 4%.
        if (a.blocks_per_seq == 1)
          each<WIN>([&](auto n) {
            dma16_unseen<n * 128, n * 1024, true>(src, voff, (g & 1) * GROUP, to);
          });
        else
          each<WIN>([&](auto n) {
            dma16_unseen<n * 128, n * 1024>(src, voff, (g & 1) * GROUP, to);
          });
        if constexpr (FP8) {
          const DmaBuffer scales = dma_buffer(a.scales + p * kPage + (g & 1) * 8, 32);
          if (l < 8) dma4_unseen(scales, l * 4, lds0 + F::kScale + (st * TILE + g * 8) * 4);
        }
      }
    };

    wait_vmem<0>();
    __syncthreads();  // the piece before is done with LDS
    look();
    push(p_begin, 0);
    // This wave's row tile of the first product; a lane's query row c, dims by q.
    const int rq = wave < RT ? wave : 0;
    bf16x8 qr[2], qf[FP8 ? 1 : 2 * LW];
    i32x8 qh[LW], ql[LW];  // of E4M3 pages
    int q_exp = 0;
    {
      const int l0 = lane_now(), c16 = l0 & 15, q4 = l0 >> 4;
      const int row = min(rq * 16 + c16, rows - 1);  // rows past the block's repeat its last
      if (wave < RT && q4 == 0)  // the keys that a row sees
        *(int*)(lds + F::kLim + (rq * 16 + c16) * 4) = base_lim + (row0 + row) / a.n_heads;
      const uint16_t* src = (const uint16_t*)a.q + (q_row0 + row) * (R + kRope) + q4 * 8;
#pragma unroll
      for (int c = 0; c < 2; ++c) qr[c] = *(const bf16x8*)(src + R + c * 32);
      if constexpr (FP8) {
        bf16x8 x[4 * LW];
        read_query<LW>(src - q4 * 8, q4, x);
        __builtin_amdgcn_sched_barrier(0);  // all of them under way
        q_exp = split_query<LW>(x, qh, ql);
      } else {
#pragma unroll
        for (int c = 0; c < 2 * LW; ++c) qf[c] = *(const bf16x8*)(src + c * 32);
#pragma unroll
        for (int c = 0; c < 2 * LW; ++c) asm volatile("" : "+v"(qf[c]));
      }
    }
    // Here the queries are waited for, and the first tile with them; the next one's loads follow.
#pragma unroll
    for (int c = 0; c < 2; ++c) asm volatile("" : "+v"(qr[c]));

    float m = -INFINITY, l = 0.f;  // a reference for the row's scores; this lane's part of its sum
    f32x4 acc[RT][DT];
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
      for (int d = 0; d < DT; ++d) acc[t][d] = f32x4{0.f, 0.f, 0.f, 0.f};

    // Step p: the first product and the weights of tile p, the second product of tile p - 1.
    // Neither needs the other, so half the waves take one first, half the other, and one
    // barrier a step serves both.
    int st = 0, before = NST - 1;  // stages of tiles p and p - 1
    for (int p = p_begin; p <= p_end; ++p) {
      wait_vmem<0>();
      wg_barrier();  // tile p and the weights of p - 1 are here, and tile p - 2 has been used
      const int next = NST - st - before, buf = p & 1;
      push(p + 1, next);
#pragma unroll 1
      for (int half = 0; half < 2; ++half) {
        if ((half == 0) == (RT < 8 || wave >= kWaves / 2)) {
          // ---- scores and weights of tile p
          if (wave >= RT || p == p_end) continue;
          const int l1 = lane_now(), c16 = l1 & 15, q4 = l1 >> 4;
          const uint8_t* tile = lds + st * F::kStage;
          const int key0 = p * TILE;
          // Keys that some row does not see, or that are not there.
          const int here = ok >> (4 * st) & 15;
          const bool cut = key0 + TILE > min_lim || here != (1 << PPT) - 1;
          uint8_t* p_row = lds + F::kP + buf * F::kWeights;
          const int row = rq * 16 + c16;
          int moved = 0;
          float alpha = 1.f;
          // The row's reference follows a top that outgrows it by more than the slack.
          auto follow = [&](float top) {
            const float now = top * a.scale_log2;
            const bool need = now > m + kSlack, begun = m > -INFINITY;
            const float f = need && begun ? __builtin_amdgcn_exp2f(m - now) : 1.f;
            if (need) m = now;
            l *= f;
            alpha *= f;
            moved |= __any(need && begun);
          };
          // Where a row does not see a key its score is -inf, and the token's scale, which may
          // be anything, 0.
          auto mask = [&](int blk, int t, f32x4& x, f32x4& vs) {
            // Of bf16 pages eight keys of one page; of E4M3 pages too (8 q4 ..).
            int lim = *(const int*)(lds + F::kLim + row * 4) - key0 - blk * 32;
            if (!(here >> (blk * 2 + (q4 >> 1)) & 1)) lim = 0;
            asm volatile("" : "+v"(lim));  // compared here, not ahead of the branch
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (key_of(q4, t, e) >= lim) {
                x[e] = -INFINITY;
                vs[e] = 0.f;
              }
          };
          // Scores of a block, their top, and the tokens' scales.
          auto scores = [&](int blk, f32x4 (&x)[2], f32x4 (&vs)[2]) {
#pragma unroll
            for (int t = 0; t < 2; ++t) x[t] = f32x4{0.f, 0.f, 0.f, 0.f};
            // The lane's key of tile t, as a row of the product: key_of(c16 / 4, t, c16 % 4).
            const uint8_t* from = tile + (blk * 4 + (c16 >> 2)) * GROUP;
            if constexpr (FP8) {
              from += spot<FP8>(8 * (c16 >> 2) + (c16 & 3), 0) & ~127;
              const int sw = spot<FP8>(8 * (c16 >> 2) + (c16 & 3), 0) & 127;  // of t = 1: ^ 64
              constexpr int D = RT == 8 ? 2 : 4;  // reads under way
              i32x8 k[D];
              auto read = [&](int n) {  // window n / 2 of key tile n % 2; the rotary part last
                const uint8_t* src = from + (n >> 1) * 1024 + (n & 1) * 512;
                const bool rope = n >= 2 * LW;
                // Chunks 2 q4 and 2 q4 + 1, odd q4 the other way round, as the query has them;
                // of the rotary part q4 and 4 + q4.
                const int at = ((rope ? q4 << 4 : q4 << 5 | (q4 & 1) << 4) ^ sw) ^ (n & 1) << 6;
                const u32x4 y = *(const u32x4*)(src + at), z = *(const u32x4*)(src + (at ^ (rope ? 64 : 16)));
                k[n % D] = i32x8{(int)y.x, (int)y.y, (int)y.z, (int)y.w,
                                 (int)z.x, (int)z.y, (int)z.z, (int)z.w};
              };
#pragma unroll
              for (int n = 0; n < D; ++n) read(n);
#pragma unroll
              for (int n = 0; n < 2 * LW; ++n) {
                x[n & 1] = mx_mfma(k[n % D], qh[n >> 1], x[n & 1], q_exp);
                x[n & 1] = mx_mfma(k[n % D], ql[n >> 1], x[n & 1], q_exp);
                if (n + D < 2 * LW + 2) read(n + D);
                __builtin_amdgcn_sched_barrier(0);
              }
#pragma unroll
              for (int t = 0; t < 2; ++t) {
                vs[t] = *(const f32x4*)(lds + F::kScale + (st * TILE + blk * 32 + 8 * q4 + 4 * t) * 4);
                x[t] *= vs[t];  // the latent part alone
                const i32x8 r = k[(2 * LW + t) % D];
#pragma unroll
                for (int c = 0; c < 2; ++c)
                  x[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                      __builtin_bit_cast(bf16x8, i32x4{r[4 * c], r[4 * c + 1], r[4 * c + 2], r[4 * c + 3]}),
                      qr[c], x[t], 0, 0, 0);
              }
            } else {
              constexpr int N = 4 * LW + 4, D = RT == 8 ? 4 : 8;  // reads; of them under way
              const int sw = spot<FP8>(8 * (c16 >> 2) + 2 * (c16 & 3), q4);
              bf16x8 k[D];
              auto read = [&](int n) {  // step n / 2 of key tile n % 2
                const int c = n >> 1;
                k[n % D] = *(const bf16x8*)(from + (c >> 1) * 1024 + (sw ^ (c & 1) << 6 ^ (n & 1) << 7));
              };
#pragma unroll
              for (int n = 0; n < D; ++n) read(n);
#pragma unroll
              for (int n = 0; n < N; ++n) {
                const int c = n >> 1;
                x[n & 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                    k[n % D], c < 2 * LW ? qf[c] : qr[c - 2 * LW], x[n & 1], 0, 0, 0);
                if (n + D < N) read(n + D);
                if (n & 1) __builtin_amdgcn_sched_barrier(0);
              }
            }
            float top = -INFINITY;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
              if (cut) mask(blk, t, x[t], vs[t]);
              top = max2(max2(top, max2(x[t][0], x[t][1])),
                         max2(x[t][2], x[t][3]));
            }
            return max_over_key_groups(top);
          };
          // Their weights, into LDS; returns the lane's part of their sum.  They enter the second
          // product in bf16, each off by at most half a step (2^-8).  Of bf16 pages the
          // normaliser sums them as they were rounded, so that what the rounding does to a row's
          // large weights cancels; E4M3 tokens' scales go with their weights, and the sum is of
          // the weights before either.
          auto weigh = [&](int blk, const f32x4 (&x)[2], const f32x4 (&vs)[2]) {
            const float base = m == -INFINITY ? 0.f : m;
            uint32_t pw[4];
            float sum = 0.f;
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
              const f32x4 &v = x[e >> 2], &f = vs[e >> 2];
              f32x2 y = {__builtin_amdgcn_exp2f(__builtin_fmaf(v[e & 3], a.scale_log2, -base)),
                         __builtin_amdgcn_exp2f(__builtin_fmaf(v[(e & 3) + 1], a.scale_log2, -base))};
              if constexpr (FP8) {
                sum += y[0] + y[1];
                y[0] *= f[e & 3];
                y[1] *= f[(e & 3) + 1];
              }
              pw[e / 2] = __builtin_bit_cast(uint32_t, __builtin_convertvector(y, bf16x2));
              if constexpr (!FP8)
                sum += __uint_as_float(pw[e / 2] << 16) + __uint_as_float(pw[e / 2] & 0xFFFF0000u);
            }
            *(u32x4*)(p_row + p_at(row, blk * 4 + q4)) = u32x4{pw[0], pw[1], pw[2], pw[3]};
            return sum;
          };
          if constexpr (RT < 8 && NB == 2) {
            f32x4 x[2][2], vs[2][2];
            const float t0 = scores(0, x[0], vs[0]), t1 = scores(1, x[1], vs[1]);
            follow(max2(t0, t1));
            l += weigh(0, x[0], vs[0]);
            l += weigh(1, x[1], vs[1]);
          } else {
            // A block at a time, for its registers; where the second moves the reference, which
            // is hardly ever, the first again.
            float sum = 0.f;
#pragma unroll 1
            for (int blk = 0; blk < NB; ++blk) {
              f32x4 x[2], vs[2];
              const float was = m;
              follow(scores(blk, x, vs));
              if (NB > 1 && blk > 0 && __any(m != was)) {
                sum = 0.f;
                blk = -1;
                continue;
              }
              sum += weigh(blk, x, vs);
            }
            l += sum;
          }
          if (moved && q4 == 0) *(float*)(lds + F::kAlpha + (buf * F::kRows + row) * 4) = alpha;
          if (l1 == 0) lds[F::kFlag + buf * 8 + wave] = (uint8_t)moved;
        } else if (p > p_begin) {
          // ---- the second product of tile p - 1
          uint8_t* tile = lds + before * F::kStage;
          const uint8_t* p_rows = lds + F::kP + (buf ^ 1) * F::kWeights;
          const int l2 = lane_now(), c16 = l2 & 15, q4 = l2 >> 4;
          const int key0 = (p - 1) * TILE, here = ok >> (4 * before) & 15;
          uint64_t flags = *(const uint64_t*)(lds + F::kFlag + (buf ^ 1) * 8);
          if constexpr (RT < 8) flags &= (1ull << (8 * RT % 64)) - 1;
          if (__builtin_amdgcn_readfirstlane((int)(flags | flags >> 32))) {
#pragma unroll
            for (int t = 0; t < RT; ++t) {
              // Not written where none of the row tile's rows moved.
              const float f = *(const float*)(lds + F::kAlpha + ((buf ^ 1) * F::kRows + c16) * 4 + t * 64);
              const float alpha = flags >> (8 * t) & 1 ? f : 1.f;
#pragma unroll
              for (int d = 0; d < DT; ++d) acc[t][d] *= alpha;
              __builtin_amdgcn_sched_barrier(0);
            }
          }
          if (key0 + TILE > min_lim || here != (1 << PPT) - 1) {
            // 0 times what a key without data holds may be NaN: it becomes 0, each wave's part of
            // the latent by itself.  So does what only some rows see and is not finite, behind
            // its own sums for the rows that see it.
            constexpr int CW = (FP8 ? DW : 2 * DW) / 16;  // chunks of a wave's part of a key
            auto chunk = [&](int key, int c) {
              const int byte = wave * (FP8 ? DW : 2 * DW) + c * 16;
              return tile + (key >> 3) * GROUP + (byte >> 7) * 1024 + spot<FP8>(key, byte >> 4 & 7);
            };
            auto is_there = [&](int key) {
              return key0 + key < kv_lim && (here >> (key / kPage) & 1);
            };
            uint32_t nil;  // made here: as a constant it is kept in registers over the loop
            asm volatile("v_mov_b32 %0, 0" : "=v"(nil));
            uint64_t bad = 0;
#pragma unroll 1
            for (int i = l2; i < TILE * CW; i += 64) {
              const int key = i / CW;
              u32x4* at = (u32x4*)chunk(key, i % CW);
              bool odd = false;
              if (!is_there(key)) {
                *at = u32x4{nil, nil, nil, nil};
              } else if (key0 + key >= min_lim) {
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
              }
              // Chunks of 64 / CW keys, in order.
              const uint64_t hit = __ballot(odd);
              const int key_first = __builtin_amdgcn_readfirstlane(i) / CW;
#pragma unroll
              for (int n = 0; n < 64 / CW; ++n)
                if (hit >> (n * CW) & ((1ull << CW) - 1)) bad |= 1ull << (key_first + n);
            }
#pragma unroll 1
            for (uint64_t rest = bad; rest; rest &= rest - 1) {
              const int key = __builtin_ctzll(rest), l3 = lane_now(), c16 = l3 & 15, q4 = l3 >> 4;
              const int in8 = key & 7, pos = FP8 ? key & 31 : (key & 24) + (in8 >> 1) + (in8 & 1) * 4;
#pragma unroll
              for (int d = 0; d < DT; ++d) {
                const int in = (d * 16 + 4 * q4) * (FP8 ? 1 : 2);
                const uint8_t* src = chunk(key, in >> 4) + (in & 15);
                f32x4 v;
                if constexpr (FP8) {
                  const bf16x8 x = decode8(u32x2{*(const uint32_t*)src, 0});
                  v = f32x4{(float)x[0], (float)x[1], (float)x[2], (float)x[3]};
                } else {
                  const u32x2 x = *(const u32x2*)src;
                  v = f32x4{__uint_as_float(x.x << 16), __uint_as_float(x.x & 0xFFFF0000u),
                            __uint_as_float(x.y << 16), __uint_as_float(x.y & 0xFFFF0000u)};
                }
#pragma unroll
                for (int t = 0; t < RT; ++t) {
                  const float wt = bf16_to_f32(
                      *(const uint16_t*)(p_rows + p_at(c16, (key >> 5) * 4 + (pos >> 3)) +
                                         (pos & 7) * 2 + t * (32 * TILE)));
                  if (key0 + key < *(const int*)(lds + F::kLim + c16 * 4 + t * 64))
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                      acc[t][d][e] = __builtin_fmaf(wt, v[e], acc[t][d][e]);
                  __builtin_amdgcn_sched_barrier(0);
                }
              }
              if (l3 < CW) *(u32x4*)chunk(key, l3) = u32x4{nil, nil, nil, nil};
            }
          }
          // The lane's keys of a block of 32, and its place among the wave's dims.
          const int byte = wave * DW * (FP8 ? 1 : 2);
          const int key = FP8 ? c16 >> 1 : 2 * (c16 >> 2);
          const int ch = (byte >> 4 & 7) + (FP8 ? 0 : (c16 & 3) >> 1);
          const int v_base = q4 * GROUP + (byte >> 7) * 1024 + spot<FP8>(8 * q4 + key, ch) + ((c16 & 1) << 3);
          bf16x8 pf[2];
          auto weights = [&](int n) {  // of block n / RT, row tile n % RT
            pf[n & 1] = *(const bf16x8*)(p_rows + p_at(c16, n / RT * 4 + q4) + n % RT * (32 * TILE));
          };
          weights(0);
#pragma unroll
          for (int blk = 0; blk < NB; ++blk) {
            bf16x8 v[DT];
#pragma unroll
            for (int d = 0; d < DT; ++d) {
              if constexpr (FP8) {
                const uint8_t* from = tile + ((v_base ^ (d << 4)) + blk * 4 * GROUP);
                v[d] = decode8(__builtin_bit_cast(
                    u32x2, __builtin_amdgcn_ds_read_tr8_b64_v2i32((PDEC_LDS s32x2*)from)));
              } else {
                const uint8_t* even = tile + ((v_base ^ (d << 5)) + blk * 4 * GROUP);
                const uint8_t* odd = tile + ((v_base ^ (d << 5 | 128)) + blk * 4 * GROUP);
                const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((PDEC_LDS s16x4*)even);
                const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((PDEC_LDS s16x4*)odd);
                v[d] = __builtin_bit_cast(
                    bf16x8, s16x8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]});
              }
            }
#pragma unroll
            for (int t = 0; t < RT; ++t) {
              const int n = blk * RT + t;
              if (n + 1 < NB * RT) weights(n + 1);
#pragma unroll
              for (int d = 0; d < DT; ++d)
                acc[t][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[d], pf[n & 1], acc[t][d], 0, 0, 0);
              __builtin_amdgcn_sched_barrier(0);
            }
          }
        }
      }
      before = st;
      st = next;
    }

    // The rows' sums and references meet every wave's part of the output.
    wg_barrier();
    const int l4 = lane_now(), c16 = l4 & 15, q4 = l4 >> 4;
    float* sums = (float*)(lds + F::kAlpha);
    float* tops = sums + F::kRows;
    if (wave < RT) {
      const float sum = sum_over_key_groups(l);
      if (q4 == 0) {
        sums[rq * 16 + c16] = sum;
        tops[rq * 16 + c16] = m;
      }
    }
    wg_barrier();
    const bool whole = p_begin == 0 && p_end == tiles;
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      const int row = t * 16 + c16;
      if (row >= rows) continue;
      const float sum = sums[row];
      if (whole) {
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        uint16_t* o = (uint16_t*)a.out + (q_row0 + row) * R + wave * DW + 4 * q4;
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
        float* o = a.part_acc + pr * R + wave * DW + 4 * q4;
#pragma unroll
        for (int d = 0; d < DT; ++d) *(f32x4*)(o + d * 16) = acc[t][d];
      }
    }
  }
  wait_vmem<0>();  // no LDS write may still be in flight when the group ends
}

// Merges the pieces of each unit, and writes zeros for the rows of a unit that sees no key.
// R / 4 lanes hold a row.  A row of up to eight pieces is theirs alone, all its pieces under way
// at once; of more pieces the S rows' worth of lanes share each row, their results joined in
// order.  A work group takes several rows (rows_per_group), so that what it looks up about the
// units first is paid once for them.
template <int R, int TILE>
__global__ __launch_bounds__(512) void latent_merge_kernel(LatentAttnArgs a, int rows_per_unit,
                                                           int rows_per_group) {
  constexpr int L = R / 4, S = 512 / L;  // lanes of a row, rows or pieces at once
  __shared__ int red[2][8];
  __shared__ float sh[S - 1][6][L];
  const int u = blockIdx.x, row0 = unit_row0(a, u);
  const int row_begin = blockIdx.y * rows_per_group;
  const int row_end = min(row_begin + rows_per_group, unit_rows(a, row0));
  if (row_begin >= row_end) return;
  int all = 0, before = 0;
  for (int v = threadIdx.x; v < a.n_units; v += 512) {
    const int n = unit_size<TILE>(a, v);
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
  const int tiles = unit_tiles<TILE>(a, u), body = first + unit_head<TILE>(a), w0 = body / per;
  const int w1 = tiles > 0 ? (body + tiles - 1) / per : w0 - 1;
  if (tiles > 0 && w0 == w1) return;
  const int lane = threadIdx.x % L, part = threadIdx.x / L;
  float m, l;
  f32x4 o;
  auto join = [&](float mi, float li, f32x4 oi) {
    const float mn = fmaxf(m, mi), mu = mn == -INFINITY ? 0.f : mn;
    const float so = exp2f(m - mu), si = exp2f(mi - mu);
    l = l * so + li * si;
    o = o * so + oi * si;
    m = mn;
  };
  auto join_from = [&](int row, int begin, int step) {
    m = -INFINITY;
    l = 0.f;
    o = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int w = begin; w <= w1; w += 8 * step) {
      float2 ml[8];
      f32x4 x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (w + i * step <= w1) {
          const int64_t pr = ((int64_t)(w + i * step) + u) * rows_per_unit + row;
          ml[i] = *(const float2*)(a.part_ml + pr * 2);
          x[i] = *(const f32x4*)(a.part_acc + pr * R + lane * 4);
        }
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (w + i * step <= w1) join(ml[i].x, ml[i].y, x[i]);
    }
  };
  auto write = [&](int row) {
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const f32x2 lo = {o[0] * inv, o[1] * inv}, hi = {o[2] * inv, o[3] * inv};
    *(u32x2*)((uint16_t*)a.out +
              ((int64_t)(u / a.blocks_per_seq) * a.n_q * a.n_heads + row0 + row) * R + lane * 4) =
        u32x2{__builtin_bit_cast(uint32_t, __builtin_convertvector(lo, bf16x2)),
              __builtin_bit_cast(uint32_t, __builtin_convertvector(hi, bf16x2))};
  };
  if (w1 - w0 < 8) {
    for (int row = row_begin + part; row < row_end; row += S) {
      join_from(row, w0, 1);
      write(row);
    }
    return;
  }
  for (int row = row_begin; row < row_end; ++row) {
    join_from(row, w0 + part, S);
    if (part > 0) {
      float(*d)[L] = sh[part - 1];
      d[0][lane] = m;
      d[1][lane] = l;
#pragma unroll
      for (int e = 0; e < 4; ++e) d[2 + e][lane] = o[e];
    }
    __syncthreads();
    if (part == 0) {
#pragma unroll
      for (int i = 0; i < S - 1; ++i) {
        const float(*d)[L] = sh[i];
        join(d[0][lane], d[1][lane], f32x4{d[2][lane], d[3][lane], d[4][lane], d[5][lane]});
      }
      write(row);
    }
    __syncthreads();
  }
}

// Rows of a merge group: one where units are so few that each may have more than eight pieces,
// which all its lanes then share.  us of the call at 1 / 4: 16 heads over 64 sequences 49.2 / 47.6;
// at 1 / 8: 128 heads 182 / 154.
int merge_rows(int rows, const LatentAttnArgs& a) {
  if ((int64_t)rows * a.n_units >= 4096) return 8;
  return a.n_groups / a.n_units + 2 <= 8 ? 4 : 1;
}

}  // namespace

hipError_t launch_latent_attention(int fp8, int latent, int row_tiles, const LatentAttnArgs& a,
                                   hipStream_t stream) {
  const int grid = a.unit_groups ? a.n_units : a.n_groups;
#define PDEC_LATENT(R_, FP8_)                                                                    \
  do {                                                                                           \
    hipError_t e = hipSuccess;                                                                   \
    if (row_tiles == 1)                                                                          \
      e = launch_latent_few(FP8_, R_, grid, a, stream);                                          \
    else if (row_tiles == 2)                                                                     \
      latent_attn_kernel<R_, 2, FP8_><<<grid, kThreads, 0, stream>>>(a);                         \
    else if (row_tiles == 4)                                                                     \
      latent_attn_kernel<R_, 4, FP8_><<<grid, kThreads, 0, stream>>>(a);                         \
    else                                                                                         \
      latent_attn_kernel<R_, 8, FP8_><<<grid, kThreads, 0, stream>>>(a);                         \
    if (e == hipSuccess) e = hipGetLastError();                                                  \
    if (e != hipSuccess || a.unit_groups) return e;                                              \
    const int rows = std::min(a.block_rows, a.n_q * a.n_heads);                                  \
    const int each = merge_rows(rows, a);                                                        \
    const dim3 mgrid(a.n_units, (rows + each - 1) / each);                                       \
    latent_merge_kernel<R_, latent_tile(FP8_, R_)>                                               \
        <<<mgrid, 512, 0, stream>>>(a, 16 * row_tiles, each);                                    \
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
