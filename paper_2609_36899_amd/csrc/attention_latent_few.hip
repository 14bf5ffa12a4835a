// Attention over latent pages where a unit has at most sixteen query rows (a few heads' share, or
// small models): attention_latent.hip's formula, units and split of the work.
//
// Bound by HBM: a key's 2 (2 R + 64) operations a row are a few cycles of the matrix units beside
// its R + 132 (E4M3) or 2 R + 128 bytes.  Such a call needs bytes on their way at all times, and
// the chain from a page to its part of the output, which one wave takes thousands of cycles for,
// off their path.  So a group's waves go in teams, each over every n-th page of the piece with a
// ring of four pages in LDS: one wave multiplies S^T = K Q^T, two take the weights through LDS a
// step later and multiply O^T = C^T P^T, each half of the latent.  Two waves more do nothing but
// bring the pages: a load holds its wave for 60 cycles and more.  A page's sixteen keys are one
// tile of the first product, and a lane's four weights are the operand P of the second, over
// sixteen keys, as they are.  At the end of a piece the teams' sums are joined through LDS.  A
// unit reads its pages once, so they do not stay in the caches.  us so / kept there, 16 heads: 64
// sequences of 4K that share nothing 45 / 51 (E4M3) and 61 / 70 (bf16); eight forks each of eight
// prompts, of 4K shared and 50 to 400 tokens of their own 45 / 42 and 49 / 35, of 2K shared and 0.5K
// to 4K 46 / 44 and 62 / 58, of 0.5K and 0.5K to 4K 40 / 37 and 44 / 46, of 1K and 1K to 8K 55 / 57
// and 75 / 76.  Which pages are shared only the tables on the device say.
//
// 16 heads over 64 x 1K to 8K E4M3 43 us and the merge's 6 (205 MB): a step of three pages takes
// 2450 cycles, 6.7 TB/s over all units, and the pieces' beginnings and ends 13 us.  Four short
// sequences of R = 256 7.5 to 8.6 us.  By the form for more rows 61 us, by waves that do all of a
// page by themselves 51, with the loads among the first product's 49.
#include "latent_attn.h"

namespace pdec {

namespace {

template <int R, bool FP8>
struct FewForm {
  static constexpr int kRow = FP8 ? R + 2 * kRope : (R + kRope) * 2;  // a key's bytes
  static constexpr int kTile = kPage * kRow, kStages = 4;
  // Teams of three waves, by what four pages each leave room for: 2 with bf16 latents of 512,
  // else 3.
  static constexpr int kTeams = 12 * kTile <= 144 * 1024 ? 3 : 2;
  static constexpr int kThreads = 192 * kTeams + 128;
  static constexpr int kRing = kStages * kTile * kTeams, kJoin = kTeams * 16 * R * 4;
  // LDS offsets.
  static constexpr int kScale = kRing > kJoin ? kRing : kJoin;  // [kTeams][kStages][16]
  static constexpr int kP = kScale + (FP8 ? kTeams * kStages * kPage * 4 : 0);  // [kTeams][2][64] x 8
  static constexpr int kAlpha = kP + kTeams * 2 * 512;          // [kTeams][2][16]
  static constexpr int kSums = kAlpha + kTeams * 2 * 64;        // [kTeams][2][16]
  static constexpr int kFlag = kSums + kTeams * 2 * 64;         // [kTeams][2]: references that moved
  static constexpr int kBytes = kFlag + kTeams * 2 * 4;
  static_assert(kBytes <= 160 * 1024 - 64 && kTile % 256 == 0, "LDS layout");
};

template <int R, bool FP8, int UNIT_TILE>
__global__ __launch_bounds__((FewForm<R, FP8>::kThreads)) void latent_few_kernel(LatentAttnArgs a) {
  typedef FewForm<R, FP8> F;
  constexpr int ROW = F::kRow, NST = F::kStages, TEAMS = F::kTeams, THREADS = F::kThreads;
  constexpr int WIN = ROW / 128, LW = (FP8 ? R : 2 * R) / 128;
  constexpr int GROUP = 8 * ROW, DT = R / 16, DH = DT / 2, PPT = UNIT_TILE / kPage;
  constexpr int NL = WIN + (FP8 ? 1 : 0);  // loads of half a page
  __shared__ __attribute__((aligned(256))) uint8_t lds[F::kBytes];
  __shared__ int red[THREADS / 64];
  __shared__ int found[2];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), w = blockIdx.x;
  // A team's waves: one takes the first product, two the second, each half of the latent.  The
  // last two waves of the group, of no team, load.
  const bool scorer = wave < TEAMS, loader = wave >= 3 * TEAMS;
  const int team = scorer ? wave : (wave - TEAMS) >> 1, half = (wave - TEAMS) & 1;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(PDEC_LDS uint8_t*)lds;
  float* scales = (float*)(lds + F::kScale) + team * NST * kPage;
  uint8_t* p_at = lds + F::kP + team * 2 * 512;
  float* alphas = (float*)(lds + F::kAlpha) + team * 2 * 16;
  int* flags = (int*)(lds + F::kFlag) + team * 2;

  int at = 0, end, u = w, first = 0;
  if (a.unit_groups) {
    end = unit_tiles<UNIT_TILE>(a, u);
    if (end == 0) {
      const int row0 = unit_row0(a, u), rows = unit_rows(a, row0);
      uint16_t* o = (uint16_t*)a.out +
                    ((int64_t)(u / a.blocks_per_seq) * a.n_q * a.n_heads + row0) * R;
      for (int i = threadIdx.x; i < rows * (R / 8); i += THREADS)
        *(u32x4*)(o + i * 8) = u32x4{0, 0, 0, 0};
      return;
    }
  } else {
    const Stretch mine = stretch_of<THREADS>(a.n_units, a.n_groups, a.min_tiles, w, red, found,
                                              [&](int v) { return unit_size<UNIT_TILE>(a, v); });
    at = w * mine.per;
    if (at >= mine.total) return;
    end = min(at + mine.per, mine.total);
    u = __builtin_amdgcn_readfirstlane(mine.unit);
    first = __builtin_amdgcn_readfirstlane(mine.first);
    at = __builtin_amdgcn_readfirstlane(at);
    end = __builtin_amdgcn_readfirstlane(end);
  }

  // Score e of a lane belongs to key_of(q4, e): of bf16 pages a group of sixteen lanes has the
  // even or the odd keys of eight, since a transposing read brings four keys, which must differ
  // in their place by more than one; of E4M3 pages, where it brings eight, they go in order.
  auto key_of = [](int q, int e) { return FP8 ? 4 * q + e : 2 * e + (q & 1) + 8 * (q >> 1); };

  // A row's reference and sum over all teams, and what this team's part of the output is times.
  struct Join {
    float top, sum, own;
  };
  auto join_of = [&](int row) {
    const float* sums = (const float*)(lds + F::kSums) + row;  // references, then sums
    Join o = {-INFINITY, 0.f, 0.f};
#pragma unroll
    for (int v = 0; v < TEAMS; ++v) o.top = fmaxf(o.top, sums[v * 32]);
#pragma unroll
    for (int v = 0; v < TEAMS; ++v) {
      const float m = sums[v * 32], f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - o.top);
      o.sum = __builtin_fmaf(sums[v * 32 + 16], f, o.sum);
      if (v == team) o.own = f;
    }
    return o;
  };

  for (; at < end; ++u) {
    const int tiles = unit_tiles<UNIT_TILE>(a, u), size = unit_size<UNIT_TILE>(a, u);
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
    // The team's pages: g_begin, g_begin + TEAMS ...; a step takes one of each team's.
    const int g_begin = p_begin * PPT + team, g_end = min(p_end * PPT, n_pages);
    const int steps = max(g_end - p_begin * PPT + TEAMS - 1, 0) / TEAMS;
    const bool whole = p_begin == 0 && p_end == tiles;
    __syncthreads();  // the piece before is done with LDS

    if (scorer) {
      // Ids of 64 of the team's pages, one a lane.
      int ids;
      auto look = [&](int i0) {
        const int n = g_begin + (i0 + lane_now()) * TEAMS;
        ids = n < g_end ? a.block_table[(int64_t)b * a.bt_stride + n] : -1;
        if (ids >= a.n_pages) ids = -1;
      };
      look(0);
      uint32_t ok = 0;  // which stages' pages are there
      auto note = [&](int i) {  // page i, and returns its id or -1
        if ((i & 63) == 0 && i > 0) look(i);
        const int id = __builtin_amdgcn_readlane(ids, i & 63);
        ok = (ok & ~(1u << (i & (NST - 1)))) | (uint32_t)(id >= 0) << (i & (NST - 1));
        return id;
      };
      bf16x8 qr[2], x[(FP8 ? 4 : 2) * LW];
      int row_lim;
      {
        const int l0 = lane_now(), c16 = l0 & 15, q4 = l0 >> 4;
        const int row = min(c16, rows - 1);  // rows past the unit's repeat its last
        row_lim = base_lim + (row0 + row) / a.n_heads;
        const uint16_t* src = (const uint16_t*)a.q + (q_row0 + row) * (R + kRope);
#pragma unroll
        for (int c = 0; c < 2; ++c) qr[c] = *(const bf16x8*)(src + R + c * 32 + q4 * 8);
        if constexpr (FP8) read_query<LW>(src, q4, x);
        else
#pragma unroll
          for (int c = 0; c < 2 * LW; ++c) x[c] = *(const bf16x8*)(src + c * 32 + q4 * 8);
      }
      i32x8 qh[LW], ql[LW];  // of E4M3 pages
      int q_exp = 0;
      if constexpr (FP8) q_exp = split_query<LW>(x, qh, ql);

      note(0);
      note(1);
      float m = -INFINITY, l = 0.f;  // a reference for the row's scores; this lane's part of its sum
#pragma unroll 1
      for (int j = 0; j <= steps; ++j) {
        wg_barrier();  // page j and the weights of page j - 1 are here, and page j - 2 has been used
        if (j == steps) break;
        const int st = j & (NST - 1);
        const int here = ok >> st & 1;
        int moved = 0;
        u32x2 weights = {0, 0};
        note(j + 2);
        if (here) {
          const uint8_t* tile = lds + (team * NST + st) * F::kTile;
          const int key0 = (g_begin + j * TEAMS) * kPage;
          const bool cut = key0 + kPage > min_lim;
          const int l1 = lane_now(), c16 = l1 & 15, q4 = l1 >> 4;
          // Where the lane reads keys' chunks.
          const int k_key = key_of(c16 >> 2, c16 & 3);
          const int k_at = (k_key >> 3) * GROUP +
                           (FP8 ? spot<FP8>(k_key, 0) & ~127 : spot<FP8>(k_key, q4));
          const int k_sw = spot<FP8>(k_key, 0) & 127;  // of E4M3 pages
          f32x4 s = {0.f, 0.f, 0.f, 0.f}, vs = {1.f, 1.f, 1.f, 1.f};
          if constexpr (FP8) {
            f32x4 s2 = {0.f, 0.f, 0.f, 0.f};
            auto read = [&](int at, int flip) {  // chunks 2 q4 and 2 q4 + 1, exchanged for odd q4
              const u32x4 y = *(const u32x4*)(tile + at), z = *(const u32x4*)(tile + (at ^ flip));
              return i32x8{(int)y.x, (int)y.y, (int)y.z, (int)y.w,
                           (int)z.x, (int)z.y, (int)z.z, (int)z.w};
            };
            i32x8 k[LW + 1];
#pragma unroll
            for (int n = 0; n < LW; ++n)
              k[n] = read(k_at + n * 1024 + ((q4 << 5 | (q4 & 1) << 4) ^ k_sw), 16);
            k[LW] = read(k_at + LW * 1024 + (q4 << 4 ^ k_sw), 64);
            __builtin_amdgcn_sched_barrier(0);  // all of them under way
#pragma unroll
            for (int n = 0; n < LW; ++n) {
              s = mx_mfma(k[n], qh[n], s, q_exp);
              s2 = mx_mfma(k[n], ql[n], s2, q_exp);
            }
            vs = *(const f32x4*)(scales + st * kPage + 4 * q4);
            s = (s + s2) * vs;  // the latent part alone
            const i32x8 r = k[LW];
#pragma unroll
            for (int c = 0; c < 2; ++c)
              s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                  __builtin_bit_cast(bf16x8, i32x4{r[4 * c], r[4 * c + 1], r[4 * c + 2], r[4 * c + 3]}),
                  qr[c], s, 0, 0, 0);
          } else {
            constexpr int N = 2 * LW + 2, D = 10;  // reads; of them under way
            bf16x8 k[D];
            auto read = [&](int c) {
              k[c % D] = *(const bf16x8*)(tile + (k_at ^ (c & 1) << 6) + (c >> 1) * 1024);
            };
#pragma unroll
            for (int c = 0; c < D; ++c) read(c);
#pragma unroll
            for (int c = 0; c < N; ++c) {
              s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[c % D], c < 2 * LW ? x[c] : qr[c - 2 * LW],
                                                          s, 0, 0, 0);
              if (c + D < N) read(c + D);
              __builtin_amdgcn_sched_barrier(0);
            }
          }
          // Where a row does not see a key its score is -inf, and the token's scale, which may be
          // anything, 0.
          if (cut) {
            int lim = row_lim - key0;
            asm volatile("" : "+v"(lim));
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (key_of(q4, e) >= lim) {
                s[e] = -INFINITY;
                vs[e] = 0.f;
              }
          }
          const float now =
              max_over_key_groups(max2(max2(s[0], s[1]), max2(s[2], s[3]))) * a.scale_log2;
          if (__any(!(now <= m + kSlack))) {
            const bool need = now > m + kSlack;
            const float f = need ? __builtin_amdgcn_exp2f(m - now) : 1.f;
            if (need) m = now;
            l *= f;
            if (q4 == 0) alphas[(j & 1) * 16 + c16] = f;
            moved = 1;
          }
          // The weights enter the second product in bf16, each off by at most half a step (2^-8).
          // Of bf16 pages the normaliser sums them as they were rounded; E4M3 tokens' scales go
          // with their weights, and the sum is of the weights before either.
          const float base = m == -INFINITY ? 0.f : m;
          uint32_t pw[2];
#pragma unroll
          for (int e = 0; e < 4; e += 2) {
            f32x2 y = {__builtin_amdgcn_exp2f(__builtin_fmaf(s[e], a.scale_log2, -base)),
                       __builtin_amdgcn_exp2f(__builtin_fmaf(s[e + 1], a.scale_log2, -base))};
            if constexpr (FP8) {
              l += y[0] + y[1];
              y[0] *= vs[e];
              y[1] *= vs[e + 1];
            }
            pw[e / 2] = __builtin_bit_cast(uint32_t, __builtin_convertvector(y, bf16x2));
            if constexpr (!FP8)
              l += __uint_as_float(pw[e / 2] << 16) + __uint_as_float(pw[e / 2] & 0xFFFF0000u);
          }
          weights = u32x2{pw[0], pw[1]};
        }
        const int l2 = lane_now();
        *(u32x2*)(p_at + (j & 1) * 512 + l2 * 8) = weights;
        if (l2 == 0) flags[j & 1] = moved;
      }
      // The rows' references and sums.
      const int l0 = lane_now();
      const float sum = sum_over_key_groups(l);
      float* sums = (float*)(lds + F::kSums) + team * 32;
      if (l0 < 16) {
        sums[l0] = m;
        sums[16 + l0] = sum;
      }
      wg_barrier();  // every ring has been read, and no load is in flight
    } else if (loader) {
      // A loader, of half of every page's keys.  Ids of 256 of the piece's pages, four a lane:
      // looking for more waits for the pages in flight.
      const int g = wave - 3 * TEAMS, lane = lane_now();
      const int offset = window_offset<FP8, ROW>(lane, g) + g * GROUP;
      int ids[4];
      // Every team's page j into its ring.  A page that is not there, or behind the last, is a
      // buffer without bytes: zeros come, and count.  All of the place is in the lane's offset,
      // the one that is certain to be held against the buffer's size.
      auto load = [&](int j) {
#pragma unroll
        for (int k = 0; k < TEAMS; ++k) {
          const int i = j * TEAMS + k, st = j & (NST - 1);
          if ((i & 255) == 0)
#pragma unroll
            for (int h = 0; h < 4; ++h) {
              const int n = p_begin * PPT + i + h * 64 + lane;
              ids[h] = n < g_end ? a.block_table[(int64_t)b * a.bt_stride + n] : -1;
              if (ids[h] >= a.n_pages) ids[h] = -1;
            }
          const int which = i >> 6 & 3, at = i & 63;
          const int id = __builtin_amdgcn_readlane(
              which == 0 ? ids[0] : which == 1 ? ids[1] : which == 2 ? ids[2] : ids[3], at);
          const int64_t p = max(id, 0);
          const DmaBuffer from =
              dma_buffer((const uint8_t*)a.pages + p * F::kTile, id >= 0 ? F::kTile : 0);
          const uint32_t to = lds0 + (k * NST + st) * F::kTile + g * GROUP;
          each<WIN>([&](auto n) {
            dma16_unseen<n * 128, n * 1024, true>(from, offset, 0, to);
          });
          if constexpr (FP8) {
            const DmaBuffer f = dma_buffer(a.scales + p * kPage + g * 8, id >= 0 ? 32 : 0);
            if (lane < 8)
              dma4_unseen(f, lane * 4, lds0 + F::kScale + ((k * NST + st) * kPage + g * 8) * 4);
          }
        }
      };
      load(0);
      load(1);
#pragma unroll 1
      for (int j = 0; j <= steps; ++j) {
        wait_vmem<TEAMS * NL>();  // the pages j are here
        wg_barrier();
        if (j < steps) load(j + 2);
      }
      wait_vmem<0>();
      wg_barrier();
    } else {
      f32x4 acc[DH];
#pragma unroll
      for (int d = 0; d < DH; ++d) acc[d] = f32x4{0.f, 0.f, 0.f, 0.f};
      wg_barrier();
#pragma unroll 1
      for (int j = 1; j <= steps; ++j) {  // page i; one that is not there is zeros, and so are its weights
        wg_barrier();
        const int i = j - 1, st = i & (NST - 1);
        const int moved = __builtin_amdgcn_readfirstlane(flags[i & 1]);
        uint8_t* tile = lds + (team * NST + st) * F::kTile + half * (LW * 512);  // its windows
        const uint8_t* weights = p_at + (i & 1) * 512;
        const int key0 = (g_begin + i * TEAMS) * kPage;
        if (moved) {
          const float f = alphas[(i & 1) * 16 + (lane_now() & 15)];
#pragma unroll
          for (int d = 0; d < DH; ++d) {
            acc[d] *= f;
            __builtin_amdgcn_sched_barrier(0);
          }
        }
        if (key0 + kPage > min_lim) {
          // 0 times what a key without data holds may be NaN: it becomes 0.  So does what only
          // some rows see and is not finite, behind its own sums for the rows that see it.
          constexpr int CW = (FP8 ? R : 2 * R) / 32;  // chunks of half a key's latent
          auto chunk = [&](int key, int c) {
            return (u32x4*)(tile + (key >> 3) * GROUP + (c >> 3) * 1024 + spot<FP8>(key, c & 7));
          };
          uint32_t nil, bad = 0;  // made here: as a constant it is kept in registers over the loop
          asm volatile("v_mov_b32 %0, 0" : "=v"(nil));
#pragma unroll 1
          for (int n = lane_now(); n < kPage * CW; n += 64) {
            const int key = n / CW;
            u32x4* to = chunk(key, n % CW);
            bool odd = false;
            if (key0 + key >= kv_lim) {
              *to = u32x4{nil, nil, nil, nil};
            } else if (key0 + key >= min_lim) {
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const uint32_t y = (*to)[e];
                if constexpr (FP8) {
#pragma unroll
                  for (int h = 0; h < 32; h += 8) odd |= (y >> h & 0x7F) == 0x7F;
                } else {
                  odd |= (y & 0x7F80) == 0x7F80 || (y >> 16 & 0x7F80) == 0x7F80;
                }
              }
            }
            const uint64_t hit = __ballot(odd);
            const int key_first = __builtin_amdgcn_readfirstlane(n) / CW;
#pragma unroll
            for (int k = 0; k < 64 / CW; ++k)
              if (hit >> (k * CW) & ((1ull << CW) - 1)) bad |= 1u << (key_first + k);
          }
#pragma unroll 1
          for (uint32_t rest = bad; rest; rest &= rest - 1) {
            const int key = __builtin_ctz(rest);
            // The group of lanes that had the key's weights, and which of theirs it is.
            const int l1 = lane_now(), c16 = l1 & 15, q4 = l1 >> 4;
            const int q = FP8 ? key >> 2 : (key >> 3) * 2 + (key & 1);
            const int e = FP8 ? key & 3 : key >> 1 & 3;
            const float wt = bf16_to_f32(*(const uint16_t*)(weights + (q * 16 + c16) * 8 + e * 2));
            const bool seen = key0 + key < base_lim + (row0 + min(c16, rows - 1)) / a.n_heads;
#pragma unroll
            for (int d = 0; d < DH; ++d) {
              const int in = (d * 16 + 4 * q4) * (FP8 ? 1 : 2);
              const uint8_t* from = (const uint8_t*)chunk(key, in >> 4) + (in & 15);
              f32x4 v;
              if constexpr (FP8) {
                const bf16x8 y = decode8(u32x2{*(const uint32_t*)from, 0});
                v = f32x4{(float)y[0], (float)y[1], (float)y[2], (float)y[3]};
              } else {
                const u32x2 y = *(const u32x2*)from;
                v = f32x4{__uint_as_float(y.x << 16), __uint_as_float(y.x & 0xFFFF0000u),
                          __uint_as_float(y.y << 16), __uint_as_float(y.y & 0xFFFF0000u)};
              }
              if (seen)
#pragma unroll
                for (int h = 0; h < 4; ++h) acc[d][h] = __builtin_fmaf(wt, v[h], acc[d][h]);
              __builtin_amdgcn_sched_barrier(0);
            }
            if (l1 < CW) *chunk(key, l1) = u32x4{nil, nil, nil, nil};
          }
        }
        const s16x4 pf = *(const s16x4*)(weights + lane_now() * 8);
        // Values, transposed.  Of E4M3 pages eight keys of a dim; the lane's four are the first or
        // the last of them.
        const int l3 = lane_now(), v_c = l3 & 15, v_q = l3 >> 4;
        const int v_key = FP8 ? 8 * (v_q >> 1) + (v_c >> 1) : key_of(v_q, v_c >> 2);
        const int v_at = (v_q >> 1) * GROUP + spot<FP8>(v_key, FP8 ? 0 : (v_c & 3) >> 1) + ((v_c & 1) << 3);
        constexpr int D = 8;  // reads under way
        u32x2 v[D];
        auto read = [&](int d) {
          if constexpr (FP8)
            v[d % D] = __builtin_bit_cast(
                u32x2, __builtin_amdgcn_ds_read_tr8_b64_v2i32(
                           (PDEC_LDS s32x2*)(tile + (d >> 3) * 1024 + (v_at ^ (d & 7) << 4))));
          else
            v[d % D] = __builtin_bit_cast(
                u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                           (PDEC_LDS s16x4*)(tile + (d >> 2) * 1024 + (v_at ^ (d & 3) << 5))));
        };
#pragma unroll
        for (int d = 0; d < D; ++d) read(d);
#pragma unroll
        for (int d0 = 0; d0 < DH; d0 += 4) {
          u32x2 y[4];
#pragma unroll
          for (int h = 0; h < 4; ++h) y[h] = v[(d0 + h) % D];
          if constexpr (FP8)
#pragma unroll
            for (int h = 0; h < 4; ++h) {
              const uint32_t codes = v_q & 1 ? y[h].y : y[h].x;
              y[h].x = __builtin_bit_cast(
                  uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, 1.f, false));
              y[h].y = __builtin_bit_cast(
                  uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, 1.f, true));
            }
#pragma unroll
          for (int h = 0; h < 4; ++h) {
            acc[d0 + h] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(
                __builtin_bit_cast(s16x4, y[h]), pf, acc[d0 + h], 0, 0, 0);
            if (d0 + h + D < DH) read(d0 + h + D);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      wg_barrier();  // every ring has been read, and no load is in flight
      const int l0 = lane_now();
      const float f = join_of(l0 & 15).own;
#pragma unroll
      for (int d = 0; d < DH; ++d) ((f32x4*)lds)[(team * DT + half * DH + d) * 64 + l0] = acc[d] * f;
    }

    // The teams' sums meet, in order; the waves share the latent's tiles.
    wg_barrier();
    const int l2 = lane_now(), c16 = l2 & 15, q4 = l2 >> 4;
    const Join all = join_of(c16);
    const float inv = all.sum == 0.f ? 0.f : 1.f / all.sum;
    const f32x4* join = (const f32x4*)lds;  // [TEAMS][DT][64]
    const int64_t pr = ((int64_t)w + u) * 16 + c16;
    if (c16 < rows) {
      if (!whole && wave == 0 && q4 == 0) *(float2*)(a.part_ml + pr * 2) = float2{all.top, all.sum};
      for (int d = wave; d < DT; d += THREADS / 64) {
        f32x4 o = join[d * 64 + l2];
#pragma unroll
        for (int v = 1; v < TEAMS; ++v) o += join[(v * DT + d) * 64 + l2];
        if (whole) {
          const f32x2 lo = {o[0] * inv, o[1] * inv}, hi = {o[2] * inv, o[3] * inv};
          *(u32x2*)((uint16_t*)a.out + (q_row0 + c16) * R + d * 16 + 4 * q4) =
              u32x2{__builtin_bit_cast(uint32_t, __builtin_convertvector(lo, bf16x2)),
                    __builtin_bit_cast(uint32_t, __builtin_convertvector(hi, bf16x2))};
        } else {
          *(f32x4*)(a.part_acc + pr * R + d * 16 + 4 * q4) = o;
        }
      }
    }
  }
}

}  // namespace

hipError_t launch_latent_few(int fp8, int latent, int grid, const LatentAttnArgs& a,
                             hipStream_t stream) {
#define PDEC_FEW(R_, FP8_) \
  latent_few_kernel<R_, FP8_, latent_tile(FP8_, R_)>            \
      <<<grid, FewForm<R_, FP8_>::kThreads, 0, stream>>>(a)
  if (latent == 512) {
    if (fp8) PDEC_FEW(512, true);
    else PDEC_FEW(512, false);
  } else {
    if (fp8) PDEC_FEW(256, true);
    else PDEC_FEW(256, false);
  }
#undef PDEC_FEW
  return hipGetLastError();
}

}  // namespace pdec
