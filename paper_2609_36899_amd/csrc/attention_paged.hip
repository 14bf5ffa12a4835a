// Attention of one or several query tokens per sequence over caller-owned pages,
// with the sequence lengths on the device.
//
//   out[b][j][h] = softmax(q[b][j][h] . K^T / sqrt(Dh)) V  over positions
//   0 .. lens[b] - n_q + j of sequence b (query token j's own position among
//   them), or over the pages that `selected` lists for (b, KV head).
//
// K and V pages are bf16, or E4M3 codes with a scale for each page and KV head.
// Every cached byte is read once for up to 128 query rows (tokens x heads) of a KV head,
// again for the next 128.  Up to 32 rows the call is bound by HBM; from there on arithmetic
// counts: over 16 x 4K to 16K 52 rows take twice what their reads would (E4M3 92 us, 43),
// 104 rows three times (140), by some 250 vector instructions a pair of pages beside its 34
// MFMAs and, of E4M3 pages and of bf16 ones at 104 rows, registers spilled (4 and 17).
// Prompts of n tokens alone, 32 heads on 8, E4M3 / bf16: 256 18 / 18 us, 1024 62 / 66, 4096
// 309 / 329 (0.44 / 0.42 PFLOP/s); 256 tokens each over 4 x 16K 389 (0.70 PFLOP/s).
//
// Work split.  A unit is a block of query tokens of one sequence (their n_tok * G
// rows, 16 to 128 of them); its work is its key range in pairs of pages.  The units' pairs
// laid end to end are cut into n_groups equal stretches, one for each work group of a
// KV head, whatever the lengths: a group finds its stretch from a prefix sum of the
// lengths that it makes itself, so no plan is built on the host or uploaded, and a
// captured graph follows lengths that change on the device.  A stretch may cover the end of
// one unit and the beginning of the next: the piece of unit u in group w leaves its
// softmax partial (maximum, sum, unnormalised output) in slot w + u, which no other
// piece has, and the merge pass finds a unit's pieces side by side.  A unit that one
// group covers whole is written out at once.  Where no unit can be long, each has a group
// of its own.
#include "hip_common.h"
#include "kernels.h"
#include "stretch.h"

#include <algorithm>
#include <type_traits>

namespace pdec {

namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kPair = 2 * kPage;        // keys of a pair of pages
constexpr int kNowhere = 0x40000000;    // a key position past every limit
constexpr float kMinScale = 0x1p-100f;

__device__ __forceinline__ int clamp_len(const PagedAttnArgs& a, int b) {
  return min(max(a.lens[b], 0), a.max_len);
}

// Keys (exclusive end) that any row of unit u sees, and the pairs of pages they fill.
__device__ __forceinline__ int unit_keys(const PagedAttnArgs& a, int u) {
  const int b = u / a.blocks_per_seq, j1 = min((u % a.blocks_per_seq + 1) * a.tok_per_block, a.n_q);
  return max(clamp_len(a, b) - a.n_q + j1, 0);
}
__device__ __forceinline__ int unit_pages(const PagedAttnArgs& a, int u) {
  const int n = (unit_keys(a, u) + kPage - 1) / kPage;
  return a.selected ? min(n, a.n_selected) : n;
}
__device__ __forceinline__ int unit_pairs(const PagedAttnArgs& a, int u) {
  return (unit_pages(a, u) + 1) / 2;
}

// Offset of row `row` (token, query head) of a block in q and out.
template <int DH>
__device__ __forceinline__ int64_t row_at(const PagedAttnArgs& a, int b, int j0, int g, int row) {
  const int G = a.n_q_heads / a.n_kv_heads;
  return (((int64_t)b * a.n_q + j0 + row / G) * a.n_q_heads + g * G + row % G) * DH;
}

// Eight codes (code i in byte i of the two dwords) to bf16, exactly, two an instruction.
__device__ __forceinline__ bf16x8 decode8(u32x2 w) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w.x, 1.f, false);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w.x, 1.f, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w.y, 1.f, false);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w.y, 1.f, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// What a pair of pages needs beside the products.
enum Cut {
  kNone,   // every row sees every key
  kLimit,  // keys past a row's limit count as -inf, and V of keys without data as 0
  kToken,  // the block's tokens see different keys of the pair
};

// RT row tiles of 16 a wave, RW waves side by side along the rows, the others along the
// pairs.  RW = 1: each wave loads its own pages.  RW = 2: two load the same, from HBM once and
// from L1 and L2 after that (no non-temporal hint then), where a block for each would have
// read them again.  RW = 4: the waves bring each page once, into LDS, and decode E4M3 once,
// which is worth its LDS traffic for bf16 pages and for two row tiles a wave (13 tokens, 52
// rows, over 16 x 4K to 16K: bf16 137 us with RW = 2, 118 with 4; E4M3 94 and 101; 26 tokens,
// each wave loading its own pages, 209 and 151, E4M3 150 and 138).
//
// Lane l: c16 = l % 16, q4 = l / 16.  The MFMA operand order is the one of the
// engine's decode attention: S^T = K Q^T with the keys permuted so that a lane's
// eight scores are eight consecutive tokens of one page (page q4 / 2 of the pair,
// tokens 8 (q4 % 2) ..), which is the P operand of O^T = V^T P^T against one load
// of the transposed V page.
template <int DH, int RT, int RW, typename KT, bool LIST>
__global__ __launch_bounds__(kThreads)
__attribute__((amdgpu_waves_per_eu(RW > 1 ? 2 : (sizeof(KT) == 1 ? 3 : 4) - RT))) void
paged_attn_kernel(
    PagedAttnArgs a, const int32_t* __restrict__ table, const int32_t* __restrict__ lists) {
  constexpr int KC = DH / 32, DT = DH / 16;
  constexpr bool kFp8 = sizeof(KT) == 1;
  // Whether the next pair's loads are in flight while one is used.  The registers that this
  // takes of bf16 pages cost a resident group, and more (64 x 1K to 8K: 179 us without, 188
  // with; four tokens over 16 x 1K to 16K: 97 and 102), and so do those of E4M3 pages where
  // two waves share them (13 tokens over 53 x 0.5K to 4K 105 without, 117 with).
  constexpr bool kStaged = RW == kWaves, kAhead = kFp8 && (RW == 1 || RT == 1);
  constexpr int PW = kWaves / RW;  // waves that share a row tile's pairs
  typedef typename std::conditional<kFp8, u32x2, u32x4>::type VRaw;
  __shared__ int red[kWaves];
  __shared__ int found[2];
  __shared__ float sm[PW > 1 ? (PW - 1) * RW : 1][64][PW > 1 ? RT * (4 * DT + 2) : 1];
  // kStaged: K and V^T of four pages in bf16, their scales and the positions of their first
  // keys, twice.  The 16-byte chunks of a K row lie exchanged by the token, so that the eight
  // lanes that read at once meet different banks.
  constexpr int kRegion = kPage * DH;
  __shared__ __attribute__((aligned(16))) uint16_t stage[2][kStaged ? 8 * kRegion : 8];
  __shared__ float scale[2][kStaged ? 8 : 1];
  __shared__ int place[2][kStaged ? 4 : 1];
  auto swz = [](int tok) { return (tok & 3) | (tok >> 1 & 4); };
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int c16 = lane & 15, q4 = lane >> 4;
  const int rw = wave % RW, pw = wave / RW, row0 = rw * RT * 16;
  const int g = blockIdx.x, w = blockIdx.y;
  const int G = a.n_q_heads / a.n_kv_heads;
  int at = 0, end, u = w, first = 0;
  if (a.unit_groups) {  // a group takes unit w whole
    end = unit_pairs(a, u);
    if (end == 0) {
      const int b = u / a.blocks_per_seq, j0 = u % a.blocks_per_seq * a.tok_per_block;
      const int rows = min(a.tok_per_block, a.n_q - j0) * G;
      for (int i = threadIdx.x; i < rows * (DH / 4); i += kThreads) {
        const int row = i / (DH / 4);
        *(u32x2*)((uint16_t*)a.out + row_at<DH>(a, b, j0, g, row) + i % (DH / 4) * 4) = u32x2{0, 0};
      }
      return;
    }
  } else {
    const Stretch mine = stretch_of<kThreads>(a.n_units, a.n_groups, a.min_pairs, w, red, found,
                                              [&](int v) { return unit_pairs(a, v); });
    at = w * mine.per;
    if (at >= mine.total) return;
    end = min(at + mine.per, mine.total);
    u = mine.unit;
    first = mine.first;
  }
  const uint16_t* q = (const uint16_t*)a.q;
  auto qk_dim = [](int c, int q4_) {
    return kFp8 && !kStaged ? q4_ * (DH / 4) + c * 8 : c * 32 + q4_ * 8;
  };
  const int k_tok = 8 * ((c16 >> 2) & 1) + (c16 & 3);  // + 4u
  const int k_sel = c16 >> 3, v_sel = q4 >> 1, v_tok0 = 8 * (q4 & 1);
  const int64_t page_stride = (int64_t)a.n_kv_heads * kPage * DH, head_off = (int64_t)g * kPage * DH;

  for (; at < end; ++u) {
    const int pairs = unit_pairs(a, u);
    if (first + pairs <= at) {  // empty unit
      first += pairs;
      continue;
    }
    const int b = u / a.blocks_per_seq, j0 = u % a.blocks_per_seq * a.tok_per_block;
    const int n_tok = min(a.tok_per_block, a.n_q - j0);
    const int len = clamp_len(a, b), pos0 = len - a.n_q + j0;  // position of token j0
    const int kv_lim = max(pos0 + n_tok, 0), n_pages = unit_pages(a, u);
    const int p_begin = at - first, p_end = min(pairs, end - first);

    bf16x8 qf[RT][KC];
    int row_lim[RT];  // keys a row sees (exclusive end); nothing for rows past the block's
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      const int row = row0 + t * 16 + c16, j = row / G;
      const bool on = j < n_tok;
      row_lim[t] = on ? pos0 + j + 1 : 0;
      const uint16_t* src = q + row_at<DH>(a, b, j0, g, row);
#pragma unroll
      for (int c = 0; c < KC; ++c)
        qf[t][c] = on ? *(const bf16x8*)(src + qk_dim(c, q4)) : bf16x8{};
    }
    float m[RT];
    f32x4 acc[RT][DT], sum[RT];  // sum: see `ones`
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      m[t] = -INFINITY;
      sum[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int d = 0; d < DT; ++d) acc[t][d] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    const int32_t* bt = table + (int64_t)b * a.bt_stride;
    const int32_t* list =
        LIST ? lists + ((int64_t)b * a.n_kv_heads + g) * a.n_selected : nullptr;
    // A page's place in the pool and the position of its first key.  One that the table or
    // the list does not name has no keys.  All uniform over the wave and from pointers of the
    // kernel's own that nothing aliases, so these are scalar loads: vector loads return in
    // order, so waiting for one would drain the pages' in flight (five tokens over 8 x 64K to
    // 128K: 326 us with both waits, 267 without).
    struct Spot {
      int page, key0;
    };
    auto spot = [&](int n) {
      int logical = n;
      if constexpr (LIST) logical = n < n_pages ? list[n] : -1;
      const bool in = LIST ? logical >= 0 && logical < a.bt_stride : n < n_pages;
      const int page = in ? bt[logical] : -1;
      const bool ok = page >= 0 && page < a.n_pages;
      return Spot{ok ? page : 0, ok ? logical * kPage : kNowhere};
    };
    struct Pair {
      Spot at[2];
    };
    auto look = [&](int pr) { return Pair{{spot(2 * pr), spot(2 * pr + 1)}}; };
    auto read = [](auto* p, auto v) {
      if constexpr (RW == 1) return load_stream<decltype(v)>(p);
      else return *(const decltype(v)*)p;
    };
    // The pair's bytes as they are in memory, and its scales.
    struct Raw {
      u32x4 k[2][kFp8 ? KC / 2 : KC];
      VRaw v[DT];
      float ks, vs;  // of the page of this lane's keys
      int key0[2];
    };
    auto load = [&](const Pair& p, Raw& r) {
      const int64_t base0 = p.at[0].page * page_stride + head_off;
      const int64_t base1 = p.at[1].page * page_stride + head_off;
      const KT* kb = (const KT*)a.k_pages + (k_sel ? base1 : base0);
      const KT* vb = (const KT*)a.v_pages + (v_sel ? base1 : base0) + v_tok0;
      // The scales come as vector loads, in order with the pages': scalar loads return out
      // of order, so that using one would wait for all, the next pair's among them.
      if constexpr (kFp8) {
        const int64_t at = (int64_t)(v_sel ? p.at[1].page : p.at[0].page) * a.n_kv_heads + g;
        r.ks = a.k_scales[at];
        r.vs = a.v_scales[at];
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        r.key0[i] = p.at[i].key0;
#pragma unroll
        for (int c = 0; c < (kFp8 ? KC / 2 : KC); ++c)
          r.k[i][c] = read(kb + (k_tok + 4 * i) * DH + qk_dim(kFp8 ? 2 * c : c, q4), u32x4{});
      }
#pragma unroll
      for (int d = 0; d < DT; ++d)
        r.v[d] = read(vb + (d * 16 + c16) * kPage, VRaw{});
    };
    // The pair as the products take it.
    struct Tile {
      bf16x8 k[2][KC];
      u16x8 v[DT];
      float ks, vs;
      int key0[2];
    };
    auto decode = [&](const Raw& r) {
      Tile o;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        o.key0[i] = r.key0[i];
#pragma unroll
        for (int c = 0; c < KC; ++c) {
          if constexpr (kFp8) {
            const u32x4 w4 = r.k[i][c / 2];
            o.k[i][c] = decode8(c % 2 ? u32x2{w4.z, w4.w} : u32x2{w4.x, w4.y});
          } else {
            o.k[i][c] = __builtin_bit_cast(bf16x8, r.k[i][c]);
          }
        }
      }
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        if constexpr (kFp8) o.v[d] = __builtin_bit_cast(u16x8, decode8(r.v[d]));
        else o.v[d] = __builtin_bit_cast(u16x8, r.v[d]);
      }
      o.ks = r.ks;
      o.vs = r.vs;
      return o;
    };
    // Pair p of a stage.  l is the lane, as a value that the compiler takes for new each time:
    // addresses kept over the loop would cost registers that the products need.
    auto fetch_k = [&](int st, int p, int l, Tile& o) {
      const int tok = 8 * (l >> 2 & 1) + (l & 3), x = (l >> 4 ^ swz(tok)) * 8;
      const uint16_t* at = stage[st] + (4 * p + 2 * (l >> 3 & 1)) * kRegion + tok * DH;
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int c = 0; c < KC; ++c)
          o.k[i][c] = *(const bf16x8*)(at + (x ^ (c & 1) * 32) + i * 4 * DH + (c >> 1) * 64);
    };
    auto fetch_v = [&](int st, int p, int l, Tile& o) {
      const uint16_t* at = stage[st] + (4 * p + 2 * (l >> 5) + 1) * kRegion +
                           (l & 15) * kPage + (l >> 1 & 8);
#pragma unroll
      for (int i = 0; i < 2; ++i) o.key0[i] = __builtin_amdgcn_readfirstlane(place[st][2 * p + i]);
      o.ks = kFp8 ? scale[st][4 * p + 2 * (l >> 5)] : 1.f;
      o.vs = kFp8 ? scale[st][4 * p + 2 * (l >> 5) + 1] : 1.f;
#pragma unroll
      for (int d = 0; d < DT; ++d) o.v[d] = *(const u16x8*)(at + d * 16 * kPage);
    };
    auto products = [&](const Tile& r, int t, f32x4* s) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        s[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < KC; ++c)
          s[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(r.k[i][c], qf[t][c], s[i], 0, 0, 0);
      }
    };
    auto use = [&](Tile r, auto scores, auto cut_) {
      constexpr Cut kCut = decltype(cut_)::value;
      auto& vf = r.v;
      const int kbase = (v_sel ? r.key0[1] : r.key0[0]) + v_tok0;  // position of this lane's key 0
      // Scales of pages without keys (of page 0, which stands in for no page, or of one that
      // is listed from behind the length) may be anything.
      const bool scaled = kFp8 && kbase < kv_lim;
      // A scale of 0 would meet -inf (masked scores, its logarithm) and its inverse: what lies
      // below the least scale that the append writes counts as that one.
      const float k_mul = scaled ? a.scale_log2 * max2(r.ks, kMinScale) : a.scale_log2;
      const float v_mul = scaled ? max2(r.vs, kMinScale) : 1.f;
      const float v_log = kFp8 ? __builtin_amdgcn_logf(v_mul) : 0.f;
      // The weights' sum is a product too, by rows of ones, or of the inverse of the V scale
      // that the weights carry: its high half in even rows and the rest in odd ones (2^-16
      // of it is lost), so that a lane's first two results add up to its row's sum.
      u32x4 ones;
      {
        const float inv = kFp8 ? __builtin_amdgcn_rcpf(v_mul) : 1.f;
        uint32_t bits = __float_as_uint(inv) & 0xFFFF0000u;
        if constexpr (kFp8)
          if (c16 & 1) bits = __float_as_uint(inv - __uint_as_float(bits)) & 0xFFFF0000u;
        bits |= bits >> 16;
        ones = u32x4{bits, bits, bits, bits};
      }
      // Keys without data: 0 times what they hold may be NaN.  (Uniform over the wave;
      // with kNone only where the table names no page.)
      const bool hole = max(r.key0[0], r.key0[1]) + kPage > kv_lim;
      if (kCut == kToken || hole) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (kbase + e >= kv_lim)
#pragma unroll
            for (int d = 0; d < DT; ++d) vf[d][e] = 0;
      }
      // Whether a weight of 0 leaves nothing of any key: 0 times all of V is 0 unless
      // something in it is infinite or NaN.
      bool finite = true;
      if constexpr (kCut == kToken) {
        f32x4 z = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int d = 0; d < DT; ++d)
          z = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vf[d]), bf16x8{},
                                                      z, 0, 0, 0);
        finite = !__any(z[0] + z[1] + z[2] + z[3] != 0.f);
      }
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        f32x4 s[2];
        scores(r, t, s);
        if (kCut == kNone && hole) {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (kbase >= kNowhere) s[e / 4][e % 4] = -INFINITY;
        }
        auto seen = [&](int e) { return kCut == kNone || kbase + e < row_lim[t]; };
        float mloc = -INFINITY;
#pragma unroll
        for (int e = 0; e < 8; ++e) mloc = fmaxf(mloc, seen(e) ? s[e / 4][e % 4] : -INFINITY);
        mloc = max_over_key_groups(mloc * k_mul);  // a lane's keys are of one page
        const float m_new = fmaxf(m[t], mloc), m_use = m_new == -INFINITY ? 0.f : m_new;
        if (__any(m_new != m[t])) {
          const float alpha = __builtin_amdgcn_exp2f(m[t] - m_use);
          sum[t][0] *= alpha;
          if constexpr (kFp8) sum[t][1] *= alpha;
#pragma unroll
          for (int d = 0; d < DT; ++d) acc[t][d] *= alpha;
        }
        m[t] = m_new;
        // The weights enter the second product in bf16, each off by at most half a step
        // (2^-8), a page's V scale with them: its logarithm (exact for powers of two, else
        // within 2^-18) less the row's maximum, which rounds the exponent by half a step of the
        // difference (2^-17 where that is 128 to 256); the normaliser is the fp32 sum of the
        // weights as they were rounded, so that what the rounding does to a row's large weights
        // cancels.
        const float base = v_log - m_use;
        uint32_t pw[4];
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
          const float x0 = __builtin_fmaf(s[e / 4][e % 4], k_mul, base);
          const float x1 = __builtin_fmaf(s[e / 4][e % 4 + 1], k_mul, base);
          const f32x2 pv = {__builtin_amdgcn_exp2f(seen(e) ? x0 : -INFINITY),
                            __builtin_amdgcn_exp2f(seen(e + 1) ? x1 : -INFINITY)};
          pw[e / 2] = __builtin_bit_cast(uint32_t, __builtin_convertvector(pv, bf16x2));
        }
        const u16x8 pbits = __builtin_bit_cast(u16x8, u32x4{pw[0], pw[1], pw[2], pw[3]});
        sum[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
            __builtin_bit_cast(bf16x8, ones), __builtin_bit_cast(bf16x8, pbits), sum[t], 0, 0, 0);
        if constexpr (kCut == kToken) {
          // Keys that some of the block's tokens do not see: token by token, with the
          // keys past its own taken as 0 and the sums of its rows alone, since a weight
          // of 0 times an infinity in V would not be 0.  All at once where V is finite.
          const int r0 = row0 + t * 16, j_begin = r0 / G;
          const int j_end = finite ? j_begin + 1 : min((r0 + 15) / G + 1, n_tok);
          for (int j = j_begin; j < j_end; ++j) {
            const bool mine = finite || (r0 + c16) / G == j;
            const int own = finite ? kNowhere : pos0 + j;
#pragma unroll
            for (int d = 0; d < DT; ++d) {
              u16x8 v = vf[d];
#pragma unroll
              for (int e = 0; e < 8; ++e)
                if (kbase + e > own) v[e] = 0;
              const f32x4 o = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                  __builtin_bit_cast(bf16x8, v), __builtin_bit_cast(bf16x8, pbits), acc[t][d], 0, 0, 0);
              acc[t][d] = mine ? o : acc[t][d];
            }
          }
        } else {
          const bf16x8 pf = __builtin_bit_cast(bf16x8, pbits);
#pragma unroll
          for (int d = 0; d < DT; ++d)
            acc[t][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vf[d]),
                                                                pf, acc[t][d], 0, 0, 0);
        }
      }
    };
    auto attend = [&](const Tile& r, auto cut) { use(r, products, cut); };
    // Pairs that every row sees whole, and the one or few at the block's end.  A list's
    // pages come in any order: each pair looks whether its keys end.
    const int p_cut = LIST ? p_end : min(p_end, max(max(pos0 + 1, 0) / kPair, p_begin));
    int pr = p_begin + pw;
    typedef std::integral_constant<Cut, LIST ? kLimit : kNone> Main;
    if constexpr (kStaged) {
      // A stage is two pairs, of which wave w brings page w: loads into registers, one stage
      // ahead, and from there, E4M3 decoded on the way, into the one of the two in LDS that is
      // not in use.
      constexpr int LP = kRegion * sizeof(KT) / 1024, EL = 16 / sizeof(KT);  // loads; elements
      const int last = 2 * p_end - 1;
      auto lane_now = [&] {
        int l = threadIdx.x & 63;
        asm volatile("" : "+v"(l));
        return l;
      };
      auto ahead = [&](int p) { return spot(min(2 * p + wave, last)); };
      u32x4 part[2][LP];
      float part_scale[2];
      int part_key0;
      auto load = [&](const Spot& at) {
        const int64_t from = at.page * page_stride + head_off + lane * EL;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const KT* src = (const KT*)(i ? a.v_pages : a.k_pages) + from;
#pragma unroll
          for (int j = 0; j < LP; ++j) part[i][j] = load_stream<u32x4>(src + j * 64 * EL);
          if constexpr (kFp8)
            part_scale[i] = (i ? a.v_scales : a.k_scales)[(int64_t)at.page * a.n_kv_heads + g];
        }
        part_key0 = at.key0;
      };
      auto put = [&](int st, int l) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          uint16_t* to = stage[st] + (2 * wave + i) * kRegion;
#pragma unroll
          for (int j = 0; j < LP; ++j) {
            const int n = (j * 64 + l) * EL, x = i ? n : n ^ swz(n / DH) * 8;
            if constexpr (kFp8) {
              *(bf16x8*)(to + x) = decode8(u32x2{part[i][j].x, part[i][j].y});
              *(bf16x8*)(to + (x ^ 8)) = decode8(u32x2{part[i][j].z, part[i][j].w});
            } else {
              *(u32x4*)(to + x) = part[i][j];
            }
          }
        }
        if (l == 0) {
          if constexpr (kFp8) {
            scale[st][2 * wave] = part_scale[0];
            scale[st][2 * wave + 1] = part_scale[1];
          }
          place[st][wave] = part_key0;
        }
      };
      auto one = [&](int st, int p, auto cut) {
        Tile r;
        f32x4 s[RT][2];
        fetch_k(st, p, lane_now(), r);
#pragma unroll
        for (int t = 0; t < RT; ++t) products(r, t, s[t]);
        __builtin_amdgcn_sched_barrier(0);  // K's registers are V's now
        fetch_v(st, p, lane_now(), r);
        use(r, [&](const Tile&, int t, f32x4* o) { o[0] = s[t][0], o[1] = s[t][1]; }, cut);
      };
      load(ahead(p_begin));
      __syncthreads();  // the unit before has been used
      put(0, lane);
      load(ahead(p_begin + 2));
      Spot next = ahead(p_begin + 4);
      int st = 0, p = p_begin;
      auto turn = [&](auto cut) {
        wg_barrier();
        put(st ^ 1, lane_now());
        load(next);
        next = ahead(p + 6);
#pragma unroll
        for (int i = 0; i < 2; ++i)
          if (decltype(cut)::value == kNone || p + i < p_end) one(st, i, cut);
        st ^= 1;
        p += 2;
      };
      while (p + 2 <= p_cut) turn(std::integral_constant<Cut, kNone>{});
      while (p < p_end) turn(std::integral_constant<Cut, kToken>{});
    } else if constexpr (kAhead) {
      // The next pair's bytes are in flight while one is used, in two buffers in turn, and
      // the page after it is looked up.  Past the end the last pair stands in.  (A third
      // buffer, and refilling each behind its use, measured the same or up to 8% slower.)
      if (pr < p_cut) {
        auto next = [&](int i) { return i + PW < p_cut ? i + PW : i; };
        Raw r[2];
        load(look(pr), r[0]);
        int fetch = next(pr);
        Pair ahead = look(fetch);
        for (bool more = true; more;) {
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            load(ahead, r[1 - i]);
            fetch = next(fetch);
            ahead = look(fetch);
            __builtin_amdgcn_sched_barrier(0);
            attend(decode(r[i]), Main{});
            pr += PW;
            more = pr < p_cut;
            if (!more) break;
          }
        }
      }
    } else {
      for (; pr < p_cut; pr += PW) {
        Raw r;
        load(look(pr), r);
        attend(decode(r), Main{});
      }
    }
    if constexpr (!LIST && !kStaged) {
      for (; pr < p_end; pr += PW) {
        Raw r;
        load(look(pr), r);
        attend(decode(r), std::integral_constant<Cut, kToken>{});
      }
    }

    // The partials of the waves that share a row tile meet in the first of them, in wave
    // order.
    float l[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) l[t] = kFp8 ? sum[t][0] + sum[t][1] : sum[t][0];
    if constexpr (PW > 1) {
      __syncthreads();  // the piece before has been read
      if (pw > 0) {
        float* d = sm[(pw - 1) * RW + rw][lane];
#pragma unroll
        for (int t = 0; t < RT; ++t) {
          d[t * (4 * DT + 2)] = m[t];
          d[t * (4 * DT + 2) + 1] = l[t];
#pragma unroll
          for (int i = 0; i < 4 * DT; ++i) d[t * (4 * DT + 2) + 2 + i] = acc[t][i / 4][i % 4];
        }
      }
      __syncthreads();
    }
    if (pw == 0) {
      const bool whole = p_begin == 0 && p_end == pairs;
#pragma unroll
      for (int t = 0; t < RT; ++t) {
#pragma unroll
        for (int v = 0; v < PW - 1; ++v) {
          const float* d = sm[v * RW + rw][lane] + t * (4 * DT + 2);
          const float mn = fmaxf(m[t], d[0]), mu = mn == -INFINITY ? 0.f : mn;
          const float so = exp2f(m[t] - mu), sw = exp2f(d[0] - mu);
          l[t] = l[t] * so + d[1] * sw;
#pragma unroll
          for (int i = 0; i < 4 * DT; ++i)
            acc[t][i / 4][i % 4] = acc[t][i / 4][i % 4] * so + d[2 + i] * sw;
          m[t] = mn;
        }
        const int row = row0 + t * 16 + c16, j = row / G;
        if (j >= n_tok) continue;
        if (whole) {
          const float inv = l[t] == 0.f ? 0.f : 1.f / l[t];
          uint16_t* o = (uint16_t*)a.out + row_at<DH>(a, b, j0, g, row);
#pragma unroll
          for (int d = 0; d < DT; ++d) {
            const f32x2 lo = {acc[t][d][0] * inv, acc[t][d][1] * inv};
            const f32x2 hi = {acc[t][d][2] * inv, acc[t][d][3] * inv};
            *(u32x2*)(o + d * 16 + 4 * q4) =
                u32x2{__builtin_bit_cast(uint32_t, __builtin_convertvector(lo, bf16x2)),
                      __builtin_bit_cast(uint32_t, __builtin_convertvector(hi, bf16x2))};
          }
        } else {
          const int64_t pr = (((int64_t)w + u) * a.n_kv_heads + g) * (16 * RT * RW) + row;
          if (q4 == 0) {
            a.part_ml[pr * 2] = m[t];
            a.part_ml[pr * 2 + 1] = l[t];
          }
#pragma unroll
          for (int d = 0; d < DT; ++d) *(f32x4*)(a.part_acc + pr * DH + d * 16 + 4 * q4) = acc[t][d];
        }
      }
    }
    at = first + p_end;
    first += pairs;
  }
}

// Merges the pieces of each unit, and writes zeros for the rows of a unit that sees
// no key.  A work group per (unit, KV head, four rows): 16 lanes a row, wave v taking
// pieces v, v + 4, .. in order, four loads of each in flight, then the four results in
// wave order.
template <int DH>
__global__ __launch_bounds__(kThreads) void paged_merge_kernel(PagedAttnArgs a, int rows_per_unit) {
  constexpr int DPL = DH / 16;
  __shared__ int red[2][kWaves];
  __shared__ float sh[kWaves - 1][64][DPL + 2];
  const int u = blockIdx.x, g = blockIdx.y, G = a.n_q_heads / a.n_kv_heads;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  int all = 0, before = 0;
  for (int v = threadIdx.x; v < a.n_units; v += kThreads) {
    const int n = unit_pairs(a, v);
    all += n;
    before += v < u ? n : 0;
  }
  all = wave_add(all);
  before = wave_add(before);
  if (lane == 0) {
    red[0][wave] = all;
    red[1][wave] = before;
  }
  __syncthreads();
  const int total = red[0][0] + red[0][1] + red[0][2] + red[0][3];
  const int first = red[1][0] + red[1][1] + red[1][2] + red[1][3];
  const int per = max((total + a.n_groups - 1) / a.n_groups, a.min_pairs);
  const int pairs = unit_pairs(a, u), w0 = first / per;
  const int w1 = pairs > 0 ? (first + pairs - 1) / per : w0 - 1;
  if (pairs > 0 && w0 == w1) return;
  const int b = u / a.blocks_per_seq, j0 = u % a.blocks_per_seq * a.tok_per_block;
  const int rows = min(a.tok_per_block, a.n_q - j0) * G, row = blockIdx.z * 4 + lane / 16;
  if (blockIdx.z * 4 >= rows) return;
  const int d0 = (lane & 15) * DPL, r = min(row, rows - 1);
  float m = -INFINITY, l = 0.f, o[DPL];
#pragma unroll
  for (int e = 0; e < DPL; ++e) o[e] = 0.f;
  auto join = [&](float mi, float li, const float* oi) {
    const float mn = fmaxf(m, mi), mu = mn == -INFINITY ? 0.f : mn;
    const float so = exp2f(m - mu), si = exp2f(mi - mu);
    l = l * so + li * si;
#pragma unroll
    for (int e = 0; e < DPL; ++e) o[e] = o[e] * so + oi[e] * si;
    m = mn;
  };
  for (int w = w0 + wave; w <= w1; w += 4 * kWaves) {
    float2 ml[4];
    float x[4][DPL];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t pr =
          (((int64_t)min(w + i * kWaves, w1) + u) * a.n_kv_heads + g) * rows_per_unit + r;
      ml[i] = *(const float2*)(a.part_ml + pr * 2);
#pragma unroll
      for (int e = 0; e < DPL; e += 4) *(f32x4*)(x[i] + e) = *(const f32x4*)(a.part_acc + pr * DH + d0 + e);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (w + i * kWaves <= w1) join(ml[i].x, ml[i].y, x[i]);
  }
  if (wave > 0) {
    float* d = sh[wave - 1][lane];
    d[0] = m;
    d[1] = l;
#pragma unroll
    for (int e = 0; e < DPL; ++e) d[2 + e] = o[e];
  }
  __syncthreads();
  if (wave > 0 || row >= rows) return;
#pragma unroll
  for (int v = 0; v < kWaves - 1; ++v) join(sh[v][lane][0], sh[v][lane][1], &sh[v][lane][2]);
  const float inv = l == 0.f ? 0.f : 1.f / l;
  uint16_t* dst = (uint16_t*)a.out + row_at<DH>(a, b, j0, g, row) + d0;
#pragma unroll
  for (int e = 0; e < DPL; e += 4) {
    const f32x2 lo = {o[e] * inv, o[e + 1] * inv}, hi = {o[e + 2] * inv, o[e + 3] * inv};
    *(u32x2*)(dst + e) = u32x2{__builtin_bit_cast(uint32_t, __builtin_convertvector(lo, bf16x2)),
                               __builtin_bit_cast(uint32_t, __builtin_convertvector(hi, bf16x2))};
  }
}

}  // namespace

hipError_t launch_paged_attention(int kv_fp8, int head_dim, int row_tiles, const PagedAttnArgs& a,
                                  hipStream_t stream) {
  const dim3 grid(a.n_kv_heads, a.unit_groups ? a.n_units : a.n_groups), block(kThreads);
  const PagedAttnForm f = paged_attention_form(kv_fp8, head_dim, row_tiles, a.n_units, a.max_len,
                                               a.n_kv_heads);
#define PDEC_PAGED(DH_, RT_, RW_, KT_, LIST_)                          \
  paged_attn_kernel<DH_, RT_, RW_, KT_, LIST_><<<grid, block, 0, stream>>>(a, a.block_table, \
                                                                           a.selected)
#define PDEC_PAGED_RT(DH_, KT_)                                  \
  do {                                                           \
    if (a.selected) PDEC_PAGED(DH_, 1, 1, KT_, true);            \
    else if (f.waves == 4 && f.tiles == 1) PDEC_PAGED(DH_, 1, 4, uint16_t, false); \
    else if (f.waves == 4) PDEC_PAGED(DH_, 2, 4, KT_, false);    \
    else if (f.waves == 2 && f.tiles == 2) PDEC_PAGED(DH_, 2, 2, uint8_t, false); \
    else if (f.waves == 2) PDEC_PAGED(DH_, 1, 2, KT_, false);    \
    else if (f.tiles == 2) PDEC_PAGED(DH_, 2, 1, KT_, false);    \
    else PDEC_PAGED(DH_, 1, 1, KT_, false);                      \
  } while (0)
  if (head_dim == 128) {
    if (kv_fp8) PDEC_PAGED_RT(128, uint8_t);
    else PDEC_PAGED_RT(128, uint16_t);
  } else {
    if (kv_fp8) PDEC_PAGED_RT(64, uint8_t);
    else PDEC_PAGED_RT(64, uint16_t);
  }
#undef PDEC_PAGED_RT
#undef PDEC_PAGED
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.unit_groups) return e;
  const int rows = std::min(a.tok_per_block, a.n_q) * (a.n_q_heads / a.n_kv_heads);
  const dim3 mgrid(a.n_units, a.n_kv_heads, (rows + 3) / 4);
  if (head_dim == 128)
    paged_merge_kernel<128><<<mgrid, block, 0, stream>>>(a, 16 * row_tiles);
  else
    paged_merge_kernel<64><<<mgrid, block, 0, stream>>>(a, 16 * row_tiles);
  return hipGetLastError();
}

}  // namespace pdec
