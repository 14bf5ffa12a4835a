// Attention of one or several query tokens per sequence over caller-owned pages,
// with the sequence lengths on the device.
//
//   out[b][j][h] = softmax(q[b][j][h] . K^T / sqrt(Dh)) V  over positions
//   0 .. lens[b] - n_q + j of sequence b (query token j's own position among
//   them), or over the pages that `selected` lists for (b, KV head).
//
// K and V pages are bf16, or E4M3 codes with a scale for each page and KV head.
// Every cached byte is read once for all of a KV head's query rows, so the call is
// bound by HBM up to a few hundred rows per head.
//
// Work split.  A unit is a block of query tokens of one sequence (their n_tok * G
// rows, at most 16 RT); its work is its key range in pairs of pages.  The units' pairs
// laid end to end are cut into n_groups equal stretches, one for each work group of a
// KV head, whatever the lengths: a group finds its stretch from a prefix sum of the
// lengths that it makes itself, so no plan is built on the host or uploaded, and a
// captured graph follows lengths that change on the device.  A stretch may cover the end of
// one unit and the beginning of the next: the piece of unit u in group w leaves its
// softmax partial (maximum, sum, unnormalised output) in slot w + u, which no other
// piece has, and the merge pass finds a unit's pieces side by side.  A unit that one
// group covers whole is written out at once.
#include "hip_common.h"
#include "kernels.h"

#include <algorithm>

namespace pdec {

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kThreads = 256, kWaves = 4;
constexpr int kPair = 2 * kPage;        // keys of a pair of pages
constexpr int kNowhere = 0x40000000;    // a key position past every limit

// Sizes of a call that both passes derive their split from.
struct Split {
  int total;  // pairs of pages of all units
  int per;    // pairs per work group
};

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

__device__ __forceinline__ int wave_scan(int v) {  // inclusive
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int t = __shfl_up(v, o, 64);
    if (lane >= o) v += t;
  }
  return v;
}

// Sum of v over the work group's threads before this one, and of all of them.
__device__ __forceinline__ int group_scan(int v, int* red, int* total) {
  const int incl = wave_scan(v), wave = threadIdx.x >> 6, nw = blockDim.x >> 6;
  __syncthreads();
  if ((threadIdx.x & 63) == 63) red[wave] = incl;
  __syncthreads();
  int before = incl - v, sum = 0;
  for (int w = 0; w < nw; ++w) {
    before += w < wave ? red[w] : 0;
    sum += red[w];
  }
  *total = sum;
  return before;
}

__device__ __forceinline__ Split split_of(const PagedAttnArgs& a, int* red) {
  int mine = 0, total;
  for (int u = threadIdx.x; u < a.n_units; u += blockDim.x) mine += unit_pairs(a, u);
  group_scan(mine, red, &total);
  return {total, max((total + a.n_groups - 1) / a.n_groups, a.min_pairs)};
}

// The unit that pair `at` (< total) belongs to and its first pair, to all threads.
__device__ __forceinline__ void find_unit(const PagedAttnArgs& a, int at, int* red, int* found) {
  int base = 0;
  for (int u0 = 0; u0 < a.n_units; u0 += blockDim.x) {
    const int u = u0 + threadIdx.x, n = u < a.n_units ? unit_pairs(a, u) : 0;
    int total;
    const int first = base + group_scan(n, red, &total);
    if (first <= at && at < first + n) {
      found[0] = u;
      found[1] = first;
    }
    base += total;
    if (base > at) break;
  }
  __syncthreads();
}

template <typename KT>
__device__ __forceinline__ bf16x8 load8(const KT* p) {
  if constexpr (sizeof(KT) == 2) return load_stream<bf16x8>(p);
  else return e4m3x8_to_bf16(load_stream<u32x2>(p));
}

// Lane l: c16 = l % 16, q4 = l / 16.  The MFMA operand order is the one of the
// engine's decode attention: S^T = K Q^T with the keys permuted so that a lane's
// eight scores are eight consecutive tokens of one page (page q4 / 2 of the pair,
// tokens 8 (q4 % 2) ..), which is the P operand of O^T = V^T P^T against one load
// of the transposed V page.
template <int DH, int RT, typename KT, bool LIST>
__global__ __launch_bounds__(kThreads) void paged_attn_kernel(PagedAttnArgs a) {
  constexpr int KC = DH / 32, DT = DH / 16;
  constexpr bool kFp8 = sizeof(KT) == 1;
  __shared__ int red[kWaves];
  __shared__ int found[2];
  __shared__ float sm[kWaves - 1][64][RT * (4 * DT + 2)];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int c16 = lane & 15, q4 = lane >> 4;
  const int g = blockIdx.x, w = blockIdx.y;
  const Split split = split_of(a, red);
  int at = w * split.per;
  if (at >= split.total) return;
  const int end = min(at + split.per, split.total);
  find_unit(a, at, red, found);
  int u = found[0], first = found[1];
  const int G = a.n_q_heads / a.n_kv_heads;
  const uint16_t* q = (const uint16_t*)a.q;
  auto qk_dim = [](int c, int q4_) { return kFp8 ? q4_ * (DH / 4) + c * 8 : c * 32 + q4_ * 8; };
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
      const int row = t * 16 + c16, j = row / G;
      const bool on = j < n_tok;
      row_lim[t] = on ? pos0 + j + 1 : 0;
      const uint16_t* src =
          q + (((int64_t)b * a.n_q + j0 + j) * a.n_q_heads + g * G + row % G) * DH;
#pragma unroll
      for (int c = 0; c < KC; ++c)
        qf[t][c] = on ? *(const bf16x8*)(src + qk_dim(c, q4)) : bf16x8{};
    }
    float m[RT], l[RT];
    f32x4 acc[RT][DT];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      m[t] = -INFINITY;
      l[t] = 0.f;
#pragma unroll
      for (int d = 0; d < DT; ++d) acc[t][d] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    const int32_t* bt = a.block_table + (int64_t)b * a.bt_stride;
    const int32_t* list =
        LIST ? a.selected + ((int64_t)b * a.n_kv_heads + g) * a.n_selected : nullptr;
    // Page i of the unit: its place in the pool and the position of its first key.
    // An entry that names no page of the pool has no keys.
    auto page_at = [&](int i, int* key0) -> int {
      int logical = i;
      if constexpr (LIST) logical = i < n_pages ? list[i] : -1;
      const bool in = LIST ? logical >= 0 && logical < a.bt_stride : i < n_pages;
      const int page = in ? bt[logical] : -1;
      const bool ok = page >= 0 && page < a.n_pages;
      *key0 = ok ? logical * kPage : kNowhere;
      return ok ? page : 0;
    };

    for (int pr = p_begin + wave; pr < p_end; pr += kWaves) {
      int key0[2];
      const int page0 = page_at(2 * pr, &key0[0]), page1 = page_at(2 * pr + 1, &key0[1]);
      const int64_t base0 = page0 * page_stride + head_off, base1 = page1 * page_stride + head_off;
      const KT* kb = (const KT*)a.k_pages + (k_sel ? base1 : base0);
      const KT* vb = (const KT*)a.v_pages + (v_sel ? base1 : base0) + v_tok0;
      float k_mul = a.scale_log2, v_mul = 1.f;
      if constexpr (kFp8) {
        const int64_t at0 = (int64_t)page0 * a.n_kv_heads + g, at1 = (int64_t)page1 * a.n_kv_heads + g;
        k_mul *= v_sel ? a.k_scales[at1] : a.k_scales[at0];
        v_mul = v_sel ? a.v_scales[at1] : a.v_scales[at0];
      }
      bf16x8 kf[2][KC];
      u16x8 vf[DT];
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int c = 0; c < KC; ++c) kf[i][c] = load8<KT>(kb + (k_tok + 4 * i) * DH + qk_dim(c, q4));
#pragma unroll
      for (int d = 0; d < DT; ++d)
        vf[d] = __builtin_bit_cast(u16x8, load8<KT>(vb + (d * 16 + c16) * kPage));

      const int kbase = (v_sel ? key0[1] : key0[0]) + v_tok0;  // position of this lane's key 0
      const int pair_end = max(key0[0], key0[1]) + kPage;      // uniform over the wave
      if (pair_end > kv_lim) {  // keys without data: 0 times what they hold may be NaN
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (kbase + e >= kv_lim)
#pragma unroll
            for (int d = 0; d < DT; ++d) vf[d][e] = 0;
      }
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        f32x4 s[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          s[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int c = 0; c < KC; ++c)
            s[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[i][c], qf[t][c], s[i], 0, 0, 0);
        }
        float sv[8], mloc = -INFINITY;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          sv[e] = kbase + e < row_lim[t] ? s[e / 4][e % 4] * k_mul : -INFINITY;
          mloc = fmaxf(mloc, sv[e]);
        }
        mloc = max_over_key_groups(mloc);
        const float m_new = fmaxf(m[t], mloc), m_use = m_new == -INFINITY ? 0.f : m_new;
        if (__any(m_new != m[t])) {
          const float alpha = __builtin_amdgcn_exp2f(m[t] - m_use);
          l[t] *= alpha;
#pragma unroll
          for (int d = 0; d < DT; ++d) acc[t][d] *= alpha;
        }
        m[t] = m_new;
        // The weights enter the second product in bf16 (half a step, 2^-9 of each,
        // as the values are E4M3 or bf16 themselves); their sum is kept in fp32.  A
        // page's V scale goes into its weights.
        uint32_t pw[4];
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
          const float p0 = __builtin_amdgcn_exp2f(sv[e] - m_use);
          const float p1 = __builtin_amdgcn_exp2f(sv[e + 1] - m_use);
          l[t] += p0 + p1;
          const f32x2 pv = {kFp8 ? p0 * v_mul : p0, kFp8 ? p1 * v_mul : p1};
          pw[e / 2] = __builtin_bit_cast(uint32_t, __builtin_convertvector(pv, bf16x2));
        }
        const u16x8 pbits = __builtin_bit_cast(u16x8, u32x4{pw[0], pw[1], pw[2], pw[3]});
        if (pair_end > pos0 + 1 && n_tok > 1) {
          // Keys that some of the block's tokens do not see: token by token, with the
          // keys past its own taken as 0 and the sums of its rows alone, since a weight
          // of 0 times an infinity in V would not be 0.
          for (int j = 0; j < n_tok; ++j) {
            const bool mine = (t * 16 + c16) / G == j;
#pragma unroll
            for (int d = 0; d < DT; ++d) {
              u16x8 v = vf[d];
#pragma unroll
              for (int e = 0; e < 8; ++e)
                if (kbase + e > pos0 + j) v[e] = 0;
              const f32x4 r = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                  __builtin_bit_cast(bf16x8, v), __builtin_bit_cast(bf16x8, pbits), acc[t][d], 0, 0, 0);
              acc[t][d] = mine ? r : acc[t][d];
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
    }

    // The waves' partials meet in wave 0, in wave order.
#pragma unroll
    for (int t = 0; t < RT; ++t) l[t] = sum_over_key_groups(l[t]);
    __syncthreads();  // the piece before has been read
    if (wave > 0) {
      float* d = sm[wave - 1][lane];
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        d[t * (4 * DT + 2)] = m[t];
        d[t * (4 * DT + 2) + 1] = l[t];
#pragma unroll
        for (int i = 0; i < 4 * DT; ++i) d[t * (4 * DT + 2) + 2 + i] = acc[t][i / 4][i % 4];
      }
    }
    __syncthreads();
    if (wave == 0) {
      const bool whole = p_begin == 0 && p_end == pairs;
#pragma unroll
      for (int t = 0; t < RT; ++t) {
#pragma unroll
        for (int v = 0; v < kWaves - 1; ++v) {
          const float* d = sm[v][lane] + t * (4 * DT + 2);
          const float mn = fmaxf(m[t], d[0]), mu = mn == -INFINITY ? 0.f : mn;
          const float so = exp2f(m[t] - mu), sw = exp2f(d[0] - mu);
          l[t] = l[t] * so + d[1] * sw;
#pragma unroll
          for (int i = 0; i < 4 * DT; ++i)
            acc[t][i / 4][i % 4] = acc[t][i / 4][i % 4] * so + d[2 + i] * sw;
          m[t] = mn;
        }
        const int row = t * 16 + c16, j = row / G;
        if (j >= n_tok) continue;
        if (whole) {
          const float inv = l[t] == 0.f ? 0.f : 1.f / l[t];
          uint16_t* o = (uint16_t*)a.out +
                        (((int64_t)b * a.n_q + j0 + j) * a.n_q_heads + g * G + row % G) * DH;
#pragma unroll
          for (int d = 0; d < DT; ++d) {
            const f32x2 lo = {acc[t][d][0] * inv, acc[t][d][1] * inv};
            const f32x2 hi = {acc[t][d][2] * inv, acc[t][d][3] * inv};
            *(u32x2*)(o + d * 16 + 4 * q4) =
                u32x2{__builtin_bit_cast(uint32_t, __builtin_convertvector(lo, bf16x2)),
                      __builtin_bit_cast(uint32_t, __builtin_convertvector(hi, bf16x2))};
          }
        } else {
          const int64_t pr = (((int64_t)w + u) * a.n_kv_heads + g) * (16 * RT) + row;
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
// no key.  A work group per (unit, KV head); 16 lanes a row, pieces in slot order.
template <int DH>
__global__ __launch_bounds__(kThreads) void paged_merge_kernel(PagedAttnArgs a, int rows_per_unit) {
  constexpr int DPL = DH / 16;
  __shared__ int red[kWaves];
  const int u = blockIdx.x, g = blockIdx.y, G = a.n_q_heads / a.n_kv_heads;
  const Split split = split_of(a, red);
  int mine = 0, first;
  for (int v = threadIdx.x; v < u; v += blockDim.x) mine += unit_pairs(a, v);
  group_scan(mine, red, &first);
  const int pairs = unit_pairs(a, u), w0 = first / split.per;
  const int w1 = (first + pairs - 1) / split.per;
  if (pairs > 0 && w0 == w1) return;
  const int b = u / a.blocks_per_seq, j0 = u % a.blocks_per_seq * a.tok_per_block;
  const int rows = min(a.tok_per_block, a.n_q - j0) * G;
  const int d0 = (threadIdx.x & 15) * DPL;
  for (int row = threadIdx.x / 16; row < rows; row += kThreads / 16) {
    float m = -INFINITY, l = 0.f, o[DPL];
#pragma unroll
    for (int e = 0; e < DPL; ++e) o[e] = 0.f;
    if (pairs > 0) {
      for (int w = w0; w <= w1; ++w) {
        const int64_t pr = (((int64_t)w + u) * a.n_kv_heads + g) * rows_per_unit + row;
        const float mi = a.part_ml[pr * 2], li = a.part_ml[pr * 2 + 1];
        const float mn = fmaxf(m, mi), mu = mn == -INFINITY ? 0.f : mn;
        const float so = exp2f(m - mu), si = exp2f(mi - mu);
        l = l * so + li * si;
#pragma unroll
        for (int e = 0; e < DPL; ++e) o[e] = o[e] * so + a.part_acc[pr * DH + d0 + e] * si;
        m = mn;
      }
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    uint16_t* dst = (uint16_t*)a.out +
                    (((int64_t)b * a.n_q + j0 + row / G) * a.n_q_heads + g * G + row % G) * DH + d0;
#pragma unroll
    for (int e = 0; e < DPL; ++e) dst[e] = f32_to_bf16(o[e] * inv);
  }
}

}  // namespace

// Row tiles per block of query rows.
static int row_tiles(int n_q, int group) {
  const int rows = n_q * group;
  return rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
}

PagedAttnPlan plan_paged_attention(int batch, int n_q, int n_q_heads, int n_kv_heads) {
  PagedAttnPlan p;
  const int G = n_q_heads / n_kv_heads;
  p.row_tiles = row_tiles(n_q, G);
  p.tok_per_block = 16 * p.row_tiles / G;
  p.blocks_per_seq = (n_q + p.tok_per_block - 1) / p.tok_per_block;
  p.n_units = (int64_t)batch * p.blocks_per_seq;
  p.n_groups = std::max(1, 1536 / n_kv_heads);
  return p;
}

hipError_t launch_paged_attention(int kv_fp8, int head_dim, int row_tiles, const PagedAttnArgs& a,
                                  hipStream_t stream) {
  const dim3 grid(a.n_kv_heads, a.n_groups), block(kThreads);
#define PDEC_PAGED(DH_, RT_, KT_)                                                       \
  do {                                                                                  \
    if (a.selected) paged_attn_kernel<DH_, RT_, KT_, true><<<grid, block, 0, stream>>>(a);  \
    else paged_attn_kernel<DH_, RT_, KT_, false><<<grid, block, 0, stream>>>(a);        \
  } while (0)
#define PDEC_PAGED_RT(DH_, KT_)                    \
  do {                                             \
    if (row_tiles == 1) PDEC_PAGED(DH_, 1, KT_);   \
    else if (row_tiles == 2) paged_attn_kernel<DH_, 2, KT_, false><<<grid, block, 0, stream>>>(a); \
    else paged_attn_kernel<DH_, 4, KT_, false><<<grid, block, 0, stream>>>(a);             \
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
  if (e != hipSuccess) return e;
  const dim3 mgrid(a.n_units, a.n_kv_heads);
  if (head_dim == 128)
    paged_merge_kernel<128><<<mgrid, block, 0, stream>>>(a, 16 * row_tiles);
  else
    paged_merge_kernel<64><<<mgrid, block, 0, stream>>>(a, 16 * row_tiles);
  return hipGetLastError();
}

}  // namespace pdec
