// Appending keys and values to caller-owned pages, with the rotary embedding
// applied on the way.
//
// Row r of the call belongs to the sequence b with row_start[b] <= r <
// row_start[b + 1] and sits at position p = lens[b] - (row_start[b + 1] - r).
// Its q and k heads are rotated by the table's angle of p, pairs (i, i + Dh/2);
// k and v go to slot p % 16 of page block_table[b][p / 16].
//
// E4M3 pages carry one scale per page and KV head, for K and for V: the smallest
// power of two s with max|x| <= 448 s over the tokens written.  A page that is
// part full keeps the larger of its own scale and what the new tokens need; where
// it grows, the codes written earlier are rounded again at the new scale, which is
// exact but for codes that become subnormal, since both scales are powers of two.
// So one work group handles all of a page's new tokens of one head: the first of
// them (the page's leader) finds the page, and the others' rows do nothing.
//
// Prompts are bound by HBM (4096 fp32 rows of 32 + 8 + 8 heads into bf16 pages, 153 MB read
// and written: 34 us, 4.5 TB/s, where a copy reaches 4.9; 1600 rows into E4M3 pages, 52 MB,
// 17), single tokens by one chain of loads: row, length, page, scale (64 sequences 7 us).
// V is taken eight slots of a dim a thread, so that a whole page half is one store.
#include "hip_common.h"
#include "kernels.h"
#include "rows.h"
#include "wave.h"

#include <algorithm>
#include <type_traits>

namespace pdec {

namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;

__device__ __forceinline__ float e4m3_to_f32(uint32_t code) {
  return __builtin_amdgcn_cvt_f32_fp8((int)code, 0);
}

template <typename T>
struct alignas(4 * sizeof(T)) Vec4 {
  T e[4];
};
template <typename T>
struct alignas(8 * sizeof(T) > 16 ? 16 : 8 * sizeof(T)) Vec8 {
  T e[8];
};

// Page elements, to nearest even.  inv: one over the page's scale (a power of two), 1
// where pages are not scaled; back() is what a reader of the page sees, over the scale.
template <typename T>
struct Elem;
template <>
struct Elem<float> {
  static __device__ __forceinline__ void put2(float* e, float a, float b, float) {
    e[0] = a;
    e[1] = b;
  }
  static __device__ __forceinline__ float back(float e) { return e; }
};
template <>
struct Elem<uint16_t> {  // the hardware conversion: NaN of any payload stays NaN
  static __device__ __forceinline__ void put2(uint16_t* e, float a, float b, float) {
    const uint32_t bits =
        __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
    e[0] = (uint16_t)bits;
    e[1] = (uint16_t)(bits >> 16);
  }
  static __device__ __forceinline__ float back(uint16_t e) { return bf16_to_f32(e); }
};
template <>
struct Elem<uint8_t> {
  static __device__ __forceinline__ void put2(uint8_t* e, float a, float b, float inv) {
    e[0] = (uint8_t)e4m3_from_f32(a * inv);
    e[1] = (uint8_t)e4m3_from_f32(b * inv);
  }
  static __device__ __forceinline__ float back(uint8_t e) { return e4m3_to_f32(e); }
};
template <typename T>
__device__ __forceinline__ Vec4<T> put4(f32x4 v, float inv) {
  Vec4<T> r;
  Elem<T>::put2(r.e, v.x, v.y, inv);
  Elem<T>::put2(r.e + 2, v.z, v.w, inv);
  return r;
}
template <typename T>
__device__ __forceinline__ f32x4 back4(const Vec4<T>& v) {
  return f32x4{Elem<T>::back(v.e[0]), Elem<T>::back(v.e[1]), Elem<T>::back(v.e[2]),
               Elem<T>::back(v.e[3])};
}

// The power of two that a part-full page's scale is kept at: the scale itself where
// this file made it, the next larger power of two where a caller did.
__device__ __forceinline__ float kept_scale(float s) {
  const uint32_t b = __float_as_uint(s);
  const int e = (int)(b >> 23) - 127 + ((b & 0x7FFFFFu) != 0);
  return __uint_as_float((uint32_t)(min(max(s > 0.f ? e : -100, -100), 100) + 127) << 23);
}
// Over the work group; `turn` counts its calls, which take two places in red in turn.
__device__ __forceinline__ float group_max(float v, float (*red)[kWaves], int turn) {
  float* at = red[turn & 1];
  v = wave_top(v);
  if ((threadIdx.x & 63) == 0) at[threadIdx.x >> 6] = v;
  __syncthreads();
  float t = at[0];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) t = fmaxf(t, at[w]);
  return t;
}

__device__ __forceinline__ void rotate4(f32x4& x, f32x4& y, const float2* cs) {
  const float4 t01 = *(const float4*)cs, t23 = *(const float4*)(cs + 2);
  const f32x4 c = {t01.x, t01.z, t23.x, t23.z}, s = {t01.y, t01.w, t23.y, t23.w};
  const f32x4 a = x, b = y;
  x = a * c - b * s;
  y = a * s + b * c;
}

// A run of m new tokens of one page: rows r .. r + m - 1, slots s0 .. s0 + m - 1,
// positions p0 .. p0 + m - 1.
struct Run {
  int64_t page;
  int r, m, s0, p0;
};

template <typename ST, typename KT, int DH>
__device__ __forceinline__ void append_k(const AppendArgs& a, const Run& run, int g, int turn,
                                         float (*red)[kWaves], float (*cols)[DH]) {
  constexpr int QR = DH / 8, H = DH / 2;  // threads per slot: four pairs each
  constexpr bool kFp8 = sizeof(KT) == 1;
  const int slot = threadIdx.x / QR, i = threadIdx.x % QR * 4;
  const bool fresh = slot >= run.s0 && slot < run.s0 + run.m, earlier = slot < run.s0;
  KT* dst = (KT*)a.k_pages + ((run.page * a.n_kv_heads + g) * kPage + slot) * DH;
  f32x4 x = {0.f, 0.f, 0.f, 0.f}, y = x;
  if (fresh) {
    const ST* src = (const ST*)a.k + (int64_t)(run.r + slot - run.s0) * a.k_stride + g * DH;
    x = read4(src + i);
    y = read4(src + i + H);
    rotate4(x, y, a.rope + (int64_t)(run.p0 + slot - run.s0) * H + i);
  }
  float scale = 1.f, inv = 1.f, old = 1.f;
  if constexpr (kFp8) {
    const int64_t at = run.page * a.n_kv_heads + g;
    if (run.s0 > 0) old = a.k_scales[at];
    float m = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) m = fmaxf(m, fmaxf(fabsf(x[e]), fabsf(y[e])));
    scale = scale_for(group_max(m, red, turn));
    if (run.s0 > 0) scale = fmaxf(scale, kept_scale(old));
    inv = inverse_pow2(scale);
    if (threadIdx.x == 0) a.k_scales[at] = scale;
  }
  Vec4<KT> lo, hi;
  bool held = fresh;
  if (fresh) {
    lo = put4<KT>(x, inv);
    hi = put4<KT>(y, inv);
  } else if (earlier && (a.k_means || (kFp8 && scale != old))) {
    lo = *(const Vec4<KT>*)(dst + i);
    hi = *(const Vec4<KT>*)(dst + i + H);
    held = true;
    if constexpr (kFp8) {
      if (scale != old) {
        lo = put4<KT>(back4<KT>(lo) * old, inv);
        hi = put4<KT>(back4<KT>(hi) * old, inv);
      }
    }
  }
  if (fresh || (held && kFp8 && scale != old)) {
    *(Vec4<KT>*)(dst + i) = lo;
    *(Vec4<KT>*)(dst + i + H) = hi;
  }
  if (a.k_means) {
    __syncthreads();  // the columns of the run before are read
    if (held) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        cols[slot][i + e] = Elem<KT>::back(lo.e[e]);
        cols[slot][i + H + e] = Elem<KT>::back(hi.e[e]);
      }
    }
    __syncthreads();
    const int n = run.s0 + run.m;
    if (threadIdx.x < DH) {
      float sum = 0.f;
      for (int s = 0; s < n; ++s) sum += cols[s][threadIdx.x];
      a.k_means[(run.page * a.n_kv_heads + g) * DH + threadIdx.x] =
          __builtin_bit_cast(uint16_t, (__bf16)(sum * scale / (float)n));
    }
  }
}

template <typename ST, typename KT, int DH>
__device__ __forceinline__ void append_v(const AppendArgs& a, const Run& run, int g, int turn,
                                         float (*red)[kWaves]) {
  constexpr bool kFp8 = sizeof(KT) == 1;
  const int d = threadIdx.x / 2, t0 = threadIdx.x % 2 * 8;  // one dim, eight slots
  const bool on = d < DH;
  KT* dst = (KT*)a.v_pages + ((run.page * a.n_kv_heads + g) * DH + d) * kPage + t0;
  float x[8];
  float m = 0.f;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int k = t0 + j - run.s0;
    x[j] = on && k >= 0 && k < run.m
               ? read1((const ST*)a.v + (int64_t)(run.r + k) * a.v_stride + g * DH + d)
               : 0.f;
    m = fmaxf(m, fabsf(x[j]));
  }
  float scale = 1.f, inv = 1.f, old = 1.f;
  if constexpr (kFp8) {
    const int64_t at = run.page * a.n_kv_heads + g;
    if (run.s0 > 0) old = a.v_scales[at];
    scale = scale_for(group_max(m, red, turn));
    if (run.s0 > 0) scale = fmaxf(scale, kept_scale(old));
    inv = inverse_pow2(scale);
    if (threadIdx.x == 0) a.v_scales[at] = scale;
  }
  if (!on) return;
  const bool moved = kFp8 && run.s0 > t0 && scale != old;
  Vec8<KT> e;
  if (moved) {
    e = *(const Vec8<KT>*)dst;
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (t0 + j < run.s0) x[j] = Elem<KT>::back(e.e[j]) * old;
  }
#pragma unroll
  for (int j = 0; j < 8; j += 2) Elem<KT>::put2(e.e + j, x[j], x[j + 1], inv);
  const int first = moved ? 0 : run.s0, end = run.s0 + run.m;
  if (first <= t0 && t0 + 8 <= end) {
    *(Vec8<KT>*)dst = e;
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (t0 + j >= first && t0 + j < end) dst[j] = e.e[j];
  }
}

// Work groups [0, n_rows) rotate one row's q heads (none without q); the others
// take (window of `window` rows, KV head, K or V) and handle the pages whose
// leader lies in the window.
template <typename ST, typename KT, int DH>
__global__ __launch_bounds__(kThreads) void kv_append_kernel(AppendArgs a, int q_groups,
                                                             int window) {
  typedef typename std::conditional<sizeof(KT) == 4, float, uint16_t>::type QT;
  __shared__ float red[2][kWaves];
  __shared__ float cols[kPage][DH];
  const int limit = (int)min((int64_t)a.max_pos, (int64_t)a.bt_stride * kPage);
  if ((int)blockIdx.x < q_groups) {
    constexpr int H = DH / 2, QR = DH / 8;
    const int r = blockIdx.x, b = find_seq(a.row_start, a.n_seqs, a.n_rows, r);
    if (b < 0) return;
    const int64_t pos = (int64_t)a.lens[b] - ((int64_t)a.row_start[b + 1] - r);
    if (pos < 0 || pos >= limit) return;
    const ST* src = (const ST*)a.q + (int64_t)r * a.q_stride;
    QT* dst = (QT*)a.q_out + (int64_t)r * a.n_q_heads * DH;
    for (int t = threadIdx.x; t < a.n_q_heads * QR; t += kThreads) {
      const int at = t / QR * DH + t % QR * 4;
      f32x4 x = read4(src + at), y = read4(src + at + H);
      rotate4(x, y, a.rope + pos * H + t % QR * 4);
      *(Vec4<QT>*)(dst + at) = put4<QT>(x, 1.f);
      *(Vec4<QT>*)(dst + at + H) = put4<QT>(y, 1.f);
    }
    return;
  }
  const int id = blockIdx.x - q_groups, part = id % (2 * a.n_kv_heads), g = part / 2;
  const int r_end = min((id / (2 * a.n_kv_heads) + 1) * window, a.n_rows);
  int r = id / (2 * a.n_kv_heads) * window;
  int b = -1, seq_row0 = 0, seq_end = 0, turn = 0;
  int64_t end_pos = 0;  // position behind row seq_end - 1; whatever the lengths hold fits
  while (r < r_end) {
    if (b < 0 || r >= seq_end) {
      b = find_seq(a.row_start, a.n_seqs, a.n_rows, r);
      if (b < 0) {
        ++r;
        continue;
      }
      seq_row0 = max(a.row_start[b], 0);  // its rows before the call's first are not here
      seq_end = min(a.row_start[b + 1], a.n_rows);
      end_pos = (int64_t)a.lens[b] - ((int64_t)a.row_start[b + 1] - seq_end);
    }
    const int64_t at = end_pos - (seq_end - r);
    if (at < 0) {  // more rows than the sequence has tokens
      r = -at < seq_end - r ? r + (int)-at : seq_end;
      continue;
    }
    if (at >= limit) {
      r = seq_end;
      continue;
    }
    const int pos = (int)at;
    const int slot = pos % kPage, m = min(min(kPage - slot, seq_end - r), limit - pos);
    if (r == seq_row0 || slot == 0) {
      const int64_t page = a.block_table[(int64_t)b * a.bt_stride + pos / kPage];
      if (page >= 0 && page < a.n_pages) {
        const Run run = {page, r, m, slot, pos};
        ++turn;
        if (part & 1)
          append_v<ST, KT, DH>(a, run, g, turn, red);
        else
          append_k<ST, KT, DH>(a, run, g, turn, red, cols);
      }
    }
    r += m;
  }
}

}  // namespace

// Long runs: a leader in 16 rows, so a window of 16 holds about one page; single
// tokens: every row is a leader.
static int append_window(const AppendArgs& a) {
  return a.n_rows >= 4 * (int64_t)a.n_seqs ? kPage : 1;
}
static int64_t append_groups(const AppendArgs& a) {
  const int64_t windows = ((int64_t)a.n_rows + append_window(a) - 1) / append_window(a);
  return (a.q ? a.n_rows : 0) + windows * 2 * a.n_kv_heads;
}
int64_t append_threads(const AppendArgs& a) { return append_groups(a) * kThreads; }

hipError_t launch_kv_append(int src_dtype, int kv_dtype, int head_dim, const AppendArgs& a,
                            hipStream_t stream) {
  if (a.n_rows == 0) return hipSuccess;
  const int window = append_window(a), q_groups = a.q ? a.n_rows : 0;
  const dim3 grid((uint32_t)append_groups(a)), block(kThreads);
#define PDEC_APPEND(ST_, KT_)                                                              \
  do {                                                                                     \
    if (head_dim == 128)                                                                   \
      kv_append_kernel<ST_, KT_, 128><<<grid, block, 0, stream>>>(a, q_groups, window);    \
    else                                                                                   \
      kv_append_kernel<ST_, KT_, 64><<<grid, block, 0, stream>>>(a, q_groups, window);     \
  } while (0)
  if (kv_dtype == 0) {
    PDEC_APPEND(float, float);
  } else if (kv_dtype == 1) {
    if (src_dtype == 0) PDEC_APPEND(float, uint16_t);
    else PDEC_APPEND(uint16_t, uint16_t);
  } else {
    if (src_dtype == 0) PDEC_APPEND(float, uint8_t);
    else PDEC_APPEND(uint16_t, uint8_t);
  }
#undef PDEC_APPEND
  return hipGetLastError();
}

}  // namespace pdec
