// Choosing the pages of a cache that a query token's attention reads.
//
// A page's score for KV head g is max over g's query heads h of q_h . mean, mean being
// the page's key mean.  The n_selected pages of the highest scores are taken, ties to
// the lower page, the first keep_first and last keep_last pages whatever their scores,
// and listed in page order.
//
// The scores are summed in 64 bits, where the products of bf16 values are exact, and
// rounded to fp32 once: which page is the last one taken is decided by the values and
// not by the order of a sum.
#include "hip_common.h"
#include "kernels.h"
#include "stretch.h"

#include <algorithm>
#include <cfloat>
#include <type_traits>

namespace pdec {

namespace {

constexpr int kThreads = 512, kWaves = kThreads / 64;  // of the scores
constexpr int kTile = 16;  // pages a wave scores at a time

__device__ __forceinline__ int seq_pages(const int32_t* lens, int b, int bt_stride) {
  const int len = max(lens[b], 0);
  return min(len / kPage + (len % kPage != 0), bt_stride);
}

template <int CTRL>
__device__ __forceinline__ double swapped(double v) {
  return __longlong_as_double((int64_t)dpp<CTRL>((uint64_t)__double_as_longlong(v)));
}

// Scores.  A wave takes tiles of 16 pages of one KV head.  The product runs on
// v_mfma_f64_4x4x4_4b, whose four blocks of 4 x 4 x 4 multiply 16 pages with four query
// heads, every lane busy and no sum across lanes: lane l holds page l % 16 and the dims
// 32 j + 8 (l / 16) + e of chunk j, one 16-byte load each, and the same dims of query head
// l % 4; result lane l has page 4 (l / 4 % 4) + l / 16 and head l % 4.  The next tile's
// means are in flight meanwhile.
//
// The bound is HBM: Dh bf16 a page and KV head, 256 bytes, the KV heads of a page side by
// side.  They are taken by the waves of one work group, so that a page's means are read as
// one run, and as many groups as stay resident have equal stretches of tiles, so that the
// lengths, the queries and the first pages are waited for once.  64 sequences of 8K to 32K,
// 168 MB: 38 us; with groups of one KV head 41, with groups of 256 pages each 42.  The
// products (9 us, 17 cycles a tile and dim quad) hide behind the loads: 37 without them.  A
// quarter of the lengths takes 15 us and four times them 144, so 6 us are the beginning and
// the rest goes at 4.8 to 5.3 TB/s, with one tile of 4 KB in flight a wave.  The non-temporal
// hint costs 8%: an instruction takes half of a line, and the other half's finds it gone.
constexpr int kScoreGroups = 512;

template <int DH, int HG>  // HG groups of four query heads; more than one in LDS
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(4))) void page_scores_kernel(
    SelectArgs a, const int32_t* __restrict__ table, const int32_t* __restrict__ lens, int heads) {
  constexpr int NJ = DH / 32;
  __shared__ int red[kWaves], found[2];
  // Converted already where two groups of waves still share a compute unit's LDS.
  typedef typename std::conditional<HG == 2, double, float>::type QT;
  __shared__ QT qs[HG > 1 ? kWaves : 1][HG][HG > 1 ? NJ * 8 : 1][16];
  const int w = blockIdx.y;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  // This wave's KV head, and its row among the rows of waves that share the tiles.
  const int g = blockIdx.x * heads + wave % heads, row = wave / heads, rows = kWaves / heads;
  const int c16 = lane & 15, k4 = lane >> 4;
  const int G = a.n_q_heads / a.n_kv_heads;
  auto tiles_of = [&](int b) { return (seq_pages(lens, b, a.bt_stride) + kTile - 1) / kTile; };
  const Stretch mine = stretch_of<kThreads>(a.batch, gridDim.y, rows, w, red, found, tiles_of);
  int at = w * mine.per, first = mine.first;
  if (at >= mine.total || g >= a.n_kv_heads || row >= rows) return;
  const int stop = min(at + mine.per, mine.total);
  for (int b = mine.unit; at < stop; ++b) {
    const int tiles = tiles_of(b);
    if (tiles == 0) continue;
    const int n = seq_pages(lens, b, a.bt_stride);
    // This stretch's pages of the sequence.
    const int begin = (at - first) * kTile, end = min(n, min(tiles, stop - first) * kTile);
    first += tiles;
    at = min(first, stop);
    const uint16_t* q0 = a.q + ((int64_t)b * a.n_q_heads + g * G) * DH;
    // Groups of four heads; past the last one the first stands in, which moves no maximum.
    auto q_at = [&](int hg, int j, int col, int k) {
      const int h = 4 * hg + col;
      return *(const u16x8*)(q0 + (int64_t)(h < G ? h : 0) * DH + j * 32 + k * 8);
    };
    double q[NJ * 8];
    if constexpr (HG > 1) {
      // A wave writes and reads its own part, in order: no barrier.
      for (int i = lane; i < HG * NJ * 16; i += 64) {
        const int l = i % 16, j = i / 16 % NJ, hg = i / 16 / NJ;
        const u16x8 v = q_at(hg, j, l % 4, l / 4);
#pragma unroll
        for (int e = 0; e < 8; ++e) qs[wave][hg][j * 8 + e][l] = bf16_to_f32(v[e]);
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    } else {
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        const u16x8 v = q_at(0, j, lane & 3, k4);
#pragma unroll
        for (int e = 0; e < 8; ++e) q[j * 8 + e] = bf16_to_f32(v[e]);
      }
    }
    const int32_t* bt = table + (int64_t)b * a.bt_stride;
    auto page_of = [&](int p0) { return bt[min(p0 + c16, n - 1)]; };
    auto load = [&](int page, u16x8(&m)[NJ]) {
      const bool ok = page >= 0 && page < a.n_pages;
      const uint16_t* src = a.k_means + ((int64_t)(ok ? page : 0) * a.n_kv_heads + g) * DH + k4 * 8;
#pragma unroll
      for (int j = 0; j < NJ; ++j) m[j] = *(const u16x8*)(src + j * 32);
    };
    const int step = rows * kTile;
    int p0 = begin + row * kTile;
    if (p0 >= end) continue;
    float* scores = a.scores + ((int64_t)b * a.n_kv_heads + g) * a.bt_stride;
    u16x8 next[NJ];
    int page = page_of(p0), page1 = page_of(p0 + step);
    load(page, next);
    for (; p0 < end; p0 += step) {
      u16x8 m[NJ];
#pragma unroll
      for (int j = 0; j < NJ; ++j) m[j] = next[j];
      const bool ok = page >= 0 && page < a.n_pages;
      page = page1;
      if (p0 + step < end) {
        load(page, next);
        page1 = page_of(p0 + 2 * step);
      }
      // Two chains for each group, so that a product does not wait for the last.
      double s[HG][2] = {};
      int col = k4 * 4 + (lane & 3);
      asm volatile("" : "+v"(col));  // else all the queries of LDS are kept in registers
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const double mean = bf16_to_f32(m[j][e]);
#pragma unroll
          for (int hg = 0; hg < HG; ++hg)
            s[hg][e % 2] = __builtin_amdgcn_mfma_f64_4x4x4f64(
                mean, HG > 1 ? (double)qs[wave][hg][j * 8 + e][col] : q[j * 8 + e],
                s[hg][e % 2], 0, 0, 0);
        }
      double best = -INFINITY;
#pragma unroll
      for (int hg = 0; hg < HG; ++hg) best = fmax(best, s[hg][0] + s[hg][1]);  // a NaN never wins
      best = fmax(best, swapped<0xB1>(best));  // with lane ^ 1
      best = fmax(best, swapped<0x4E>(best));  // with lane ^ 2
      const int i = 4 * ((lane >> 2) & 3) + k4;  // the page of this lane's result
      const bool named = __shfl((int)ok, i, 64);
      if ((lane & 3) == 0 && p0 + i < end)
        scores[p0 + i] = named ? fminf(fmaxf((float)best, -FLT_MAX), FLT_MAX) : -FLT_MAX;
    }
  }
}

// The list: one work group of T threads per (sequence, KV head).  A histogram of T bins of
// equal width over the range of the scores leaves a few pages in the bin that holds the
// last one taken, which a wave ranks; where it leaves more than a wave's lanes (equal
// scores, an outlier that widens the range), histograms over the scores' bits narrow it
// down.  A thread holds eight scores meanwhile and reads again what is past them.  Page order
// comes from ballots and one scan of the waves' counts.  Eight bits at a time from the top of the float, a scan for each step of
// pages, took 57 us for 8188 pages; bits of the range, two or three rounds, 14; this 10.
template <int T>
__global__ __launch_bounds__(T) void take_pages_kernel(SelectArgs a) {
  constexpr int W = T / 64, BITS = T == 1024 ? 10 : T == 512 ? 9 : 8, STEPS = 8;
  __shared__ int hist[T];
  __shared__ int red[2][W];
  __shared__ uint32_t range[2][W];
  __shared__ int count[2][STEPS * W];
  __shared__ int pick[4];
  __shared__ uint32_t few[64];
  const int b = blockIdx.x / a.n_kv_heads, n = seq_pages(a.lens, b, a.bt_stride);
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const float* score = a.scores + (int64_t)blockIdx.x * a.bt_stride;
  int32_t* out = a.selected + (int64_t)blockIdx.x * a.n_selected;
  const int take = min(n, a.n_selected);
  for (int i = take + threadIdx.x; i < a.n_selected; i += T) out[i] = -1;
  if (take == n) {
    for (int i = threadIdx.x; i < n; i += T) out[i] = i;
    return;
  }
  // Larger key, larger score.
  auto read = [&](int i) {
    const uint32_t u = __float_as_uint(score[i] + 0.f);  // -0 counts as 0
    return u & 0x80000000u ? ~u : u | 0x80000000u;
  };
  auto value = [](uint32_t k) { return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k); };
  auto kept = [&](int i) { return i < a.keep_first || i >= n - a.keep_last; };
  uint32_t held[STEPS];
#pragma unroll
  for (int s = 0; s < STEPS; ++s) {
    const int i = s * T + threadIdx.x;
    if (i < n) held[s] = read(i);
  }
  // f(key) for this thread's pages that are not kept.
  auto each = [&](auto&& f) {
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      const int i = s * T + threadIdx.x;
      if (i < n && !kept(i)) f(held[s]);
    }
    for (int i = STEPS * T + threadIdx.x; i < n; i += T)
      if (!kept(i)) f(read(i));
  };
  uint32_t lo = 0xFFFFFFFFu, hi = 0;
  each([&](uint32_t k) {
    lo = min(lo, k);
    hi = max(hi, k);
  });
  hist[threadIdx.x] = 0;
  if (threadIdx.x == 0) pick[3] = 0;
  lo = wave_all(lo, [](uint32_t x, uint32_t y) { return min(x, y); });
  hi = wave_all(hi, [](uint32_t x, uint32_t y) { return max(x, y); });
  if (lane == 0) {
    range[0][wave] = lo;
    range[1][wave] = hi;
  }
  __syncthreads();
  for (int w = 0; w < W; ++w) {
    lo = min(lo, range[0][w]);
    hi = max(hi, range[1][w]);
  }
  // Of the bins' counts in hist, bin T - 1 on top: the bin that holds the left-th page from
  // the top, how many are wanted of it, and how many it has.
  auto crossing = [&](int left) {
    __syncthreads();
    const int c = hist[T - 1 - threadIdx.x];
    const int incl = wave_prefix(c);
    if (lane == 63) red[0][wave] = incl;
    __syncthreads();
    int above = incl - c;
    for (int w = 0; w < wave; ++w) above += red[0][w];
    if (above < left && left <= above + c) {
      pick[0] = T - 1 - threadIdx.x;
      pick[1] = left - above;
      pick[2] = c;
    }
    __syncthreads();
  };
  // Wanted: the `left` highest keys of [lo, hi] that are not kept; all above hi are taken.
  int left = take - a.keep_first - a.keep_last;
  bool all = false;  // every key from lo on, else those above lo and `left` of lo itself
  if (left == 0) {
    lo = 0xFFFFFFFFu;  // (no score has this key)
  } else {
    // Bins over the scores themselves: monotone, since each step of the arithmetic is.
    const float s0 = value(lo), width = value(hi) - s0, per = (float)T / width;
    const bool even = width > 0.f && width < FLT_MAX && per < FLT_MAX;
    auto bin_of = [&](uint32_t k) { return min((int)((value(k) - s0) * per), T - 1); };
    bool ranked = false;
    if (even) {
      each([&](uint32_t k) { atomicAdd(&hist[bin_of(k)], 1); });
      crossing(left);
      const int bin = pick[0], want = pick[1];
      if (pick[2] <= 64) {
        each([&](uint32_t k) {
          if (bin_of(k) == bin) few[atomicAdd(&pick[3], 1)] = k;
        });
        __syncthreads();
        // The want-th largest of them, and how many of its equals are wanted.
        const int m = pick[2];
        const uint32_t mine = lane < m ? few[lane] : 0;
        int over = 0, equal = 0;
        for (int i = 0; i < m; ++i) {
          over += few[i] > mine;
          equal += few[i] == mine;
        }
        const uint64_t hit = __ballot(lane < m && over < want && want <= over + equal);
        const int l = __builtin_ctzll(hit);
        lo = (uint32_t)lane_of((int)mine, l);
        left = want - lane_of(over, l);
        ranked = true;
      }
    }
    while (!ranked) {
      const uint32_t span = hi - lo;
      const int shift = max(32 - BITS - (span ? __builtin_clz(span) : 32), 0);
      __syncthreads();
      hist[threadIdx.x] = 0;
      __syncthreads();
      each([&](uint32_t k) {
        if (k >= lo && k <= hi) atomicAdd(&hist[(k - lo) >> shift], 1);
      });
      crossing(left);
      lo += (uint32_t)pick[0] << shift;
      hi = shift ? min(hi, lo + ((1u << shift) - 1)) : lo;
      left = pick[1];
      all = pick[2] == left;
      ranked = all || shift == 0;
    }
  }
  // Taken pages in order, STEPS x T at a time: of each step a wave's pages above the
  // threshold and at it, then where they begin.
  int done = 0, ties = 0;
  for (int i0 = 0; i0 < n; i0 += STEPS * T) {
    uint32_t over = 0, at = 0;  // this lane's pages by step
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      const int i = i0 + s * T + threadIdx.x;
      bool o = false, t = false;
      if (i < n) {
        const uint32_t k = i0 == 0 ? held[s] : read(i);
        o = kept(i) || k > lo || (all && k == lo);
        t = !o && k == lo;
      }
      over |= (uint32_t)o << s;
      at |= (uint32_t)t << s;
      const uint64_t bo = __ballot(o), bt = __ballot(t);
      if (lane == 0) {
        count[0][s * W + wave] = __popcll(bo);
        count[1][s * W + wave] = __popcll(bt);
      }
    }
    __syncthreads();
    if (wave < 2) {  // wave 0: pages above, wave 1: ties; exclusive sums in place
      int base = wave ? ties : done;
      for (int j = 0; j < STEPS * W; j += 64) {
        const int v = j + lane < STEPS * W ? count[wave][j + lane] : 0;
        const int incl = wave_prefix(v);
        if (j + lane < STEPS * W) count[wave][j + lane] = base + incl - v;
        base += lane_of(incl, 63);
      }
      if (lane == 0) red[wave][0] = base;
    }
    __syncthreads();
    const uint64_t below = lane ? ~0ull >> (64 - lane) : 0;
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      const bool o = over >> s & 1, t = at >> s & 1;
      const int n_over = count[0][s * W + wave] + __popcll(__ballot(o) & below);
      const int n_tie = count[1][s * W + wave] + __popcll(__ballot(t) & below);
      if (o || (t && n_tie < left)) out[n_over + min(n_tie, left)] = i0 + s * T + threadIdx.x;
    }
    done = red[0][0];
    ties = red[1][0];
    __syncthreads();
  }
}

}  // namespace

// Threads for eight pages each, up to what a work group holds.
static int list_threads(int bt_stride) { return bt_stride > 4096 ? 1024 : bt_stride > 512 ? 512 : 256; }
int64_t select_threads(const SelectArgs& a) {
  return (int64_t)a.batch * a.n_kv_heads * list_threads(a.bt_stride);
}

hipError_t launch_paged_select(int head_dim, const SelectArgs& a, hipStream_t stream) {
  const int64_t rows = (int64_t)a.batch * a.n_kv_heads;
  const int heads = std::min(a.n_kv_heads, kWaves), head_blocks = (a.n_kv_heads + heads - 1) / heads;
  const dim3 grid(head_blocks, std::max(1, kScoreGroups / head_blocks));
  const int groups = (a.n_q_heads / a.n_kv_heads + 3) / 4;
#define PDEC_SCORES(DH_, HG_)                                                         \
  page_scores_kernel<DH_, HG_><<<grid, kThreads, 0, stream>>>(a, a.block_table, a.lens, \
                                                              heads)
#define PDEC_SCORES_HG(DH_)                    \
  do {                                         \
    if (groups == 1) PDEC_SCORES(DH_, 1);      \
    else if (groups == 2) PDEC_SCORES(DH_, 2); \
    else PDEC_SCORES(DH_, 4);                  \
  } while (0)
  if (head_dim == 128) PDEC_SCORES_HG(128);
  else PDEC_SCORES_HG(64);
#undef PDEC_SCORES_HG
#undef PDEC_SCORES
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int threads = list_threads(a.bt_stride);
  if (threads == 1024)
    take_pages_kernel<1024><<<(uint32_t)rows, 1024, 0, stream>>>(a);
  else if (threads == 512)
    take_pages_kernel<512><<<(uint32_t)rows, 512, 0, stream>>>(a);
  else
    take_pages_kernel<256><<<(uint32_t)rows, 256, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace pdec
