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

#include <algorithm>
#include <cfloat>

namespace pdec {

namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kScorePages = 64;  // pages of one work group of the score pass

__device__ __forceinline__ int seq_pages(const SelectArgs& a, int b) {
  const int len = max(a.lens[b], 0);
  return min(len / kPage + (len % kPage != 0), a.bt_stride);
}

// 16 lanes per (page, KV head), DH / 16 dims each.
template <int DH>
__global__ __launch_bounds__(kThreads) void page_scores_kernel(SelectArgs a) {
  constexpr int E = DH / 16;
  const int b = blockIdx.x, p0 = blockIdx.y * kScorePages;
  const int n = min(seq_pages(a, b) - p0, kScorePages);
  const int G = a.n_q_heads / a.n_kv_heads, d0 = (threadIdx.x & 15) * E;
  for (int t = threadIdx.x / 16; t < n * a.n_kv_heads; t += kThreads / 16) {
    const int p = p0 + t / a.n_kv_heads, g = t % a.n_kv_heads;
    const int page = a.block_table[(int64_t)b * a.bt_stride + p];
    double best = -INFINITY;
    if (page >= 0 && page < a.n_pages) {
      const uint16_t* src = a.k_means + ((int64_t)page * a.n_kv_heads + g) * DH + d0;
      double mean[E];
#pragma unroll
      for (int e = 0; e < E; ++e) mean[e] = bf16_to_f32(src[e]);
      for (int h = 0; h < G; ++h) {
        const uint16_t* q = a.q + ((int64_t)b * a.n_q_heads + g * G + h) * DH + d0;
        double s = 0.0;
#pragma unroll
        for (int e = 0; e < E; ++e) s += mean[e] * bf16_to_f32(q[e]);
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) s += __shfl_xor(s, o, 16);
        best = fmax(best, s);  // a NaN never wins
      }
    }
    if ((threadIdx.x & 15) == 0)
      a.scores[((int64_t)b * a.n_kv_heads + g) * a.bt_stride + p] =
          fminf(fmaxf((float)best, -FLT_MAX), FLT_MAX);
  }
}

__device__ __forceinline__ int group_scan(int v, int* red, int* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int incl = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int t = __shfl_up(incl, o, 64);
    if (lane >= o) incl += t;
  }
  __syncthreads();
  if (lane == 63) red[wave] = incl;
  __syncthreads();
  int before = incl - v, sum = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    before += w < wave ? red[w] : 0;
    sum += red[w];
  }
  *total = sum;
  return before;
}

// One work group per (sequence, KV head): the threshold by a radix select over the
// order-preserving bits of the scores, eight at a time, then the list in page order.
__global__ __launch_bounds__(kThreads) void take_pages_kernel(SelectArgs a) {
  __shared__ int hist[256];
  __shared__ int red[kWaves];
  __shared__ int pick[2];
  const int b = blockIdx.x, g = blockIdx.y, n = seq_pages(a, b);
  const float* score = a.scores + ((int64_t)b * a.n_kv_heads + g) * a.bt_stride;
  int32_t* out = a.selected + ((int64_t)b * a.n_kv_heads + g) * a.n_selected;
  const int take = min(n, a.n_selected);
  for (int i = take + threadIdx.x; i < a.n_selected; i += kThreads) out[i] = -1;
  if (take == n) {
    for (int i = threadIdx.x; i < n; i += kThreads) out[i] = i;
    return;
  }
  // Larger key, better page; kept pages above every score.
  auto key_of = [&](int i) -> uint32_t {
    if (i < a.keep_first || i >= n - a.keep_last) return 0xFFFFFFFFu;
    const uint32_t u = __float_as_uint(score[i] + 0.f);  // -0 counts as 0
    return u & 0x80000000u ? ~u : u | 0x80000000u;
  };
  uint32_t prefix = 0;
  int left = take;  // pages still to be taken among those with the prefix
  for (int shift = 24; shift >= 0; shift -= 8) {
    hist[threadIdx.x] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += kThreads) {
      const uint32_t k = key_of(i);
      if (shift == 24 || (k ^ prefix) >> (shift + 8) == 0) atomicAdd(&hist[(k >> shift) & 255], 1);
    }
    __syncthreads();
    // Bins from the top: thread t holds bin 255 - t.
    int total;
    const int c = hist[255 - threadIdx.x], above = group_scan(c, red, &total);
    if (above < left && left <= above + c) {
      pick[0] = 255 - threadIdx.x;
      pick[1] = left - above;
    }
    __syncthreads();
    prefix |= (uint32_t)pick[0] << shift;
    left = pick[1];
    __syncthreads();
  }
  // Pages above the threshold, and the first `left` at it.
  int done = 0, ties = 0;
  for (int i0 = 0; i0 < n; i0 += kThreads) {
    const int i = i0 + threadIdx.x;
    const uint32_t k = i < n ? key_of(i) : 0;
    const bool tie = i < n && k == prefix;
    int n_tie, n_in;
    const int tie_rank = ties + group_scan(tie, red, &n_tie);
    const bool in = i < n && (k > prefix || (tie && tie_rank < left));
    const int at = done + group_scan(in, red, &n_in);
    if (in) out[at] = i;
    ties += n_tie;
    done += n_in;
  }
}

}  // namespace

hipError_t launch_paged_select(int head_dim, const SelectArgs& a, hipStream_t stream) {
  const dim3 grid(a.batch, (a.bt_stride + kScorePages - 1) / kScorePages), block(kThreads);
  if (head_dim == 128)
    page_scores_kernel<128><<<grid, block, 0, stream>>>(a);
  else
    page_scores_kernel<64><<<grid, block, 0, stream>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  take_pages_kernel<<<dim3(a.batch, a.n_kv_heads), block, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace pdec
