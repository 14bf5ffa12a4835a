// Verification of drafted tokens against the target's probabilities, with
// caller-supplied uniforms.
//
// Masses are whole numbers, as in the sampler (sample.hip): for a row z of logits
//   m_v = rint(exp((z_v - max z) / T) * 2^40),  S = sum_v m_v,
// P of a target row and D of a drafter's (fp64 exponential, everything after it exact
// or one IEEE operation).  With p_v = P_v * (2^50 / S_P), d_v = D_v * (2^50 / S_D)
// rounded as doubles and u24 = floor(u * 2^24), draft i is accepted while all before
// it were and  u24 d_x < 2^24 p_x;  without a drafter's logits its probability is 1,
// d_x = 2^50.  The next token is drawn from
//   r_v = rint(max(p_v - d_v, 0))   at the draft that was refused (d_v = 2^50 at the
//                                   draft alone without a drafter's logits),
//   r_v = rint(p_v)                 after the last draft, at an id outside the
//                                   vocabulary, which ends the drafts, or where the
//                                   former has no mass:
// Z = sum r_v, target = floor(u24 Z / 2^24), the first v whose running sum exceeds it.
// Sums of whole numbers do not depend on their order, so however rows are split over
// work groups the tokens are the same.  A row whose maximum is not finite has no mass,
// and NaN logits have none; with no mass at all the token is 0.
//
// Every row has to be read (which draft is the last one accepted is not known before),
// but the whole-number sums are needed of one row a sequence only:
//   1. stats: each row once, its maximum and sum of exponentials in fp32, at the HBM
//      rate; the sum is within 2^-14 of S (fp32 exponentials of arguments down to -41,
//      the rounding of masses and what is left out below 2^-41);
//   2. judge: the tests with these sums, exact where both sides are further apart than
//      2^-10 of them.  A test that is closer, one in a thousand, takes the masses' own
//      sums of its two rows, so every decision is that of the definition.  Then the
//      masses of the deciding row, summed by chunks;
//   3. rest: r summed by chunks;  4. pick: the chunk that holds the target, its tokens
//      side by side in one group's threads and one scan.
// Masses of every row in fp64, maximum first, took 313 us for 64 sequences of 4 drafts
// and their drafter's logits at 128256 tokens (87 + 125 + 62 + 51).
#include "hip_common.h"
#include "kernels.h"

#include <algorithm>
#include <cfloat>
#include <cmath>

namespace pdec {

namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr double kMinX = -28.5;  // below it the mass rounds to 0
constexpr double kUnit = 0x1p50;
constexpr int kMaxDrafts = 1024;

struct Sizes {
  int chunk, n_chunks;  // tokens of a chunk (a multiple of 1024), chunks of a row
  int rows;             // target rows, then drafter rows
};
inline Sizes sizes_of(int batch, int n_drafts, bool drafter, int vocab) {
  Sizes s;
  s.rows = batch * (n_drafts + 1 + (drafter ? n_drafts : 0));
  // 32 values a thread; few rows are cut finer, so that they meet more work groups.
  s.chunk = (int64_t)s.rows * vocab >= (1 << 23) ? 8192 : 2048;
  s.n_chunks = (vocab + s.chunk - 1) / s.chunk;
  return s;
}

// What the drafts of one sequence came to.
struct Verdict {
  int n;         // accepted drafts
  int refused;   // the draft refused (-1: none, the next token is the target's own)
  float pm, dm;  // maximum of the target row behind it, of the drafter's row at it
};

// Workspace: per (row, chunk) the maximum and the sum of exponentials over it; per
// (sequence, chunk) the two rows' masses and the two residual masses; verdicts.
struct Work {
  ulonglong2 *mass, *rest;  // (target, drafter), (r with the drafts taken off, rint p)
  float2* stat;
  Verdict* verdict;
};
__host__ __device__ inline Work work_of(void* base, const Sizes& s, int batch) {
  Work w;
  w.mass = (ulonglong2*)base;
  w.rest = w.mass + (int64_t)batch * s.n_chunks;
  w.stat = (float2*)(w.rest + (int64_t)batch * s.n_chunks);
  w.verdict = (Verdict*)(w.stat + (int64_t)s.rows * s.n_chunks);
  return w;
}

__device__ __forceinline__ const float* row_ptr(const VerifyArgs& a, int row) {
  const int n_target = a.batch * (a.n_drafts + 1);
  return row < n_target ? a.target + (int64_t)row * a.vocab
                        : a.drafter + (int64_t)(row - n_target) * a.vocab;
}

__device__ __forceinline__ uint64_t mass_of(float z, double m, double inv_t) {
#pragma clang fp contract(off)
  const double x = ((double)z - m) * inv_t;
  if (!(x >= kMinX)) return 0;
  return (uint64_t)rint(exp(x) * 0x1p40);
}

__device__ __forceinline__ uint64_t wave_sum_u64(uint64_t v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}
__device__ __forceinline__ uint64_t group_sum(uint64_t v, uint64_t* red) {
  v = wave_sum_u64(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  uint64_t t = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) t += red[w];
  return t;
}

// Four consecutive tokens from v on, those at or past end as -inf.
__device__ __forceinline__ f32x4 tokens4(const float* z, int v, int end) {
  if (v + 4 <= end) return *(const f32x4_any*)(z + v);
  f32x4 r;
#pragma unroll
  for (int e = 0; e < 4; ++e) r[e] = v + e < end ? z[v + e] : -INFINITY;
  return r;
}

// ---- 1. stats ----------------------------------------------------------------
template <int Q>  // float4s a thread: the chunk is 1024 Q
__global__ __launch_bounds__(kThreads) void verify_stats_kernel(VerifyArgs a, Sizes s, float c2) {
  __shared__ float2 sh[kWaves];
  const int row = blockIdx.x, c = blockIdx.y;
  const float* z = row_ptr(a, row);
  const int begin = c * s.chunk, end = min(begin + s.chunk, a.vocab);
  f32x4 v[Q];
#pragma unroll
  for (int k = 0; k < Q; ++k) v[k] = tokens4(z, begin + (k * kThreads + threadIdx.x) * 4, end);
  float m = -INFINITY;  // fmaxf takes no NaN
#pragma unroll
  for (int k = 0; k < Q; ++k) m = fmaxf(m, fmaxf(fmaxf(v[k].x, v[k].y), fmaxf(v[k].z, v[k].w)));
  m = wave_max(m);
  float sum = 0.f;
#pragma unroll
  for (int k = 0; k < Q; ++k)
#pragma unroll
    for (int e = 0; e < 4; ++e)  // -inf and NaN: 2^-150, which is 0
      sum += __builtin_amdgcn_exp2f(fmaxf((v[k][e] - m) * c2, -150.f));
  sum = wave_sum(sum);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = make_float2(m, sum);
  __syncthreads();
  if (threadIdx.x == 0) {
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) top = fmaxf(top, sh[w].x);
    float t = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w)
      t += sh[w].y * __builtin_amdgcn_exp2f(fmaxf((sh[w].x - top) * c2, -150.f));
    work_of(a.workspace, s, a.batch).stat[(int64_t)row * s.n_chunks + c] = make_float2(top, t);
  }
}

// A row's maximum and sum from its chunks', the same in every lane of the wave.
__device__ __forceinline__ float2 row_stat(const Work& w, const Sizes& s, int row, float c2) {
  const float2* st = w.stat + (int64_t)row * s.n_chunks;
  const int lane = threadIdx.x & 63;
  float m = -INFINITY;
  for (int c = lane; c < s.n_chunks; c += 64) m = fmaxf(m, st[c].x);
  m = wave_max(m);
  float sum = 0.f;
  for (int c = lane; c < s.n_chunks; c += 64)
    sum += st[c].y * __builtin_amdgcn_exp2f(fmaxf((st[c].x - m) * c2, -150.f));
  return make_float2(m, wave_sum(sum));
}

// ---- 2. judge ----------------------------------------------------------------
__device__ __forceinline__ double unit_over(uint64_t mass) {
  return mass ? kUnit / (double)mass : 0.0;
}
__device__ __forceinline__ uint64_t u24_of(float u) {
  return (uint64_t)floorf(fminf(fmaxf(u, 0.f), 0x1.fffffep-1f) * 0x1p24f);
}

// 2^50 over a whole row's mass, by the whole work group.
__device__ double exact_unit(const float* z, int vocab, float m, double inv_t, uint64_t* red) {
  uint64_t sum = 0;
  for (int v = threadIdx.x; v < vocab; v += kThreads) sum += mass_of(z[v], m, inv_t);
  return unit_over(group_sum(sum, red));
}

__global__ __launch_bounds__(kThreads) void verify_judge_kernel(VerifyArgs a, Sizes s, float c2,
                                                                double slack) {
#pragma clang fp contract(off)
  __shared__ uint64_t red[kWaves];
  __shared__ signed char verdicts[kMaxDrafts];
  const int b = blockIdx.x, c = blockIdx.y, T = a.n_drafts, wave = threadIdx.x >> 6;
  const Work w = work_of(a.workspace, s, a.batch);
  enum { kRefuse, kAccept, kClose, kEnd };
  // One side of test i: 2^24 p_x, and u24 d_x, with units of the row sums `pu`, `du`.
  auto lhs = [&](int i, float dm, double du) {
    const int64_t at = (int64_t)b * T + i;
    const double dx = a.drafter ? (double)mass_of(a.drafter[at * a.vocab + a.drafts[at]], dm, a.inv_t) * du
                                : kUnit;
    return (double)u24_of(a.uniforms[(int64_t)b * (T + 1) + i]) * dx;
  };
  auto rhs = [&](int i, float pm, double pu) {
    const int64_t row = (int64_t)b * (T + 1) + i;
    const double px =
        (double)mass_of(a.target[row * a.vocab + a.drafts[(int64_t)b * T + i]], pm, a.inv_t) * pu;
    return 0x1p24 * px;
  };
  const int row0 = b * (T + 1), drow0 = a.batch * (T + 1) + b * T;
  for (int i = wave; i < T; i += kWaves) {
    const int x = a.drafts[(int64_t)b * T + i];
    int verdict = kEnd;
    if (x >= 0 && x < a.vocab) {
      const float2 p = row_stat(w, s, row0 + i, c2);
      const float2 d = a.drafter ? row_stat(w, s, drow0 + i, c2) : make_float2(0.f, 1.f);
      // 2^50 / S, S in units of 2^40; no mass where the maximum is not finite
      const double l = lhs(i, d.x, fabsf(d.x) <= FLT_MAX ? 0x1p10 / (double)d.y : 0.0);
      const double r = rhs(i, p.x, fabsf(p.x) <= FLT_MAX ? 0x1p10 / (double)p.y : 0.0);
      verdict = l < r * (1.0 - slack) ? kAccept : l >= r * (1.0 + slack) ? kRefuse : kClose;
    }
    if ((threadIdx.x & 63) == 0) verdicts[i] = (signed char)verdict;
  }
  __syncthreads();
  Verdict v = {0, -1, 0.f, 0.f};
  for (; v.n < T; ++v.n) {
    int verdict = verdicts[v.n];
    if (verdict == kClose) {
      const float pm = row_stat(w, s, row0 + v.n, c2).x;
      const double pu = exact_unit(row_ptr(a, row0 + v.n), a.vocab, pm, a.inv_t, red);
      float dm = 0.f;
      double du = 0.0;
      if (a.drafter) {
        dm = row_stat(w, s, drow0 + v.n, c2).x;
        du = exact_unit(row_ptr(a, drow0 + v.n), a.vocab, dm, a.inv_t, red);
      }
      verdict = lhs(v.n, dm, du) < rhs(v.n, pm, pu) ? kAccept : kRefuse;
    }
    if (verdict == kAccept) continue;
    if (verdict == kRefuse) v.refused = a.drafts[(int64_t)b * T + v.n];
    break;
  }
  const bool drafter = a.drafter && v.refused >= 0;
  v.pm = row_stat(w, s, row0 + v.n, c2).x;
  if (drafter) v.dm = row_stat(w, s, drow0 + v.n, c2).x;
  if (c == 0 && threadIdx.x == 0) w.verdict[b] = v;
  const float* zp = row_ptr(a, row0 + v.n);
  const float* zd = drafter ? row_ptr(a, drow0 + v.n) : nullptr;
  const int begin = c * s.chunk, end = min(begin + s.chunk, a.vocab);
  uint64_t p = 0, d = 0;
  for (int t = begin + threadIdx.x * 4; t < end; t += kThreads * 4) {
    const f32x4 x = tokens4(zp, t, end);
#pragma unroll
    for (int e = 0; e < 4; ++e) p += mass_of(x[e], v.pm, a.inv_t);
    if (drafter) {
      const f32x4 y = tokens4(zd, t, end);
#pragma unroll
      for (int e = 0; e < 4; ++e) d += mass_of(y[e], v.dm, a.inv_t);
    }
  }
  p = group_sum(p, red);
  d = group_sum(d, red);
  if (threadIdx.x == 0) w.mass[(int64_t)b * s.n_chunks + c] = make_ulonglong2(p, d);
}

// ---- 3. rest, 4. pick ------------------------------------------------------------
// The distribution that a sequence's next token is drawn from.
struct Next {
  const float *zp, *zd;  // zd null: nothing or one token to take off
  double pm, pi, dm, di, inv_t;
  int refused;
  // r_v, and rint(p_v); x, y the target's and the drafter's logit of token v.
  __device__ __forceinline__ uint64_t at(int v, float x, float y, uint64_t* whole) const {
#pragma clang fp contract(off)
    const double p = (double)mass_of(x, pm, inv_t) * pi;
    *whole = (uint64_t)rint(p);
    if (refused < 0) return *whole;
    double d = v == refused ? INFINITY : 0.0;
    if (zd) d = (double)mass_of(y, dm, inv_t) * di;
    return (uint64_t)rint(fmax(p - d, 0.0));
  }
};

__device__ __forceinline__ Next next_of(const VerifyArgs& a, const Sizes& s, const Work& w, int b) {
  const Verdict v = w.verdict[b];
  uint64_t p = 0, d = 0;  // every wave for itself
  for (int c = threadIdx.x & 63; c < s.n_chunks; c += 64) {
    const ulonglong2 m = w.mass[(int64_t)b * s.n_chunks + c];
    p += m.x;
    d += m.y;
  }
  Next r;
  r.zp = a.target + ((int64_t)b * (a.n_drafts + 1) + v.n) * a.vocab;
  r.zd = a.drafter && v.refused >= 0 ? a.drafter + ((int64_t)b * a.n_drafts + v.n) * a.vocab : nullptr;
  r.pm = v.pm;
  r.dm = v.dm;
  r.pi = unit_over(wave_sum_u64(p));
  r.di = unit_over(wave_sum_u64(d));
  r.inv_t = a.inv_t;
  r.refused = v.refused;
  return r;
}

__global__ __launch_bounds__(kThreads) void verify_rest_kernel(VerifyArgs a, Sizes s) {
  __shared__ uint64_t red[kWaves];
  const int b = blockIdx.x, c = blockIdx.y;
  const Work w = work_of(a.workspace, s, a.batch);
  const Next r = next_of(a, s, w, b);
  const int begin = c * s.chunk, end = min(begin + s.chunk, a.vocab);
  uint64_t rest = 0, whole = 0;
  for (int t = begin + threadIdx.x * 4; t < end; t += kThreads * 4) {
    const f32x4 x = tokens4(r.zp, t, end);
    f32x4 y = {0.f, 0.f, 0.f, 0.f};
    if (r.zd) y = tokens4(r.zd, t, end);
#pragma unroll
    for (int e = 0; e < 4; ++e) {  // past the end: -inf, no mass of either
      uint64_t p;
      rest += r.at(t + e, x[e], y[e], &p);
      whole += p;
    }
  }
  rest = group_sum(rest, red);
  whole = group_sum(whole, red);
  if (threadIdx.x == 0) w.rest[(int64_t)b * s.n_chunks + c] = make_ulonglong2(rest, whole);
}

constexpr int kPickThreads = 1024, kPickWaves = kPickThreads / 64;

__global__ __launch_bounds__(kPickThreads) void verify_pick_kernel(VerifyArgs a, Sizes s) {
  __shared__ uint64_t red[kPickWaves];
  __shared__ int found;
  const int b = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const Work w = work_of(a.workspace, s, a.batch);
  const Next r = next_of(a, s, w, b);
  const ulonglong2* part = w.rest + (int64_t)b * s.n_chunks;
  uint64_t z = 0, whole = 0;
  for (int c = lane; c < s.n_chunks; c += 64) {
    z += part[c].x;
    whole += part[c].y;
  }
  z = wave_sum_u64(z);
  const bool own = z == 0;  // nothing left beside the drafts': the target's own
  if (own) z = wave_sum_u64(whole);
  const uint64_t u = u24_of(a.uniforms[(int64_t)b * (a.n_drafts + 1) + a.n_drafts]);
  const uint64_t goal = (uint64_t)(((unsigned __int128)u * z) >> 24);
  if (threadIdx.x == 0) found = 0;
  if (z > 0) {
    // The chunk whose running sum passes the goal, by every wave for itself.
    uint64_t run = 0;
    int at = 0;
    for (int c0 = 0; c0 < s.n_chunks; c0 += 64) {
      const uint64_t v = c0 + lane < s.n_chunks ? (own ? part[c0 + lane].y : part[c0 + lane].x) : 0;
      uint64_t incl = v;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const uint64_t t = __shfl_up(incl, o, 64);
        if (lane >= o) incl += t;
      }
      const uint64_t hit = __ballot(run + incl > goal);
      if (hit) {
        const int l = __builtin_ctzll(hit);
        at = c0 + l;
        run += __shfl(incl, l, 64) - __shfl(v, l, 64);
        break;
      }
      run += __shfl(incl, 63, 64);
    }
    // Eight tokens a thread side by side, one scan, and the thread that passes the goal
    // walks its own.
    const int begin = at * s.chunk, end = min(begin + s.chunk, a.vocab);
    const int v0 = begin + threadIdx.x * 8;
    uint64_t mine[8], sum = 0;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      f32x4 x = {-INFINITY, -INFINITY, -INFINITY, -INFINITY}, y = x;
      if (v0 + 4 * h < end) {
        x = tokens4(r.zp, v0 + 4 * h, end);
        if (r.zd) y = tokens4(r.zd, v0 + 4 * h, end);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        uint64_t p;
        const uint64_t q = r.at(v0 + 4 * h + e, x[e], y[e], &p);
        mine[4 * h + e] = own ? p : q;
        sum += mine[4 * h + e];
      }
    }
    uint64_t incl = sum;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const uint64_t t = __shfl_up(incl, o, 64);
      if (lane >= o) incl += t;
    }
    if (lane == 63) red[wave] = incl;
    __syncthreads();
    run += incl - sum;
    for (int i = 0; i < wave; ++i) run += red[i];
    if (run <= goal && goal < run + sum) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (run <= goal && goal < run + mine[e]) found = v0 + e;
        run += mine[e];
      }
    }
  }
  __syncthreads();
  const int n = w.verdict[b].n;
  for (int j = threadIdx.x; j <= a.n_drafts; j += kPickThreads)
    a.tokens[(int64_t)b * (a.n_drafts + 1) + j] =
        j < n ? a.drafts[(int64_t)b * a.n_drafts + j] : j == n ? found : -1;
  if (threadIdx.x == 0) a.accepted[b] = n;
}

}  // namespace

int64_t verify_workspace_bytes(int batch, int n_drafts, bool drafter, int vocab) {
  const Sizes s = sizes_of(batch, n_drafts, drafter, vocab);
  return ((int64_t)s.rows * 8 + (int64_t)batch * 32) * s.n_chunks +
         (int64_t)batch * (int64_t)sizeof(Verdict);
}

hipError_t launch_verify(const VerifyArgs& a, hipStream_t stream) {
  static_assert(8 * kPickThreads >= 8192, "one step of the pick covers a chunk");
  const Sizes s = sizes_of(a.batch, a.n_drafts, a.drafter != nullptr, a.vocab);
  const float c2 = std::min(1.4426950408889634f / a.temperature, 3e38f);
  // Temperatures at which fp32 arguments mean nothing: every test is a close one.
  const double slack = a.temperature < 1e-30f ? INFINITY : 0x1p-10;
  const dim3 all(s.rows, s.n_chunks), one(a.batch, s.n_chunks);
  if (s.chunk == 8192)
    verify_stats_kernel<8><<<all, kThreads, 0, stream>>>(a, s, c2);
  else
    verify_stats_kernel<2><<<all, kThreads, 0, stream>>>(a, s, c2);
  verify_judge_kernel<<<one, kThreads, 0, stream>>>(a, s, c2, slack);
  verify_rest_kernel<<<one, kThreads, 0, stream>>>(a, s);
  verify_pick_kernel<<<a.batch, kPickThreads, 0, stream>>>(a, s);
  return hipGetLastError();
}

}  // namespace pdec
