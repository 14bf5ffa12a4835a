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
//      rate; the sum is within 2^-15 of S (arguments down to -41 log2 units rounded
//      three times, 41 * 3 * 2^-24, and again with the parts' maxima; sums of 32 terms and
//      a few levels, 90 * 2^-24; the rounding of 2^22 masses, 2^-19);
//   2. judge: the tests with these sums, exact where both sides are further apart than
//      2^-13 of them.  A test that is closer, one in thousands, takes the masses' own
//      sums of its two rows, so every decision is that of the definition.  Then the
//      masses of the deciding row, summed by cuts;
//   3. rest: r summed by parts of cuts;  4. pick: the part that holds the target, its
//      tokens side by side in one group's threads and one scan.
// 64 sequences of 4 drafts and their drafter's logits at 128256 tokens, 295 MB: 94 us (50,
// 5.9 TB/s, + 22 + 20 + 6); with the masses of every row in fp64, maximum first, 313.
#include "hip_common.h"
#include "kernels.h"
#include "wave.h"

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <type_traits>

namespace pdec {

namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr double kMinX = -28.5;  // below it the mass rounds to 0
constexpr double kUnit = 0x1p50;
constexpr int kMaxDrafts = 1024;
constexpr int kParts = kWaves;  // of a cut, each summed by a wave: the pick walks one

typedef VerifySizes Sizes;

// What the drafts of one sequence came to.
struct Verdict {
  int n;         // accepted drafts
  int refused;   // the draft refused (-1: none, the next token is the target's own)
  float pm, dm;  // maximum of the target row behind it, of the drafter's row at it
};

// Workspace: per (row, chunk) the maximum and the sum of exponentials over it; per
// (sequence, cut) the two rows' masses, per part the two residual masses; verdicts.
struct Work {
  ulonglong2 *mass, *rest;  // (target, drafter), (r with the drafts taken off, rint p)
  float2* stat;
  Verdict* verdict;
};
__host__ __device__ inline Work work_of(void* base, const Sizes& s, int batch) {
  Work w;
  w.mass = (ulonglong2*)base;
  w.rest = w.mass + (int64_t)batch * s.n_cuts;
  w.stat = (float2*)(w.rest + (int64_t)batch * s.n_cuts * kParts);
  w.verdict = (Verdict*)(w.stat + (int64_t)s.rows * s.n_chunks);
  return w;
}

__device__ __forceinline__ const float* row_ptr(const VerifyArgs& a, int row) {
  const int n_target = a.batch * (a.n_drafts + 1);
  return row < n_target ? a.target + (int64_t)row * a.vocab
                        : a.drafter + (int64_t)(row - n_target) * a.vocab;
}

// exp(x) for -28.5 <= x <= 0 by exp(x) = 2^(n / 64) exp(r), n = rint(64 x / ln 2): a table
// of the 64 fractions in LDS and the series of exp(r) to the fifth power, |r| <= ln 2 / 128
// (the sixth is below 2^-54).  64 / ln 2 times x has at most 12 bits before the point, so
// n times the upper part of ln 2 / 64, 40 bits of it, is exact.  One unit in the last place
// at most, as the library's, in half of its time: of the passes over the deciding rows (64
// sequences of 128256 tokens and two rows, judge and rest: 21 and 19 us) this arithmetic is 7
// and 9 (with a comparison in its place 14 and 10, for 66 MB read again and what 1024 work
// groups do before their first mass); with the library's and masses as integers 36 and 37.
constexpr double kLn2 = 0.69314718055994530942;
constexpr double kStepHi = 0x1.62e42fefa0000p-7;  // ln 2 / 64, 40 bits
constexpr double kStepLo = 0x1.cf79abc9e3b3ap-46;  // and what is left of it
__device__ __forceinline__ void fill_fractions(double* frac) {
  for (int j = threadIdx.x; j < 64; j += blockDim.x) frac[j] = exp2((double)j / 64.0);
  __syncthreads();
}
__device__ __forceinline__ double exp_of(double x, const double* frac) {
  // n in the low bits of a double behind 1.5 * 2^52, which has no fraction.
  const double t = __builtin_fma(x, 64.0 / kLn2, 0x1.8p52);
  const int i = __double2loint(t);
  const double n = t - 0x1.8p52;
  const double r = __builtin_fma(-n, kStepLo, __builtin_fma(-n, kStepHi, x));
  double p = __builtin_fma(r, 1.0 / 120.0, 1.0 / 24.0);
  p = __builtin_fma(r, p, 1.0 / 6.0);
  p = __builtin_fma(r, p, 0.5);
  p = __builtin_fma(r * r, p, r);
  const double f = frac[i & 63];
  const double e = __builtin_fma(f, p, f);
  return __hiloint2double(__double2hiint(e) + ((i & ~63) << 14), __double2loint(e));
}

// The whole number nearest to x, 0 <= x < 2^52, ties to even: behind 2^52 a double has no
// fraction.  (Conversions to and from 64-bit integers are a score of instructions each, so
// masses stay doubles until a thread has summed its own: those sums are below 2^53, where
// doubles are exact.)
__device__ __forceinline__ double whole(double x) { return (x + 0x1p52) - 0x1p52; }
__device__ __forceinline__ uint64_t to_u64(double x) {  // of a whole number below 2^53
  return (uint64_t)(uint32_t)(x * 0x1p-32) << 32 |
         (uint32_t)(x - 0x1p32 * (double)(uint32_t)(x * 0x1p-32));
}

// m_v of a logit; m its row's maximum.
__device__ __forceinline__ double mass_of(float z, double m, double inv_t, const double* frac) {
  double x;
  {
#pragma clang fp contract(off)
    x = ((double)z - m) * inv_t;
  }
  const double e = whole(exp_of(x, frac) * 0x1p40);
  return x >= kMinX ? e : 0.0;  // (what lies below, and NaN, came to anything)
}

__device__ __forceinline__ uint64_t group_sum(uint64_t v, uint64_t* red) {
  v = wave_add(v);
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

// f(t, four tokens of row zp from t on, four of zd) for t = from, from + STEP, .. below end;
// the next tokens are in flight meanwhile.  (A rolled loop: the arithmetic of a call is long
// and runs at the fp64 rate, so waves in number hide the rest; with a chunk's loads and sums
// unrolled, two waves a SIMD, the judge took 31 us instead of 23.)
template <int STEP, typename F>
__device__ __forceinline__ void walk(const float* zp, const float* zd, int from, int end, F&& f) {
  if (from >= end) return;
  f32x4 nx = tokens4(zp, from, end), ny = {0.f, 0.f, 0.f, 0.f};
  if (zd) ny = tokens4(zd, from, end);
#pragma unroll 1
  for (int t = from; t < end; t += STEP) {
    const f32x4 x = nx, y = ny;
    if (t + STEP < end) {
      nx = tokens4(zp, t + STEP, end);
      if (zd) ny = tokens4(zd, t + STEP, end);
    }
    f(t, x, y);
  }
}

// ---- 1. stats ----------------------------------------------------------------
template <int Q>  // float4s a thread: the chunk is 1024 Q
__global__ __launch_bounds__(kThreads) void verify_stats_kernel(VerifyArgs a, Sizes s, float c2) {
  __shared__ float2 sh[kWaves];
  const int row = blockIdx.x / s.n_chunks, c = blockIdx.x % s.n_chunks;
  const float* z = row_ptr(a, row);
  const int begin = c * s.chunk, end = min(begin + s.chunk, a.vocab);
  f32x4 v[Q];
#pragma unroll
  for (int k = 0; k < Q; ++k) v[k] = tokens4(z, begin + (k * kThreads + threadIdx.x) * 4, end);
  float m = -INFINITY;  // fmaxf takes no NaN
#pragma unroll
  for (int k = 0; k < Q; ++k) m = fmaxf(m, fmaxf(fmaxf(v[k].x, v[k].y), fmaxf(v[k].z, v[k].w)));
  m = wave_top(m);
  float sum = 0.f;
#pragma unroll
  for (int k = 0; k < Q; ++k)
#pragma unroll
    for (int e = 0; e < 4; ++e)  // -inf and NaN: 2^-150, which is 0
      sum += __builtin_amdgcn_exp2f(fmaxf((v[k][e] - m) * c2, -150.f));
  sum = wave_add(sum);
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
  float2 mine = lane < s.n_chunks ? st[lane] : make_float2(-INFINITY, 0.f);
  for (int c = lane + 64; c < s.n_chunks; c += 64) {
    const float2 o = st[c];
    const float m = fmaxf(mine.x, o.x);
    mine.y = mine.y * __builtin_amdgcn_exp2f(fmaxf((mine.x - m) * c2, -150.f)) +
             o.y * __builtin_amdgcn_exp2f(fmaxf((o.x - m) * c2, -150.f));
    mine.x = m;
  }
  const float m = wave_top(mine.x);
  return make_float2(m, wave_add(mine.y * __builtin_amdgcn_exp2f(fmaxf((mine.x - m) * c2, -150.f))));
}

// ---- 2. judge ----------------------------------------------------------------
__device__ __forceinline__ double unit_over(uint64_t mass) {
  return mass ? kUnit / (double)mass : 0.0;
}
__device__ __forceinline__ uint64_t u24_of(float u) {
  return (uint64_t)floorf(fminf(fmaxf(u, 0.f), 0x1.fffffep-1f) * 0x1p24f);
}

// 2^50 over a whole row's mass, by the whole work group.
__device__ double exact_unit(const float* z, int vocab, float m, double inv_t, const double* frac,
                             uint64_t* red) {
  uint64_t sum = 0;
  for (int v = threadIdx.x; v < vocab; v += kThreads) sum += to_u64(mass_of(z[v], m, inv_t, frac));
  return unit_over(group_sum(sum, red));
}

__global__ __launch_bounds__(kThreads) void verify_judge_kernel(VerifyArgs a, Sizes s, float c2,
                                                                double slack) {
#pragma clang fp contract(off)
  __shared__ uint64_t red[kWaves];
  __shared__ signed char verdicts[kMaxDrafts];
  __shared__ float2 p_stat[kMaxDrafts + 1], d_stat[kMaxDrafts];
  __shared__ double frac[64];
  fill_fractions(frac);
  const int b = blockIdx.x, c = blockIdx.y, T = a.n_drafts, wave = threadIdx.x >> 6;
  const Work w = work_of(a.workspace, s, a.batch);
  enum { kRefuse, kAccept, kClose, kEnd };
  const int row0 = b * (T + 1), drow0 = a.batch * (T + 1) + b * T;
  // What test i looks at: the draft, its logits, its uniform number.
  struct Draft {
    int x;
    float zp, zd, u;
  };
  auto draft = [&](int i) {
    Draft r = {a.drafts[(int64_t)b * T + i], 0.f, 0.f, a.uniforms[(int64_t)b * (T + 1) + i]};
    if (r.x >= 0 && r.x < a.vocab) {
      r.zp = row_ptr(a, row0 + i)[r.x];
      if (a.drafter) r.zd = row_ptr(a, drow0 + i)[r.x];
    }
    return r;
  };
  // Its sides, with units of the row sums `pu`, `du`: u24 d_x, and 2^24 p_x.
  auto lhs = [&](const Draft& r, float dm, double du) {
    return (double)u24_of(r.u) * (a.drafter ? mass_of(r.zd, dm, a.inv_t, frac) * du : kUnit);
  };
  auto rhs = [&](const Draft& r, float pm, double pu) {
    return 0x1p24 * (mass_of(r.zp, pm, a.inv_t, frac) * pu);
  };
  // A thread a test: the loads of one follow each other, so all are under way while the
  // waves sum up the rows.
  Draft mine = {-1, 0.f, 0.f, 0.f};
  if (threadIdx.x < T) mine = draft(threadIdx.x);
  for (int i = wave; i <= T; i += kWaves) {
    const float2 p = row_stat(w, s, row0 + i, c2);
    float2 d = make_float2(0.f, 1.f);
    if (a.drafter && i < T) d = row_stat(w, s, drow0 + i, c2);
    if ((threadIdx.x & 63) == 0) {
      p_stat[i] = p;
      if (i < T) d_stat[i] = d;
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < T; i += kThreads) {
    if (i >= kThreads) mine = draft(i);
    int verdict = kEnd;
    if (mine.x >= 0 && mine.x < a.vocab) {
      const float2 p = p_stat[i], d = d_stat[i];
      // 2^50 / S, S in units of 2^40; no mass where the maximum is not finite
      const double l = lhs(mine, d.x, fabsf(d.x) <= FLT_MAX ? 0x1p10 / (double)d.y : 0.0);
      const double r = rhs(mine, p.x, fabsf(p.x) <= FLT_MAX ? 0x1p10 / (double)p.y : 0.0);
      verdict = l < r * (1.0 - slack) ? kAccept : l >= r * (1.0 + slack) ? kRefuse : kClose;
    }
    verdicts[i] = (signed char)verdict;
  }
  __syncthreads();
  Verdict v = {0, -1, 0.f, 0.f};
  for (; v.n < T; ++v.n) {
    int verdict = verdicts[v.n];
    if (verdict == kClose) {
      const float pm = p_stat[v.n].x, dm = d_stat[v.n].x;
      const double pu = exact_unit(row_ptr(a, row0 + v.n), a.vocab, pm, a.inv_t, frac, red);
      const double du =
          a.drafter ? exact_unit(row_ptr(a, drow0 + v.n), a.vocab, dm, a.inv_t, frac, red) : 0.0;
      const Draft r = draft(v.n);
      verdict = lhs(r, dm, du) < rhs(r, pm, pu) ? kAccept : kRefuse;
    }
    if (verdict == kAccept) continue;
    if (verdict == kRefuse) v.refused = a.drafts[(int64_t)b * T + v.n];
    break;
  }
  const bool drafter = a.drafter && v.refused >= 0;
  v.pm = p_stat[v.n].x;
  if (drafter) v.dm = d_stat[v.n].x;
  if (c == 0 && threadIdx.x == 0) w.verdict[b] = v;
  const float* zp = row_ptr(a, row0 + v.n);
  const float* zd = drafter ? row_ptr(a, drow0 + v.n) : nullptr;
  const int begin = c * s.cut, end = min(begin + s.cut, a.vocab);
  double mp = 0.0, md = 0.0;  // 32 masses at most
  walk<kThreads * 4>(zp, zd, begin + threadIdx.x * 4, end, [&](int, f32x4 x, f32x4 y) {
#pragma unroll
    for (int e = 0; e < 4; ++e) mp += mass_of(x[e], v.pm, a.inv_t, frac);
    if (drafter)
#pragma unroll
      for (int e = 0; e < 4; ++e) md += mass_of(y[e], v.dm, a.inv_t, frac);
  });
  const uint64_t p = group_sum(to_u64(mp), red), d = group_sum(to_u64(md), red);
  if (threadIdx.x == 0) w.mass[(int64_t)b * s.n_cuts + c] = make_ulonglong2(p, d);
}

// ---- 3. rest, 4. pick ------------------------------------------------------------
// What is taken off the target's probabilities.
enum Off { kNothing, kToken, kDrafter };

// The distribution that a sequence's next token is drawn from.
struct Next {
  const float *zp, *zd;  // zd null but for kDrafter
  double pm, pi, dm, di, inv_t;
  const double* frac;
  int refused;
  Off off;
  // r_v, and rint(p_v); x, y the target's and the drafter's logit of token v.
  template <Off OFF>
  __device__ __forceinline__ double at(int v, float x, float y, double* all) const {
#pragma clang fp contract(off)
    const double p = mass_of(x, pm, inv_t, frac) * pi;
    *all = whole(p);
    if constexpr (OFF == kNothing) return *all;
    if constexpr (OFF == kToken) return v == refused ? 0.0 : *all;
    const double d = mass_of(y, dm, inv_t, frac) * di;
    return whole(fmax(p - d, 0.0));
  }
  // f(std::integral_constant<Off, off>): one branch for a whole loop.
  template <typename F>
  __device__ __forceinline__ void by_off(F&& f) const {
    if (off == kDrafter) f(std::integral_constant<Off, kDrafter>{});
    else if (off == kToken) f(std::integral_constant<Off, kToken>{});
    else f(std::integral_constant<Off, kNothing>{});
  }
};

__device__ __forceinline__ Next next_of(const VerifyArgs& a, const Sizes& s, const Work& w, int b,
                                        const double* frac) {
  const Verdict v = w.verdict[b];
  uint64_t p = 0, d = 0;  // every wave for itself
  for (int c = threadIdx.x & 63; c < s.n_cuts; c += 64) {
    const ulonglong2 m = w.mass[(int64_t)b * s.n_cuts + c];
    p += m.x;
    d += m.y;
  }
  Next r;
  r.zp = a.target + ((int64_t)b * (a.n_drafts + 1) + v.n) * a.vocab;
  r.off = v.refused < 0 ? kNothing : a.drafter ? kDrafter : kToken;
  r.zd = r.off == kDrafter ? a.drafter + ((int64_t)b * a.n_drafts + v.n) * a.vocab : nullptr;
  r.pm = v.pm;
  r.dm = v.dm;
  r.pi = unit_over(wave_add(p));
  r.di = unit_over(wave_add(d));
  r.inv_t = a.inv_t;
  r.frac = frac;
  r.refused = v.refused;
  return r;
}

__global__ __launch_bounds__(kThreads) void verify_rest_kernel(VerifyArgs a, Sizes s) {
  __shared__ double frac[64];
  fill_fractions(frac);
  const int b = blockIdx.x, part = blockIdx.y * kParts + (threadIdx.x >> 6);
  const Work w = work_of(a.workspace, s, a.batch);
  const Next r = next_of(a, s, w, b, frac);
  const int len = s.cut / kParts, begin = part * len, end = min(begin + len, a.vocab);
  double rest = 0.0, all = 0.0;  // sums of parts of 2^50, but for roundings
  r.by_off([&](auto off) {
    walk<256>(r.zp, r.zd, begin + (threadIdx.x & 63) * 4, end, [&](int t, f32x4 x, f32x4 y) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {  // past the end: -inf, no mass of either
        double p;
        rest += r.template at<decltype(off)::value>(t + e, x[e], y[e], &p);
        all += p;
      }
    });
  });
  const uint64_t r_sum = wave_add(to_u64(rest)), p_sum = wave_add(to_u64(all));
  if ((threadIdx.x & 63) == 0)
    w.rest[(int64_t)b * s.n_cuts * kParts + part] = make_ulonglong2(r_sum, p_sum);
}

__global__ __launch_bounds__(kThreads) void verify_pick_kernel(VerifyArgs a, Sizes s) {
  __shared__ uint64_t red[kWaves];
  __shared__ int found;
  __shared__ double frac[64];
  fill_fractions(frac);
  const int b = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const Work w = work_of(a.workspace, s, a.batch);
  const Next r = next_of(a, s, w, b, frac);
  const int n_parts = s.n_cuts * kParts, len = s.cut / kParts;
  const ulonglong2* part = w.rest + (int64_t)b * n_parts;
  uint64_t z = 0, all = 0;
  for (int c = lane; c < n_parts; c += 64) {
    z += part[c].x;
    all += part[c].y;
  }
  z = wave_add(z);
  const bool own = z == 0;  // nothing left beside the drafts': the target's own
  if (own) z = wave_add(all);
  const uint64_t u = u24_of(a.uniforms[(int64_t)b * (a.n_drafts + 1) + a.n_drafts]);
  const uint64_t goal = (uint64_t)(((unsigned __int128)u * z) >> 24);
  if (threadIdx.x == 0) found = 0;
  if (z > 0) {
    // The part whose running sum passes the goal, by every wave for itself.
    uint64_t run = 0;
    int at = 0;
    for (int c0 = 0; c0 < n_parts; c0 += 64) {
      const uint64_t v = c0 + lane < n_parts ? (own ? part[c0 + lane].y : part[c0 + lane].x) : 0;
      const uint64_t incl = wave_prefix(v);
      const uint64_t hit = __ballot(run + incl > goal);
      if (hit) {
        const int l = __builtin_ctzll(hit);
        at = c0 + l;
        run += lane_of(incl, l) - lane_of(v, l);
        break;
      }
      run += lane_of(incl, 63);
    }
    // Eight tokens a thread side by side, one scan, and the thread that passes the goal
    // walks its own.
    const int begin = at * len, end = min(begin + len, a.vocab), v0 = begin + threadIdx.x * 8;
    uint64_t mine[8], sum = 0;
    f32x4 x[2], y[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      x[h] = y[h] = f32x4{-INFINITY, -INFINITY, -INFINITY, -INFINITY};
      if (v0 + 4 * h < end) {
        x[h] = tokens4(r.zp, v0 + 4 * h, end);
        if (r.zd) y[h] = tokens4(r.zd, v0 + 4 * h, end);
      }
    }
    r.by_off([&](auto off) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        double p;
        const double q = r.template at<decltype(off)::value>(v0 + e, x[e / 4][e % 4], y[e / 4][e % 4], &p);
        mine[e] = to_u64(own ? p : q);
        sum += mine[e];
      }
    });
    const uint64_t incl = wave_prefix(sum);
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
  for (int j = threadIdx.x; j <= a.n_drafts; j += kThreads)
    a.tokens[(int64_t)b * (a.n_drafts + 1) + j] =
        j < n ? a.drafts[(int64_t)b * a.n_drafts + j] : j == n ? found : -1;
  if (threadIdx.x == 0) a.accepted[b] = n;
}

}  // namespace

// What these sizes and all smaller batches and drafts take.  Smaller ones are cut finer: the
// most pieces of 2048 tokens are those of the last rows, and sequences, below the borders.
int64_t verify_workspace_bytes(int batch, int n_drafts, bool drafter, int vocab) {
  const Sizes s = verify_sizes(batch, n_drafts, drafter, vocab);
  const int64_t fine = (vocab + 2047) / 2048;
  const int64_t chunks = std::max((int64_t)s.rows * s.n_chunks,
                                  std::min<int64_t>(s.rows, (kFineLogits - 1) / vocab) * fine);
  const int64_t cuts = std::max((int64_t)batch * s.n_cuts,
                                std::min<int64_t>(batch, (kFineCuts - 1) / vocab) * fine);
  return chunks * 8 + cuts * 16 * (1 + kParts) + (int64_t)batch * (int64_t)sizeof(Verdict);
}

hipError_t launch_verify(const VerifyArgs& a, hipStream_t stream) {
  static_assert(8 * kThreads >= 8192 / kParts, "one step of the pick covers a part");
  const Sizes s = verify_sizes(a.batch, a.n_drafts, a.drafter != nullptr, a.vocab);
  const float c2 = std::min(1.4426950408889634f / a.temperature, 3e38f);
  // Temperatures at which fp32 arguments mean nothing: every test is a close one.
  const double slack = a.temperature < 1e-30f ? INFINITY : 0x1p-13;
  // A row's chunks side by side.
  const dim3 all((uint32_t)s.rows * s.n_chunks), one(a.batch, s.n_cuts);
  if (s.chunk == 8192)
    verify_stats_kernel<8><<<all, kThreads, 0, stream>>>(a, s, c2);
  else
    verify_stats_kernel<2><<<all, kThreads, 0, stream>>>(a, s, c2);
  verify_judge_kernel<<<one, kThreads, 0, stream>>>(a, s, c2, slack);
  verify_rest_kernel<<<one, kThreads, 0, stream>>>(a, s);
  verify_pick_kernel<<<a.batch, kThreads, 0, stream>>>(a, s);
  return hipGetLastError();
}

}  // namespace pdec
