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
#include "hip_common.h"
#include "kernels.h"

#include <algorithm>

namespace pdec {

namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr double kMinX = -28.5;  // below it the mass rounds to 0
constexpr double kUnit = 0x1p50;

struct Sizes {
  int chunk, n_chunks;  // tokens of a chunk, chunks of a row
  int rows;             // target rows, then drafter rows
};
__host__ __device__ inline Sizes sizes_of(int batch, int n_drafts, bool drafter, int vocab) {
  Sizes s;
  s.rows = batch * (n_drafts + 1 + (drafter ? n_drafts : 0));
  s.chunk = 8192;
  s.n_chunks = (vocab + s.chunk - 1) / s.chunk;
  return s;
}

// Workspace: per (row, chunk) the maximum and the mass, per (sequence, chunk) the two
// residual masses.
struct Work {
  uint64_t *mass, *rest, *whole;
  float* max;
};
__host__ __device__ inline Work work_of(void* base, const Sizes& s, int batch) {
  Work w;
  w.mass = (uint64_t*)base;
  w.rest = w.mass + (int64_t)s.rows * s.n_chunks;
  w.whole = w.rest + (int64_t)batch * s.n_chunks;
  w.max = (float*)(w.whole + (int64_t)batch * s.n_chunks);
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

__global__ __launch_bounds__(kThreads) void verify_max_kernel(VerifyArgs a, Sizes s) {
  __shared__ float red[kWaves];
  const int row = blockIdx.x, c = blockIdx.y;
  const Work w = work_of(a.workspace, s, a.batch);
  const float* z = row_ptr(a, row);
  const int end = min((c + 1) * s.chunk, a.vocab);
  float m = -INFINITY;
  for (int v = c * s.chunk + threadIdx.x; v < end; v += kThreads) m = fmaxf(m, z[v]);
  m = wave_max(m);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = m;
  __syncthreads();
  if (threadIdx.x == 0) {
#pragma unroll
    for (int i = 1; i < kWaves; ++i) m = fmaxf(m, red[i]);
    w.max[(int64_t)row * s.n_chunks + c] = m;
  }
}

__device__ __forceinline__ float row_max(const Work& w, const Sizes& s, int row) {
  float m = -INFINITY;
  for (int c = 0; c < s.n_chunks; ++c) m = fmaxf(m, w.max[(int64_t)row * s.n_chunks + c]);
  return m;
}
__device__ __forceinline__ uint64_t row_mass(const Work& w, const Sizes& s, int row) {
  uint64_t m = 0;
  for (int c = 0; c < s.n_chunks; ++c) m += w.mass[(int64_t)row * s.n_chunks + c];
  return m;
}

__global__ __launch_bounds__(kThreads) void verify_mass_kernel(VerifyArgs a, Sizes s) {
  __shared__ uint64_t red[kWaves];
  const int row = blockIdx.x, c = blockIdx.y;
  const Work w = work_of(a.workspace, s, a.batch);
  const float* z = row_ptr(a, row);
  const double m = row_max(w, s, row);
  const int end = min((c + 1) * s.chunk, a.vocab);
  uint64_t sum = 0;
  for (int v = c * s.chunk + threadIdx.x; v < end; v += kThreads) sum += mass_of(z[v], m, a.inv_t);
  sum = group_sum(sum, red);
  if (threadIdx.x == 0) w.mass[(int64_t)row * s.n_chunks + c] = sum;
}

// What the drafts of one sequence came to.
struct Verdict {
  int n;           // accepted drafts
  int refused;     // the draft refused (-1: none, the next token is the target's own)
  double pm, pi;   // maximum and 2^50 / S of the target row behind it
  double dm, di;   // of the drafter's row at it (with a drafter)
};

__device__ __forceinline__ double unit_over(uint64_t mass) {
  return mass ? kUnit / (double)mass : 0.0;
}
__device__ __forceinline__ uint64_t u24_of(float u) {
  return (uint64_t)floorf(fminf(fmaxf(u, 0.f), 0x1.fffffep-1f) * 0x1p24f);
}

__device__ __forceinline__ Verdict judge(const VerifyArgs& a, const Sizes& s, const Work& w, int b) {
#pragma clang fp contract(off)
  Verdict r;
  r.refused = -1;
  r.dm = r.di = 0.0;
  for (r.n = 0;; ++r.n) {
    const int row = b * (a.n_drafts + 1) + r.n;
    r.pm = row_max(w, s, row);
    r.pi = unit_over(row_mass(w, s, row));
    if (r.n == a.n_drafts) return r;
    const int x = a.drafts[b * a.n_drafts + r.n];
    if (x < 0 || x >= a.vocab) return r;
    const double px = (double)mass_of(a.target[(int64_t)row * a.vocab + x], r.pm, a.inv_t) * r.pi;
    double dx = kUnit;
    if (a.drafter) {
      const int i = b * a.n_drafts + r.n, drow = a.batch * (a.n_drafts + 1) + i;
      r.dm = row_max(w, s, drow);
      r.di = unit_over(row_mass(w, s, drow));
      dx = (double)mass_of(a.drafter[(int64_t)i * a.vocab + x], r.dm, a.inv_t) * r.di;
    }
    if (!((double)u24_of(a.uniforms[b * (a.n_drafts + 1) + r.n]) * dx < 0x1p24 * px)) {
      r.refused = x;
      return r;
    }
  }
}

// r_v of the next token's distribution, and rint(p_v).
__device__ __forceinline__ uint64_t rest_at(const VerifyArgs& a, const Verdict& r, int b, int v,
                                            uint64_t* whole) {
#pragma clang fp contract(off)
  const double p =
      (double)mass_of(a.target[((int64_t)b * (a.n_drafts + 1) + r.n) * a.vocab + v], r.pm, a.inv_t) *
      r.pi;
  *whole = (uint64_t)rint(p);
  if (r.refused < 0) return *whole;
  double d = 0.0;
  if (a.drafter)
    d = (double)mass_of(a.drafter[((int64_t)b * a.n_drafts + r.n) * a.vocab + v], r.dm, a.inv_t) *
        r.di;
  else if (v == r.refused)
    d = INFINITY;
  return (uint64_t)rint(fmax(p - d, 0.0));
}

__global__ __launch_bounds__(kThreads) void verify_rest_kernel(VerifyArgs a, Sizes s) {
  __shared__ uint64_t red[kWaves];
  const int b = blockIdx.x, c = blockIdx.y;
  const Work w = work_of(a.workspace, s, a.batch);
  const Verdict r = judge(a, s, w, b);
  const int end = min((c + 1) * s.chunk, a.vocab);
  uint64_t rest = 0, whole = 0;
  for (int v = c * s.chunk + threadIdx.x; v < end; v += kThreads) {
    uint64_t p;
    rest += rest_at(a, r, b, v, &p);
    whole += p;
  }
  rest = group_sum(rest, red);
  whole = group_sum(whole, red);
  if (threadIdx.x == 0) {
    w.rest[(int64_t)b * s.n_chunks + c] = rest;
    w.whole[(int64_t)b * s.n_chunks + c] = whole;
  }
}

__global__ __launch_bounds__(kThreads) void verify_pick_kernel(VerifyArgs a, Sizes s) {
  __shared__ uint64_t red[kWaves];
  __shared__ int found;
  const int b = blockIdx.x;
  const Work w = work_of(a.workspace, s, a.batch);
  const Verdict r = judge(a, s, w, b);
  uint64_t z = 0;
  for (int c = 0; c < s.n_chunks; ++c) z += w.rest[(int64_t)b * s.n_chunks + c];
  const bool own = z == 0;  // nothing left beside the drafter's: the target's own
  const uint64_t* part = (own ? w.whole : w.rest) + (int64_t)b * s.n_chunks;
  if (own)
    for (int c = 0; c < s.n_chunks; ++c) z += part[c];
  const uint64_t u = u24_of(a.uniforms[b * (a.n_drafts + 1) + a.n_drafts]);
  const uint64_t goal = (uint64_t)(((unsigned __int128)u * z) >> 24);
  uint64_t run = 0;
  int c = 0;
  while (c < s.n_chunks - 1 && run + part[c] <= goal) run += part[c++];
  if (threadIdx.x == 0) found = 0;
  const int end = min((c + 1) * s.chunk, a.vocab);
  if (z > 0) {
    for (int v0 = c * s.chunk; v0 < end; v0 += kThreads) {
      const int v = v0 + threadIdx.x;
      uint64_t p = 0, mine = 0;
      if (v < end) {
        mine = rest_at(a, r, b, v, &p);
        if (own) mine = p;
      }
      uint64_t incl = mine;
      const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const uint64_t t = __shfl_up(incl, o, 64);
        if (lane >= o) incl += t;
      }
      __syncthreads();
      if (lane == 63) red[wave] = incl;
      __syncthreads();
      uint64_t before = run, sum = 0;
#pragma unroll
      for (int i = 0; i < kWaves; ++i) {
        before += i < wave ? red[i] : 0;
        sum += red[i];
      }
      if (before + incl > goal && before + incl - mine <= goal) found = v;
      run += sum;
      if (run > goal) break;
    }
  }
  __syncthreads();
  for (int j = threadIdx.x; j <= a.n_drafts; j += kThreads)
    a.tokens[b * (a.n_drafts + 1) + j] =
        j < r.n ? a.drafts[b * a.n_drafts + j] : j == r.n ? found : -1;
  if (threadIdx.x == 0) a.accepted[b] = r.n;
}

}  // namespace

int64_t verify_workspace_bytes(int batch, int n_drafts, bool drafter, int vocab) {
  const Sizes s = sizes_of(batch, n_drafts, drafter, vocab);
  return ((int64_t)s.rows * 12 + (int64_t)batch * 16) * s.n_chunks;
}

hipError_t launch_verify(const VerifyArgs& a, hipStream_t stream) {
  const Sizes s = sizes_of(a.batch, a.n_drafts, a.drafter != nullptr, a.vocab);
  const dim3 all(s.rows, s.n_chunks), one(a.batch, s.n_chunks);
  verify_max_kernel<<<all, kThreads, 0, stream>>>(a, s);
  verify_mass_kernel<<<all, kThreads, 0, stream>>>(a, s);
  verify_rest_kernel<<<one, kThreads, 0, stream>>>(a, s);
  verify_pick_kernel<<<a.batch, kThreads, 0, stream>>>(a, s);
  return hipGetLastError();
}

}  // namespace pdec
