// Latent pages: appending new tokens to them, and reading them back as rows.
//
// A token's row is its latent of R elements, then its rotary key of 64.  bf16 pages hold
// [16][R + 64]; E4M3 pages [16][R + 128] bytes, the latent as codes and the rotary key in bf16,
// with a scale for each token (the smallest power of two s with max|c| <= 448 s), so that a
// token is written without a look at its page's others.
//
// Append.  c = x * rsqrt(mean(x^2) + eps) * gain over the row's first R elements, rounded once,
// to the page's type; the last 64 are rotated at the token's position, as are 64 elements of
// each query head.  A wave takes a row's latent and key, or eight query heads of a row; each
// finds its sequence, page and slot by itself.  Bound by memory: 4096 rows from fp32, with 32
// heads' queries, 65 MB in 14 us (4.6 TB/s); 64 rows 4.5 us, the chain of looks from a row to
// its page.
//
// Gather.  Bound by memory (a row's 1152 or 644 bytes read, 1152 written), and for few rows by the
// chain of looks from a row to its page, which the lanes go at once, one a row.  A wave takes four
// rows, all their loads in flight; 54 000 E4M3 rows of 512 in 24 us (4.0 TB/s); two rows a wave
// 29.3, one 35.0, six, whose registers leave few waves, 35.3.  Stores past the caches make the call
// shorter (17 us), but the projection that reads the rows next longer by more: both together, to
// 1280 / 2560 / 5120 / 8192 columns, take +25 / +3 / -1 / +2 us, of 30 000 rows +12 / +11 / +56 /
// +7, of 100 000 +9 / 0 / 0 / 0.
#include "hip_common.h"
#include "kernels.h"
#include "rows.h"
#include "wave.h"

#include <type_traits>

namespace pdec {

namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64, kRope = kLatentRope;
constexpr int kGather = 4;  // rows of a wave

typedef uint16_t u16x2_any __attribute__((ext_vector_type(2), aligned(2)));
typedef float f32x2_any __attribute__((ext_vector_type(2), aligned(4)));

__device__ __forceinline__ f32x2 read2(const float* p) { return *(const f32x2_any*)p; }
__device__ __forceinline__ f32x2 read2(const uint16_t* p) {
  const u16x2_any v = *(const u16x2_any*)p;
  return f32x2{bf16_to_f32(v.x), bf16_to_f32(v.y)};
}
// To nearest even; NaN of any payload stays NaN.
__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
}
__device__ __forceinline__ f32x2 rotate(f32x2 x, float2 cs) {
  return f32x2{x[0] * cs.x - x[1] * cs.y, x[0] * cs.y + x[1] * cs.x};
}

// Position of row r of sequence b, or -1 where the table has no place for it.
__device__ __forceinline__ int position(const int32_t* lens, const int32_t* row_start, int b, int r,
                                        int64_t limit) {
  const int64_t pos = (int64_t)lens[b] - ((int64_t)row_start[b + 1] - r);
  return pos >= 0 && pos < limit ? (int)pos : -1;
}

template <typename ST, bool FP8, int R>
__global__ __launch_bounds__(kThreads) void latent_append_kernel(LatentAppendArgs a, int q_waves) {
  constexpr int E = R / 64;  // latent elements of a lane
  const int lane = threadIdx.x & 63;
  const int64_t item = (int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6);
  const int r = (int)(item / (1 + q_waves)), part = (int)(item % (1 + q_waves));
  if (r >= a.n_rows) return;
  // The row's own loads are under way while its sequence is looked for.
  const bool latent = part == 0;
  const ST* x = (const ST*)a.x + (int64_t)r * a.x_stride;
  const int head = (part - 1) * 8 + lane / 8, i4 = lane % 8 * 4;  // a query head, four pairs of it
  const bool on = latent || head < a.n_heads;
  const ST* q = (const ST*)a.q + (int64_t)r * a.q_stride + head * a.q_head;
  f32x4 v[E / 4], lo = {0.f, 0.f, 0.f, 0.f}, hi = lo;
  f32x2 key = {0.f, 0.f};
  if (latent) {
#pragma unroll
    for (int i = 0; i < E / 4; ++i) v[i] = read4(x + lane * E + i * 4);
    if (lane < kRope / 2) {
      if (a.interleaved) key = read2(x + R + 2 * lane);
      else key = f32x2{read1(x + R + lane), read1(x + R + kRope / 2 + lane)};
    }
  } else if (on) {
    lo = read4(q + (a.interleaved ? 2 * i4 : i4));
    hi = read4(q + (a.interleaved ? 2 * i4 + 4 : i4 + kRope / 2));
  }
  const int b = find_seq(a.row_start, a.n_seqs, a.n_rows, r);
  if (b < 0) return;
  const int pos = position(a.lens, a.row_start, b, r,
                           min((int64_t)a.max_pos, (int64_t)a.bt_stride * kPage));
  if (pos < 0) return;
  const float2* cs = a.rope + (int64_t)pos * (kRope / 2);
  if (!latent) {
    if (!on) return;
    uint16_t* to = (uint16_t*)a.q_out + (int64_t)r * a.q_out_stride + head * a.q_out_head;
    const float4 t01 = *(const float4*)(cs + i4), t23 = *(const float4*)(cs + i4 + 2);
    const float2 t[4] = {{t01.x, t01.y}, {t01.z, t01.w}, {t23.x, t23.y}, {t23.z, t23.w}};
    f32x2 p[4];
    if (a.interleaved) {
      p[0] = f32x2{lo[0], lo[1]}, p[1] = f32x2{lo[2], lo[3]};
      p[2] = f32x2{hi[0], hi[1]}, p[3] = f32x2{hi[2], hi[3]};
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) p[i] = f32x2{lo[i], hi[i]};
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = rotate(p[i], t[i]);
    u32x2 s0, s1;
    if (a.interleaved) {
      s0 = u32x2{bf16_pair(p[0][0], p[0][1]), bf16_pair(p[1][0], p[1][1])};
      s1 = u32x2{bf16_pair(p[2][0], p[2][1]), bf16_pair(p[3][0], p[3][1])};
    } else {
      s0 = u32x2{bf16_pair(p[0][0], p[1][0]), bf16_pair(p[2][0], p[3][0])};
      s1 = u32x2{bf16_pair(p[0][1], p[1][1]), bf16_pair(p[2][1], p[3][1])};
    }
    *(u16x4_any*)(to + (a.interleaved ? 2 * i4 : i4)) = __builtin_bit_cast(u16x4_any, s0);
    *(u16x4_any*)(to + (a.interleaved ? 2 * i4 + 4 : i4 + kRope / 2)) =
        __builtin_bit_cast(u16x4_any, s1);
    return;
  }
  const int64_t page = a.block_table[(int64_t)b * a.bt_stride + pos / kPage];
  if (page < 0 || page >= a.n_pages) return;
  if (a.gain) {
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < E; ++i) sum += v[i / 4][i % 4] * v[i / 4][i % 4];
    const float inv = rsqrtf(wave_add(sum) * (1.f / R) + a.eps);
#pragma unroll
    for (int i = 0; i < E / 4; ++i) v[i] = v[i] * inv * *(const f32x4*)(a.gain + lane * E + i * 4);
  }
  constexpr int kRowBytes = FP8 ? R + 2 * kRope : 2 * (R + kRope);
  uint8_t* row = (uint8_t*)a.pages + (page * kPage + pos % kPage) * kRowBytes;
  uint8_t* rope = row + (FP8 ? R : 2 * R);
  if constexpr (FP8) {
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < E; ++i) top = fmaxf(top, fabsf(v[i / 4][i % 4]));
    const float scale = scale_for(wave_top(top)), inv = inverse_pow2(scale);
    uint32_t codes[E / 4];
#pragma unroll
    for (int i = 0; i < E / 4; ++i) {
      codes[i] = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) codes[i] |= e4m3_from_f32(v[i][e] * inv) << (8 * e);
    }
    if constexpr (E == 8) *(u32x2*)(row + lane * 8) = u32x2{codes[0], codes[1]};
    else *(uint32_t*)(row + lane * 4) = codes[0];
    if (lane == 0) a.scales[page * kPage + pos % kPage] = scale;
  } else {
    u32x2 w[E / 4];
#pragma unroll
    for (int i = 0; i < E / 4; ++i)
      w[i] = u32x2{bf16_pair(v[i][0], v[i][1]), bf16_pair(v[i][2], v[i][3])};
    if constexpr (E == 8) *(u32x4*)(row + lane * 16) = u32x4{w[0].x, w[0].y, w[1].x, w[1].y};
    else *(u32x2*)(row + lane * 8) = w[0];
  }
  if (lane < kRope / 2) {
    const f32x2 p = rotate(key, cs[lane]);
    const uint32_t bits = bf16_pair(p[0], p[1]);
    if (a.interleaved) {
      *(uint32_t*)(rope + lane * 4) = bits;
    } else {
      *(uint16_t*)(rope + lane * 2) = (uint16_t)bits;
      *(uint16_t*)(rope + kRope + lane * 2) = (uint16_t)(bits >> 16);
    }
  }
}

template <bool FP8, int R>
__global__ __launch_bounds__(kThreads) void latent_rows_kernel(LatentRowsArgs a) {
  constexpr int kRowBytes = FP8 ? R + 2 * kRope : 2 * (R + kRope);
  constexpr int CL = R / 8;  // lanes of a latent, eight elements each; eight more of the key
  const int lane = threadIdx.x & 63;
  const int64_t r0 = ((int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6)) * kGather;
  const int64_t limit = (int64_t)a.bt_stride * kPage;
  if (r0 >= a.n_rows) return;
  // Lane i finds row r0 + i's place in the pool, -1 for none; a wave's rows are most often of one
  // sequence, looked for once.
  int64_t place = -1;
  {
    const int64_t r = r0 + min(lane, kGather - 1);
    bool open = lane < kGather && r < a.n_rows;
    for (uint64_t rest; (rest = __ballot(open)) != 0;) {
      const int first = (int)r0 + (int)__builtin_ctzll(rest);
      const int b = find_seq(a.row_start, a.n_seqs, a.n_rows, first);
      if (b < 0) {  // of no sequence
        open = open && r != first;
      } else if (open && r < a.row_start[b + 1]) {
        open = false;
        const int pos = position(a.lens, a.row_start, b, (int)r, limit);
        const int64_t page = pos < 0 ? -1 : a.block_table[(int64_t)b * a.bt_stride + pos / kPage];
        if (page >= 0 && page < a.n_pages) place = page * kPage + pos % kPage;
      }
    }
  }
  float scale = 0.f;
  if constexpr (FP8)
    if (place >= 0) scale = a.scales[place];
  auto slot = [&](int i) {
    return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(place >> 32), i) << 32 |
                     (uint32_t)__builtin_amdgcn_readlane((int)place, i));
  };
  u32x4 x[kGather], k[kGather];
#pragma unroll
  for (int i = 0; i < kGather; ++i) {
    if (slot(i) < 0) continue;
    const uint8_t* row = (const uint8_t*)a.pages + slot(i) * kRowBytes;
    if (lane < CL) {
      if constexpr (FP8) {
        const u32x2 codes = *(const u32x2*)(row + lane * 8);
        x[i].x = codes.x, x[i].y = codes.y;
      } else {
        x[i] = *(const u32x4*)(row + lane * 16);
      }
    }
    if (lane < 8) k[i] = *(const u32x4*)(row + (FP8 ? R : 2 * R) + lane * 16);
  }
#pragma unroll
  for (int i = 0; i < kGather; ++i) {
    if (slot(i) < 0) continue;
    if constexpr (FP8) {
      const float f = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(scale), i));
      u32x4 o;
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        const int word = (int)(h < 2 ? x[i].x : x[i].y);
        const f32x2 v = h & 1 ? __builtin_amdgcn_cvt_pk_f32_fp8(word, true)
                              : __builtin_amdgcn_cvt_pk_f32_fp8(word, false);
        o[h] = bf16_pair(v[0] * f, v[1] * f);
      }
      x[i] = o;
    }
    u32x4* to = (u32x4*)((uint16_t*)a.latents + (r0 + i) * R + lane * 8);
    u32x4* key_to = (u32x4*)((uint16_t*)a.rope_keys + (r0 + i) * kRope + lane * 8);
    if (lane < CL) *to = x[i];
    if (lane < 8) *key_to = k[i];
  }
}

int q_waves_of(const LatentAppendArgs& a) { return a.q ? (a.n_heads + 7) / 8 : 0; }
int64_t append_groups(const LatentAppendArgs& a) {
  return ((int64_t)a.n_rows * (1 + q_waves_of(a)) + kWaves - 1) / kWaves;
}
int64_t rows_groups(const LatentRowsArgs& a) {
  return ((int64_t)a.n_rows + kWaves * kGather - 1) / (kWaves * kGather);
}

}  // namespace

int64_t latent_append_threads(const LatentAppendArgs& a) { return append_groups(a) * kThreads; }
int64_t latent_rows_threads(const LatentRowsArgs& a) { return rows_groups(a) * kThreads; }

hipError_t launch_latent_append(int src_bf16, int fp8, int latent, const LatentAppendArgs& a,
                                hipStream_t stream) {
  if (a.n_rows == 0) return hipSuccess;
  const dim3 grid((uint32_t)append_groups(a)), block(kThreads);
  const int qw = q_waves_of(a);
#define PDEC_LATENT(ST_, FP8_)                                                              \
  do {                                                                                      \
    if (latent == 512) latent_append_kernel<ST_, FP8_, 512><<<grid, block, 0, stream>>>(a, qw); \
    else latent_append_kernel<ST_, FP8_, 256><<<grid, block, 0, stream>>>(a, qw);           \
  } while (0)
  if (src_bf16) {
    if (fp8) PDEC_LATENT(uint16_t, true);
    else PDEC_LATENT(uint16_t, false);
  } else {
    if (fp8) PDEC_LATENT(float, true);
    else PDEC_LATENT(float, false);
  }
#undef PDEC_LATENT
  return hipGetLastError();
}

hipError_t launch_latent_rows(int fp8, int latent, const LatentRowsArgs& a, hipStream_t stream) {
  if (a.n_rows == 0) return hipSuccess;
  const dim3 grid((uint32_t)rows_groups(a)), block(kThreads);
#define PDEC_ROWS(FP8_, R_) latent_rows_kernel<FP8_, R_><<<grid, block, 0, stream>>>(a)
  if (latent == 512) {
    if (fp8) PDEC_ROWS(true, 512);
    else PDEC_ROWS(false, 512);
  } else {
    if (fp8) PDEC_ROWS(true, 256);
    else PDEC_ROWS(false, 256);
  }
#undef PDEC_ROWS
  return hipGetLastError();
}

}  // namespace pdec
