// C ABI of the operators over latent pages (append, attention of query tokens, pages as rows),
// of the attention of prompts over what latents expand to, and of page copies: argument checks
// and launches.  Lengths, starts and tables stay on the device, so nothing here waits, copies or
// allocates, and every call can be captured into a graph.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <string>

#include "../../include/pdec.h"
#include "kernels.h"
#include "paged_checks.h"
#include "paged_plan.h"
#include "status.h"

using namespace pdec;

namespace {

constexpr float kLog2E = 1.4426950408889634f;
constexpr int64_t kMaxRowStride = 1 << 24;  // elements: a tile's byte offsets stay in 32 bits

int check_pages(int32_t kv_dtype, int32_t latent_dim, const void* pages, const float* scales) {
  if (kv_dtype != PDEC_BF16 && kv_dtype != PDEC_FP8_E4M3)
    return fail(PDEC_INVALID_ARG, "kv_dtype must be PDEC_BF16 or PDEC_FP8_E4M3");
  if (latent_dim != 256 && latent_dim != 512)
    return fail(PDEC_UNSUPPORTED, "latent_dim must be 256 or 512");
  if (!pages) return fail(PDEC_INVALID_ARG, "null argument");
  if ((kv_dtype == PDEC_FP8_E4M3) != (scales != nullptr))
    return fail(PDEC_INVALID_ARG, "E4M3 pages take scales, the others none");
  if (!aligned(pages, 16) || !aligned(scales, 4))
    return fail(PDEC_INVALID_ARG, "pages must be 16-byte aligned");
  return PDEC_OK;
}

int check_queries(int32_t batch, int32_t n_q, int32_t n_heads) {
  if (batch < 1 || batch > kMaxBatch || n_q < 1 || n_q > 4096 || n_heads < 1 || n_heads > 1024)
    return fail(PDEC_INVALID_ARG,
                "batch must be positive, n_q in [1, 4096] and n_heads in [1, 1024]");
  return PDEC_OK;
}

bool good_scale(float s) { return s > 0.f && std::isfinite(s); }

struct Layout {
  int64_t ml, acc;  // byte offsets end here: ml, then ml + acc
};
Layout layout_of(int64_t n_units, const LatentPlan& p, int32_t latent) {
  const int64_t rows = (p.n_groups + n_units) * 16 * p.row_tiles;
  return {align_up(rows * 2 * 4), align_up(rows * latent * 4)};
}
Layout layout_of(const LatentPlan& p, int32_t latent) {
  if (p.unit_groups) return {0, 0};  // no partials
  return layout_of(p.n_units, p, latent);
}
Layout layout_of(const PromptPlan& p, int32_t n_heads, int32_t dim) {
  if (p.block_groups || p.n_groups == 1) return {0, 0};
  const int64_t rows = (int64_t)p.n_groups * 2 * n_heads * kPromptRows;
  return {align_up(rows * 2 * 4), align_up(rows * dim * 4)};
}

int check_prompt(int32_t n_rows, int32_t n_seqs, int32_t n_heads, int32_t dim) {
  if (n_rows < 0 || n_seqs < 1 || n_seqs > kMaxBatch || n_heads < 1 || n_heads > 1024)
    return fail(PDEC_INVALID_ARG, "bad n_rows, n_seqs or n_heads");
  if (dim != 64 && dim != 128) return fail(PDEC_UNSUPPORTED, "head_dim must be 64 or 128");
  return PDEC_OK;
}

}  // namespace

extern "C" {

int paged_latent_append(int32_t src_dtype, int32_t kv_dtype, int32_t n_rows, int32_t n_seqs,
                        int32_t n_heads, int32_t latent_dim, const void* x, int64_t x_stride,
                        const float* gain, float eps, int32_t interleaved, const void* q,
                        int64_t q_stride, int64_t q_head_stride, const int32_t* lens_dev,
                        const int32_t* row_start_dev, const int32_t* block_table_dev,
                        int32_t bt_stride, int64_t n_pages, const float* rope_dev, int32_t max_pos,
                        void* q_out, int64_t q_out_stride, int64_t q_out_head_stride, void* pages,
                        float* scales, void* stream) {
  if (src_dtype != PDEC_F32 && src_dtype != PDEC_BF16)
    return fail(PDEC_INVALID_ARG, "src_dtype must be PDEC_F32 or PDEC_BF16");
  int rc = check_pages(kv_dtype, latent_dim, pages, scales);
  if (rc == PDEC_OK) rc = check_table(n_seqs, bt_stride, n_pages);
  if (rc != PDEC_OK) return rc;
  if (!x || !lens_dev || !row_start_dev || !block_table_dev || !rope_dev ||
      (q != nullptr) != (q_out != nullptr))
    return fail(PDEC_INVALID_ARG, "null argument");
  if (n_rows < 0 || max_pos < 1) return fail(PDEC_INVALID_ARG, "bad n_rows or max_pos");
  if (interleaved != 0 && interleaved != 1)
    return fail(PDEC_INVALID_ARG, "interleaved must be 0 or 1");
  if (!(eps >= 0.f) || !std::isfinite(eps))
    return fail(PDEC_INVALID_ARG, "eps must be 0 or more, and finite");
  if (x_stride < latent_dim + kLatentRope)
    return fail(PDEC_INVALID_ARG, "row strides shorter than a row");
  if (q) {
    if (n_heads < 1 || n_heads > 1024) return fail(PDEC_INVALID_ARG, "n_heads in [1, 1024]");
    if (q_head_stride < kLatentRope || q_out_head_stride < kLatentRope ||
        q_stride < (n_heads - 1) * q_head_stride + kLatentRope ||
        q_out_stride < (n_heads - 1) * q_out_head_stride + kLatentRope)
      return fail(PDEC_INVALID_ARG, "query strides shorter than a head or a row");
  }
  if (!aligned(rope_dev, 16) || !aligned(gain, 16))
    return fail(PDEC_INVALID_ARG, "table and gain must be 16-byte aligned");
  LatentAppendArgs a{};
  a.x = x;
  a.q = q;
  a.x_stride = x_stride;
  a.q_stride = q_stride;
  a.q_head = q_head_stride;
  a.q_out_stride = q_out_stride;
  a.q_out_head = q_out_head_stride;
  a.n_rows = n_rows;
  a.n_seqs = n_seqs;
  a.n_heads = n_heads;
  a.interleaved = interleaved;
  a.lens = lens_dev;
  a.row_start = row_start_dev;
  a.block_table = block_table_dev;
  a.bt_stride = bt_stride;
  a.max_pos = max_pos;
  a.n_pages = n_pages;
  a.rope = (const float2*)rope_dev;
  a.gain = gain;
  a.eps = eps;
  a.q_out = q_out;
  a.pages = pages;
  a.scales = scales;
  if (latent_append_threads(a) > kMaxLaunch)
    return fail(PDEC_INVALID_ARG, "too many rows for one call");
  HIP_OR_FAIL(launch_latent_append(src_dtype == PDEC_BF16, kv_dtype == PDEC_FP8_E4M3, latent_dim, a,
                                   (hipStream_t)stream));
  return PDEC_OK;
}

int paged_latent_rows(int32_t kv_dtype, int32_t n_rows, int32_t n_seqs, int32_t latent_dim,
                      const void* pages, const float* scales, const int32_t* lens_dev,
                      const int32_t* row_start_dev, const int32_t* block_table_dev,
                      int32_t bt_stride, int64_t n_pages, void* latents, void* rope_keys,
                      void* stream) {
  int rc = check_pages(kv_dtype, latent_dim, pages, scales);
  if (rc == PDEC_OK) rc = check_table(n_seqs, bt_stride, n_pages);
  if (rc != PDEC_OK) return rc;
  if (!lens_dev || !row_start_dev || !block_table_dev || !latents || !rope_keys)
    return fail(PDEC_INVALID_ARG, "null argument");
  if (n_rows < 0) return fail(PDEC_INVALID_ARG, "bad n_rows");
  if (!aligned(latents, 16) || !aligned(rope_keys, 16))
    return fail(PDEC_INVALID_ARG, "rows must be 16-byte aligned");
  LatentRowsArgs a{};
  a.pages = pages;
  a.scales = scales;
  a.lens = lens_dev;
  a.row_start = row_start_dev;
  a.block_table = block_table_dev;
  a.bt_stride = bt_stride;
  a.n_rows = n_rows;
  a.n_seqs = n_seqs;
  a.n_pages = n_pages;
  a.latents = latents;
  a.rope_keys = rope_keys;
  if (latent_rows_threads(a) > kMaxLaunch)
    return fail(PDEC_INVALID_ARG, "too many rows for one call");
  HIP_OR_FAIL(launch_latent_rows(kv_dtype == PDEC_FP8_E4M3, latent_dim, a, (hipStream_t)stream));
  return PDEC_OK;
}

int64_t paged_latent_attention_workspace_bytes(int32_t kv_dtype, int32_t batch, int32_t n_q,
                                               int32_t n_heads, int32_t latent_dim,
                                               int32_t max_pages) {
  if (kv_dtype != PDEC_BF16 && kv_dtype != PDEC_FP8_E4M3)
    return fail(PDEC_INVALID_ARG, "kv_dtype must be PDEC_BF16 or PDEC_FP8_E4M3");
  if (latent_dim != 256 && latent_dim != 512)
    return fail(PDEC_UNSUPPORTED, "latent_dim must be 256 or 512");
  const int rc = check_queries(batch, n_q, n_heads);
  if (rc != PDEC_OK) return rc;
  if (max_pages < 1 || max_pages > kMaxStride) return fail(PDEC_INVALID_ARG, "bad max_pages");
  // Fewer sequences, tokens or pages of the same take blocks of as many row tiles or fewer, and
  // as many units or fewer, but have partials where these units may be too many to have any: as
  // many as just have, of this call's blocks, and of blocks of one row tile, a sequence each.
  const int64_t max_len = (int64_t)max_pages * PDEC_PAGE_TOKENS;
  const LatentPlan p = plan_latent_attention(
      batch, n_q, n_heads, max_len, latent_tile(kv_dtype == PDEC_FP8_E4M3, latent_dim));
  const int64_t most = latent_units(p.row_tiles, max_len), most_few = latent_units(1, max_len);
  if (p.unit_groups && p.n_units < most) return 0;  // no table is long
  LatentPlan few = p;
  few.row_tiles = 1;
  const Layout l = layout_of(std::min(p.n_units, most - 1), p, latent_dim);
  const Layout f = layout_of(std::min<int64_t>(batch, most_few - 1), few, latent_dim);
  return std::max(l.ml + l.acc, f.ml + f.acc);
}

int paged_latent_attention(int32_t kv_dtype, int32_t batch, int32_t n_q, int32_t n_heads,
                           int32_t latent_dim, const void* q, const void* pages,
                           const float* scales, int64_t n_pages, const int32_t* block_table_dev,
                           int32_t bt_stride, const int32_t* lens_dev, float softmax_scale,
                           void* out, void* workspace, int64_t workspace_bytes, void* stream) {
  int rc = check_pages(kv_dtype, latent_dim, pages, scales);
  if (rc == PDEC_OK) rc = check_queries(batch, n_q, n_heads);
  if (rc == PDEC_OK) rc = check_table(batch, bt_stride, n_pages);
  if (rc != PDEC_OK) return rc;
  if (!q || !block_table_dev || !lens_dev || !out) return fail(PDEC_INVALID_ARG, "null argument");
  if (!good_scale(softmax_scale))
    return fail(PDEC_INVALID_ARG, "softmax_scale must be positive and finite");
  if (!aligned(q, 16) || !aligned(out, 16) || !aligned(workspace, 16))
    return fail(PDEC_INVALID_ARG, "q, out and workspace must be 16-byte aligned");
  const bool fp8 = kv_dtype == PDEC_FP8_E4M3;
  const int tile = latent_tile(fp8, latent_dim);
  const LatentPlan p = plan_latent_attention(batch, n_q, n_heads,
                                             (int64_t)bt_stride * PDEC_PAGE_TOKENS, tile);
  if (p.n_units * ((int64_t)bt_stride + 1) > INT32_MAX || p.n_units * 512 > kMaxLaunch)
    return fail(PDEC_INVALID_ARG, "batch x bt_stride too large for one call");
  const Layout l = layout_of(p, latent_dim);
  if (workspace_bytes < l.ml + l.acc || (l.ml > 0 && !workspace))
    return fail(PDEC_INVALID_ARG, "workspace too small: need " + std::to_string(l.ml + l.acc));
  LatentAttnArgs a{};
  a.q = q;
  a.pages = pages;
  a.scales = scales;
  a.block_table = block_table_dev;
  a.lens = lens_dev;
  a.bt_stride = bt_stride;
  a.max_len = bt_stride * PDEC_PAGE_TOKENS;
  a.n_q = n_q;
  a.n_heads = n_heads;
  a.n_pages = n_pages;
  a.block_rows = p.block_rows;
  a.blocks_per_seq = p.blocks_per_seq;
  a.n_units = (int32_t)p.n_units;
  a.n_groups = p.n_groups;
  a.min_tiles = 2;
  a.unit_groups = p.unit_groups;
  a.scale_log2 = softmax_scale * kLog2E;
  a.part_ml = (float*)workspace;
  a.part_acc = (float*)((char*)workspace + l.ml);
  a.out = out;
  HIP_OR_FAIL(launch_latent_attention(fp8, latent_dim, p.row_tiles, a, (hipStream_t)stream));
  return PDEC_OK;
}

int64_t latent_prompt_attention_workspace_bytes(int32_t n_rows, int32_t n_seqs, int32_t n_heads,
                                                int32_t head_dim) {
  const int rc = check_prompt(n_rows, n_seqs, n_heads, head_dim);
  if (rc != PDEC_OK) return rc;
  // Whatever n_keys is, and what fewer rows would take.
  const Layout l = layout_of(plan_latent_prompt(0, 0, 1, n_heads), n_heads, head_dim);
  return l.ml + l.acc;
}

int latent_prompt_attention(int32_t n_rows, int32_t n_keys, int32_t n_seqs, int32_t n_heads,
                            int32_t head_dim, const void* q, int64_t q_stride,
                            int64_t q_head_stride, const void* k, int64_t k_stride,
                            int64_t k_head_stride, const void* rope_keys, int64_t rope_stride,
                            const void* v, int64_t v_stride, int64_t v_head_stride,
                            const int32_t* q_start_dev, const int32_t* k_start_dev,
                            float softmax_scale, void* out, void* workspace,
                            int64_t workspace_bytes, void* stream) {
  const int rc = check_prompt(n_rows, n_seqs, n_heads, head_dim);
  if (rc != PDEC_OK) return rc;
  if (n_keys < 0) return fail(PDEC_INVALID_ARG, "bad n_keys");
  if (!q_start_dev || !k_start_dev || (n_rows > 0 && (!q || !out)) ||
      (n_keys > 0 && (!k || !rope_keys || !v)))
    return fail(PDEC_INVALID_ARG, "null argument");
  if (!good_scale(softmax_scale))
    return fail(PDEC_INVALID_ARG, "softmax_scale must be positive and finite");
  const int64_t heads = n_heads - 1;
  if (q_head_stride < head_dim + kLatentRope ||
      q_stride < heads * q_head_stride + head_dim + kLatentRope || k_head_stride < head_dim ||
      k_stride < heads * k_head_stride + head_dim || v_head_stride < head_dim ||
      v_stride < heads * v_head_stride + head_dim || rope_stride < kLatentRope)
    return fail(PDEC_INVALID_ARG, "strides shorter than a head or a row");
  if ((q_stride | q_head_stride | k_stride | k_head_stride | rope_stride | v_stride |
       v_head_stride) % 8 ||
      !aligned(q, 16) || !aligned(k, 16) || !aligned(rope_keys, 16) || !aligned(v, 16) ||
      !aligned(out, 16) || !aligned(workspace, 16))
    return fail(PDEC_INVALID_ARG, "rows, heads, out and workspace must be 16-byte aligned");
  if (k_stride > kMaxRowStride || v_stride > kMaxRowStride || rope_stride > kMaxRowStride)
    return fail(PDEC_INVALID_ARG, "rows further than 2^24 elements apart");
  const PromptPlan p = plan_latent_prompt(n_rows, n_keys, n_seqs, n_heads);
  // Blocks are of 128 rows, tiles of 32 keys, and four count for what a block costs beside.
  if (((int64_t)n_rows / 128 + n_seqs) * ((int64_t)n_keys / 32 + 6) > INT32_MAX ||
      (int64_t)p.n_groups * n_heads * 512 > kMaxLaunch)
    return fail(PDEC_INVALID_ARG, "too many rows and keys for one call");
  const Layout l = layout_of(p, n_heads, head_dim);
  if (workspace_bytes < l.ml + l.acc || (l.ml > 0 && !workspace))
    return fail(PDEC_INVALID_ARG, "workspace too small: need " + std::to_string(l.ml + l.acc));
  if (n_rows == 0) return PDEC_OK;
  LatentPromptArgs a{};
  a.q = (const uint16_t*)q;
  a.k = (const uint16_t*)k;
  a.rope_keys = (const uint16_t*)rope_keys;
  a.v = (const uint16_t*)v;
  a.q_stride = q_stride;
  a.q_head = q_head_stride;
  a.k_stride = k_stride;
  a.k_head = k_head_stride;
  a.r_stride = rope_stride;
  a.v_stride = v_stride;
  a.v_head = v_head_stride;
  a.q_start = q_start_dev;
  a.k_start = k_start_dev;
  a.n_rows = n_rows;
  a.n_keys = n_keys;
  a.n_seqs = n_seqs;
  a.n_heads = n_heads;
  a.block_groups = p.block_groups;
  a.min_tiles = 4;
  a.scale_log2 = softmax_scale * kLog2E;
  a.part_ml = (float*)workspace;
  a.part_acc = (float*)((char*)workspace + l.ml);
  a.out = (uint16_t*)out;
  HIP_OR_FAIL(launch_latent_prompt(head_dim, p.n_groups, a, (hipStream_t)stream));
  return PDEC_OK;
}

int paged_copy_pages(int32_t n_pools, void* const* pools, const int64_t* page_bytes,
                     int64_t n_pages, int32_t n_pairs, const int32_t* src_dev,
                     const int32_t* dst_dev, void* stream) {
  if (n_pools < 1 || n_pools > 4096 || !pools || !page_bytes)
    return fail(PDEC_INVALID_ARG, "n_pools must be in [1, 4096], with pools and page_bytes");
  if (n_pages < 1 || n_pages > INT32_MAX || n_pairs < 0)
    return fail(PDEC_INVALID_ARG, "bad n_pages or n_pairs");
  if (n_pairs > 0 && (!src_dev || !dst_dev)) return fail(PDEC_INVALID_ARG, "null argument");
  if ((int64_t)n_pairs * 256 > kMaxLaunch) return fail(PDEC_INVALID_ARG, "too many pairs");
  PageCopyArgs a{};
  a.n_pages = n_pages;
  a.n_pairs = n_pairs;
  a.src = src_dev;
  a.dst = dst_dev;
  for (int i = 0; i < n_pools; ++i) {  // all are looked at before any is written
    if (!pools[i] || page_bytes[i] < 1 || page_bytes[i] > (1 << 27))
      return fail(PDEC_INVALID_ARG, "a pool is null, or its pages not in [1, 2^27] bytes");
    if (page_bytes[i] == 1 << 27 && !aligned(pools[i], 4))  // copied byte by byte
      return fail(PDEC_INVALID_ARG, "pages of unaligned pools too large");
  }
  for (int i = 0; i < n_pools;) {  // as many pools a launch as fit its arguments
    for (a.n_pools = 0; i < n_pools && a.n_pools < kCopyPools; ++i, ++a.n_pools) {
      a.pool[a.n_pools] = pools[i];
      a.bytes[a.n_pools] = page_bytes[i];
    }
    HIP_OR_FAIL(launch_page_copy(a, (hipStream_t)stream));
  }
  return PDEC_OK;
}

}  // extern "C"
