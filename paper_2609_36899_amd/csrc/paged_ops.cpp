// C ABI of the operators over caller-owned pages (append, attention of query
// tokens, page selection) and of draft verification: argument checks and launches.
// The lengths and tables stay on the device, so nothing here waits, copies or
// allocates, and every call can be captured into a graph.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <string>

#include "../../include/pdec.h"
#include "kernels.h"
#include "status.h"

using namespace pdec;

namespace {

constexpr int64_t kMaxStride = 1 << 22;  // pages of a table row: 2^26 positions
constexpr int64_t kMaxBatch = 1 << 20;

int64_t align_up(int64_t v) { return (v + 255) / 256 * 256; }
bool aligned(const void* p, int bytes) { return (uintptr_t)p % bytes == 0; }

int check_heads(int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim) {
  if (n_q_heads < 1 || n_kv_heads < 1 || n_kv_heads > 65535 || n_q_heads % n_kv_heads)
    return fail(PDEC_INVALID_ARG, "n_q_heads must be a positive multiple of n_kv_heads");
  if (n_q_heads / n_kv_heads > 16)
    return fail(PDEC_UNSUPPORTED, "GQA group size must be at most 16");
  if (head_dim != 64 && head_dim != 128)
    return fail(PDEC_UNSUPPORTED, "head_dim must be 64 or 128");
  return PDEC_OK;
}

int check_table(int32_t batch, int32_t bt_stride, int64_t n_pages) {
  if (batch < 1 || batch > kMaxBatch || bt_stride < 1 || bt_stride > kMaxStride || n_pages < 1 ||
      n_pages > INT32_MAX)
    return fail(PDEC_INVALID_ARG, "bad batch, bt_stride or n_pages");
  return PDEC_OK;
}

struct TokenAttnLayout {
  int64_t ml, acc;  // byte offsets end here: ml, then ml + acc
};
TokenAttnLayout layout_of(int64_t n_units, const PagedAttnPlan& p, int32_t n_kv_heads,
                          int32_t head_dim) {
  const int64_t rows = (p.n_groups + n_units) * n_kv_heads * 16 * p.row_tiles;
  return {align_up(rows * 2 * 4), align_up(rows * head_dim * 4)};
}
TokenAttnLayout layout_of(const PagedAttnPlan& p, int32_t n_kv_heads, int32_t head_dim) {
  if (p.unit_groups) return {0, 0};  // no partials
  return layout_of(p.n_units, p, n_kv_heads, head_dim);
}

int check_token_attention(int32_t batch, int32_t n_q, int32_t n_q_heads, int32_t n_kv_heads,
                          int32_t head_dim) {
  const int rc = check_heads(n_q_heads, n_kv_heads, head_dim);
  if (rc != PDEC_OK) return rc;
  if (batch < 1 || batch > kMaxBatch || n_q < 1 || n_q > 4096)
    return fail(PDEC_INVALID_ARG, "batch must be positive and n_q in [1, 4096]");
  return PDEC_OK;
}

}  // namespace

extern "C" {

int rope_table(int32_t max_pos, int32_t head_dim, float base, float* table_dev, void* stream) {
  if (!table_dev) return fail(PDEC_INVALID_ARG, "null argument");
  if (max_pos < 1 || head_dim < 2 || head_dim % 2 || !(base > 0.f) || !std::isfinite(base))
    return fail(PDEC_INVALID_ARG, "bad rotary table arguments");
  if (!aligned(table_dev, 8)) return fail(PDEC_INVALID_ARG, "table must be 8-byte aligned");
  HIP_OR_FAIL(launch_rope_table(max_pos, head_dim, base, (float2*)table_dev, (hipStream_t)stream));
  return PDEC_OK;
}

int paged_kv_append(int32_t src_dtype, int32_t kv_dtype, int32_t n_rows, int32_t n_seqs,
                    int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, const void* q,
                    int64_t q_stride, const void* k, int64_t k_stride, const void* v,
                    int64_t v_stride, const int32_t* lens_dev, const int32_t* row_start_dev,
                    const int32_t* block_table_dev, int32_t bt_stride, int64_t n_pages,
                    const float* rope_dev, int32_t max_pos, void* q_out, void* k_pages,
                    void* v_pages, float* k_scales, float* v_scales, void* k_means, void* stream) {
  if (src_dtype != PDEC_F32 && src_dtype != PDEC_BF16)
    return fail(PDEC_INVALID_ARG, "src_dtype must be PDEC_F32 or PDEC_BF16");
  if (kv_dtype != PDEC_F32 && kv_dtype != PDEC_BF16 && kv_dtype != PDEC_FP8_E4M3)
    return fail(PDEC_INVALID_ARG, "bad kv_dtype");
  if (kv_dtype == PDEC_F32 && src_dtype != PDEC_F32)
    return fail(PDEC_UNSUPPORTED, "fp32 pages take fp32 rows");
  if (!k || !v || !lens_dev || !row_start_dev || !block_table_dev || !rope_dev || !k_pages ||
      !v_pages || (q != nullptr) != (q_out != nullptr))
    return fail(PDEC_INVALID_ARG, "null argument");
  if (!q) n_q_heads = n_kv_heads;
  int rc = check_heads(n_q_heads, n_kv_heads, head_dim);
  if (rc == PDEC_OK) rc = check_table(n_seqs, bt_stride, n_pages);
  if (rc != PDEC_OK) return rc;
  if (n_rows < 0 || max_pos < 1) return fail(PDEC_INVALID_ARG, "bad n_rows or max_pos");
  const int64_t kv_cols = (int64_t)n_kv_heads * head_dim;
  if (k_stride < kv_cols || v_stride < kv_cols ||
      (q && q_stride < (int64_t)n_q_heads * head_dim))
    return fail(PDEC_INVALID_ARG, "row strides shorter than a row");
  const bool fp8 = kv_dtype == PDEC_FP8_E4M3;
  if (fp8 != (k_scales != nullptr) || fp8 != (v_scales != nullptr))
    return fail(PDEC_INVALID_ARG, "E4M3 pages take scales, the others none");
  if (k_means && kv_dtype == PDEC_F32)
    return fail(PDEC_UNSUPPORTED, "key means are kept of bf16 and E4M3 pages");
  if (!aligned(k_pages, 16) || !aligned(v_pages, 16) || !aligned(rope_dev, 16) ||
      !aligned(q_out, 16))
    return fail(PDEC_INVALID_ARG, "pages, table and q_out must be 16-byte aligned");
  AppendArgs a{};
  a.k = k;
  a.v = v;
  a.q = q;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.q_stride = q_stride;
  a.n_rows = n_rows;
  a.n_seqs = n_seqs;
  a.n_q_heads = n_q_heads;
  a.n_kv_heads = n_kv_heads;
  a.lens = lens_dev;
  a.row_start = row_start_dev;
  a.block_table = block_table_dev;
  a.bt_stride = bt_stride;
  a.n_pages = n_pages;
  a.rope = (const float2*)rope_dev;
  a.max_pos = max_pos;
  a.q_out = q_out;
  a.k_pages = k_pages;
  a.v_pages = v_pages;
  a.k_scales = k_scales;
  a.v_scales = v_scales;
  a.k_means = (uint16_t*)k_means;
  if (append_threads(a) > kMaxLaunch)
    return fail(PDEC_INVALID_ARG, "too many rows for one call");
  HIP_OR_FAIL(launch_kv_append(src_dtype, kv_dtype, head_dim, a, (hipStream_t)stream));
  return PDEC_OK;
}

int64_t paged_token_attention_workspace_bytes(int32_t batch, int32_t n_q, int32_t n_q_heads,
                                              int32_t n_kv_heads, int32_t head_dim,
                                              int32_t max_pages) {
  const int rc = check_token_attention(batch, n_q, n_q_heads, n_kv_heads, head_dim);
  if (rc != PDEC_OK) return rc;
  if (max_pages < 1 || max_pages > kMaxStride) return fail(PDEC_INVALID_ARG, "bad max_pages");
  const PagedAttnPlan p = plan_paged_attention(batch, n_q, n_q_heads, n_kv_heads, max_pages);
  TokenAttnLayout l = layout_of(p, n_kv_heads, head_dim);
  // Where many units have a group each and no partials, fewer of the same would have some:
  // the bytes serve every smaller batch too.
  if (p.unit_groups && p.units_for_groups > 1)
    l = layout_of(std::min<int64_t>(p.n_units, p.units_for_groups - 1), p, n_kv_heads, head_dim);
  return l.ml + l.acc;
}

int paged_token_attention(int32_t kv_dtype, int32_t batch, int32_t n_q, int32_t n_q_heads,
                          int32_t n_kv_heads, int32_t head_dim, const void* q,
                          const void* k_pages, const void* v_pages, const float* k_scales,
                          const float* v_scales, int64_t n_pages, const int32_t* block_table_dev,
                          int32_t bt_stride, const int32_t* lens_dev, const int32_t* selected_dev,
                          int32_t n_selected, void* out, void* workspace, int64_t workspace_bytes,
                          void* stream) {
  if (kv_dtype != PDEC_BF16 && kv_dtype != PDEC_FP8_E4M3)
    return fail(PDEC_INVALID_ARG, "kv_dtype must be PDEC_BF16 or PDEC_FP8_E4M3");
  if (!q || !k_pages || !v_pages || !block_table_dev || !lens_dev || !out)
    return fail(PDEC_INVALID_ARG, "null argument");
  int rc = check_token_attention(batch, n_q, n_q_heads, n_kv_heads, head_dim);
  if (rc == PDEC_OK) rc = check_table(batch, bt_stride, n_pages);
  if (rc != PDEC_OK) return rc;
  const bool fp8 = kv_dtype == PDEC_FP8_E4M3;
  if (fp8 != (k_scales != nullptr) || fp8 != (v_scales != nullptr))
    return fail(PDEC_INVALID_ARG, "E4M3 pages take scales, the others none");
  if (selected_dev && (n_q != 1 || n_selected < 1 || n_selected > kMaxStride))
    return fail(PDEC_INVALID_ARG, "selected pages take one query token and n_selected >= 1");
  if (!aligned(q, 16) || !aligned(k_pages, 16) || !aligned(v_pages, 16) || !aligned(out, 16) ||
      !aligned(workspace, 16))
    return fail(PDEC_INVALID_ARG, "q, pages, out and workspace must be 16-byte aligned");
  const PagedAttnPlan p =
      plan_paged_attention(batch, n_q, n_q_heads, n_kv_heads,
                           selected_dev ? std::min(n_selected, bt_stride) : bt_stride);
  if (p.n_units * ((int64_t)bt_stride + 1) > INT32_MAX)
    return fail(PDEC_INVALID_ARG, "batch x bt_stride too large for one call");
  const TokenAttnLayout l = layout_of(p, n_kv_heads, head_dim);
  if (workspace_bytes < l.ml + l.acc || (l.ml > 0 && !workspace))
    return fail(PDEC_INVALID_ARG, "workspace too small: need " + std::to_string(l.ml + l.acc));
  PagedAttnArgs a{};
  a.q = q;
  a.k_pages = k_pages;
  a.v_pages = v_pages;
  a.k_scales = k_scales;
  a.v_scales = v_scales;
  a.block_table = block_table_dev;
  a.lens = lens_dev;
  a.selected = selected_dev;
  a.bt_stride = bt_stride;
  a.n_selected = selected_dev ? n_selected : 0;
  a.max_len = bt_stride * PDEC_PAGE_TOKENS;
  a.n_q = n_q;
  a.n_q_heads = n_q_heads;
  a.n_kv_heads = n_kv_heads;
  a.n_pages = n_pages;
  a.tok_per_block = p.tok_per_block;
  a.blocks_per_seq = p.blocks_per_seq;
  a.n_units = (int32_t)p.n_units;
  a.n_groups = p.n_groups;
  // A pair for each wave.  us at 1, 2, 4, 8: 2 x 2200 tokens of E4M3 pages 14.5, 14.3, 14.4,
  // 15.8, five tokens over 2 x 2500 15.7, 15.8, 15.6, 16.2; 1 x 2200, and 4 sequences and more,
  // within the spread of each other.
  a.min_pairs = 4;
  a.unit_groups = p.unit_groups;
  a.scale_log2 = 1.4426950408889634f / std::sqrt((float)head_dim);
  a.part_ml = (float*)workspace;
  a.part_acc = (float*)((char*)workspace + l.ml);
  a.out = out;
  HIP_OR_FAIL(launch_paged_attention(fp8, head_dim, p.row_tiles, a, (hipStream_t)stream));
  return PDEC_OK;
}

int64_t paged_select_workspace_bytes(int32_t batch, int32_t n_kv_heads, int32_t bt_stride) {
  if (batch < 1 || batch > kMaxBatch || n_kv_heads < 1 || n_kv_heads > 65535 || bt_stride < 1 ||
      bt_stride > kMaxStride)
    return fail(PDEC_INVALID_ARG, "bad sizes");
  return align_up((int64_t)batch * n_kv_heads * bt_stride * 4);
}

int paged_select(int32_t batch, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim,
                 const void* q, const void* k_means, int64_t n_pages,
                 const int32_t* block_table_dev, int32_t bt_stride, const int32_t* lens_dev,
                 int32_t n_selected, int32_t keep_first, int32_t keep_last, int32_t* selected_dev,
                 void* workspace, int64_t workspace_bytes, void* stream) {
  if (!q || !k_means || !block_table_dev || !lens_dev || !selected_dev || !workspace)
    return fail(PDEC_INVALID_ARG, "null argument");
  int rc = check_heads(n_q_heads, n_kv_heads, head_dim);
  if (rc == PDEC_OK) rc = check_table(batch, bt_stride, n_pages);
  if (rc != PDEC_OK) return rc;
  if ((int64_t)batch * (bt_stride / 16 + 1) > INT32_MAX)
    return fail(PDEC_INVALID_ARG, "batch too large for one call");
  if (n_selected < 1 || n_selected > kMaxStride || keep_first < 0 || keep_last < 1 ||
      (int64_t)keep_first + keep_last > n_selected)
    return fail(PDEC_INVALID_ARG,
                "keep_first >= 0, keep_last >= 1 and their sum at most n_selected");
  if (!aligned(q, 16) || !aligned(k_means, 16) || !aligned(workspace, 16))
    return fail(PDEC_INVALID_ARG, "q, k_means and workspace must be 16-byte aligned");
  const int64_t need = paged_select_workspace_bytes(batch, n_kv_heads, bt_stride);
  if (workspace_bytes < need)
    return fail(PDEC_INVALID_ARG, "workspace too small: need " + std::to_string(need));
  SelectArgs a{};
  a.q = (const uint16_t*)q;
  a.k_means = (const uint16_t*)k_means;
  a.block_table = block_table_dev;
  a.lens = lens_dev;
  a.batch = batch;
  a.n_q_heads = n_q_heads;
  a.n_kv_heads = n_kv_heads;
  a.bt_stride = bt_stride;
  a.n_selected = n_selected;
  a.keep_first = keep_first;
  a.keep_last = keep_last;
  a.n_pages = n_pages;
  a.scores = (float*)workspace;
  a.selected = selected_dev;
  if (select_threads(a) > kMaxLaunch)
    return fail(PDEC_INVALID_ARG, "batch too large for one call");
  HIP_OR_FAIL(launch_paged_select(head_dim, a, (hipStream_t)stream));
  return PDEC_OK;
}

int64_t verify_drafts_workspace_bytes(int32_t batch, int32_t n_drafts, int32_t vocab,
                                      int32_t with_drafter) {
  if (batch < 1 || n_drafts < 1 || n_drafts > 1024 || vocab < 1 || vocab > (1 << 22) ||
      (int64_t)batch * (2 * n_drafts + 1) > (1 << 24) ||
      (int64_t)batch * (2 * n_drafts + 1) * (vocab / 2048 + 1) > INT32_MAX)
    return fail(PDEC_INVALID_ARG, "bad sizes");
  return align_up(verify_workspace_bytes(batch, n_drafts, with_drafter != 0, vocab));
}

int verify_drafts(int32_t batch, int32_t n_drafts, int32_t vocab, const float* target_logits_dev,
                  const float* draft_logits_dev, const int32_t* draft_tokens_dev,
                  const float* uniforms_dev, float temperature, int32_t* tokens_dev_out,
                  int32_t* accepted_dev_out, void* workspace, int64_t workspace_bytes,
                  void* stream) {
  if (!target_logits_dev || !draft_tokens_dev || !uniforms_dev || !tokens_dev_out ||
      !accepted_dev_out || !workspace)
    return fail(PDEC_INVALID_ARG, "null argument");
  if (!(temperature > 0.f) || !std::isfinite(temperature))
    return fail(PDEC_INVALID_ARG, "temperature must be positive and finite");
  const int64_t need =
      verify_drafts_workspace_bytes(batch, n_drafts, vocab, draft_logits_dev != nullptr);
  if (need < 0) return (int)need;
  if (workspace_bytes < need)
    return fail(PDEC_INVALID_ARG, "workspace too small: need " + std::to_string(need));
  if (!aligned(workspace, 16) || !aligned(target_logits_dev, 4) || !aligned(draft_logits_dev, 4))
    return fail(PDEC_INVALID_ARG, "workspace must be 16-byte aligned, logits 4-byte");
  VerifyArgs a{};
  a.target = target_logits_dev;
  a.drafter = draft_logits_dev;
  a.drafts = draft_tokens_dev;
  a.uniforms = uniforms_dev;
  a.tokens = tokens_dev_out;
  a.accepted = accepted_dev_out;
  a.batch = batch;
  a.n_drafts = n_drafts;
  a.vocab = vocab;
  a.inv_t = 1.0 / (double)temperature;
  a.temperature = temperature;
  a.workspace = workspace;
  HIP_OR_FAIL(launch_verify(a, (hipStream_t)stream));
  return PDEC_OK;
}

}  // extern "C"
