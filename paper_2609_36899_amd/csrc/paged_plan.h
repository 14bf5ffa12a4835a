// Which form of a kernel a call takes, by its sizes: the attention of query tokens over
// caller-owned pages, and draft verification.  Host code alone, so that the rules can be
// asked without a GPU.
#pragma once

#include <stdint.h>

#include <algorithm>

namespace pdec {

// ---- attention of query tokens -----------------------------------------------
// Work groups of a launch: one for each compute unit.  More of them cost their beginnings
// (lengths, queries, first pages) and their partials: us at 256 / 512 groups, 64 sequences
// of 1K to 8K tokens 120 / 119 (E4M3, 648 MB: 5.4 TB/s) and 180 / 179 (bf16, 1136 MB: 6.3),
// five tokens each over 8 x 64K to 128K 267 / 283 (E4M3, 1580 MB: 5.9), four over 16 x 1K to
// 16K 94 / 96 (bf16, 512 MB: 5.4); 1024 groups are slower by 5 to 20% more.  Blocks of more
// than 32 rows, whose waves go in step, gain from a second group on a unit: 13 tokens over 16 x
// 4K to 16K 124 / 92 (E4M3), 126 / 118 (bf16), 26 tokens 177 / 140 and 168 / 152; 768 are as
// slow as 256.
constexpr int kAttnGroups = 256;

struct PagedAttnPlan {
  int32_t row_tiles, tok_per_block, blocks_per_seq, n_groups;
  int64_t n_units;
  bool unit_groups;  // a work group for each unit and no merge, instead of equal stretches
  int32_t units_for_groups;  // the fewest units at which tables of max_pages give that
};
// max_pages: what no sequence can read more of.
inline PagedAttnPlan plan_paged_attention(int batch, int n_q, int n_q_heads, int n_kv_heads,
                                          int max_pages) {
  PagedAttnPlan p;
  const int G = n_q_heads / n_kv_heads;
  // The smallest block that holds a sequence's rows of a KV head, or blocks of 128.
  const int64_t rows = (int64_t)n_q * G;
  p.row_tiles = rows <= 16 ? 1 : rows <= 32 ? 2 : rows <= 64 ? 4 : 8;
  p.tok_per_block = 16 * p.row_tiles / G;
  p.blocks_per_seq = (n_q + p.tok_per_block - 1) / p.tok_per_block;
  p.n_units = (int64_t)batch * p.blocks_per_seq;
  p.n_groups = std::max(1, (p.row_tiles > 2 ? 512 : kAttnGroups) / n_kv_heads);
  // A work group for each unit needs no scan of the lengths and no merge, and waits for the
  // longest.  us, equal stretches / a group a unit, one token, 8 KV heads of four: table of
  // 512 tokens, 8 sequences 15.0 / 11.8 (E4M3), 14.0 / 11.4 (bf16), 64 26.1 / 16.2, 256
  // 74.9 / 53.4; 1024 tokens, 8 sequences 15.4 / 12.9 and 15.7 / 17.9 (bf16), 64 32.8 /
  // 24.9; 2048 tokens, 1 sequence 15.1 / 15.3 and 13.8 / 20.8, 64 47.9 / 42.7 and 70.6 /
  // 71.4, 256 166.9 / 151.8.
  const int pairs = (max_pages + 1) / 2;
  p.units_for_groups =
      pairs <= 24 ? 1 : pairs <= 66 ? (512 + n_kv_heads - 1) / n_kv_heads : INT32_MAX;
  p.unit_groups = p.n_units <= 65535 && p.n_units >= p.units_for_groups;
  return p;
}

// Row tiles a wave, and waves side by side along the rows (of the work group's four).
struct PagedAttnForm {
  int32_t tiles, waves;
};
inline PagedAttnForm paged_attention_form(int kv_fp8, int head_dim, int row_tiles, int64_t n_units,
                                          int max_len, int n_kv_heads) {
  if (row_tiles == 1) return {1, 1};
  if (row_tiles == 8) return {2, 4};
  if (row_tiles == 4) return kv_fp8 ? PagedAttnForm{2, 2} : PagedAttnForm{1, 4};
  // 17 to 32 rows as a tile for each of two waves that load the same pages, or as two tiles of
  // one wave: half the work at a stretch's two ends, or half the loads between them.  By what a
  // work group reads if the table is full; us, tile a wave / two tiles, at KB a group: E4M3, 5 x
  // 4 rows over 4 x 4K 17.7 / 22.7 (120), over 128 x 0.5K 31.5 / 51.1 (512), over 58 x 1.4K 56.6
  // / 57.0 (640), 8 x 3 over 41 x 0 to 4K 34.7 / 39.9 (700), 5 x 4 61.0 / 60.0 (1400), over 16 x
  // 16K 73.5 / 63.8 (2048); bf16, 5 x 4 over 4 x 4K 19.1 / 22.3 (240), 8 x 3 over 58 x 1.4K
  // 49.2 / 42.0 (640).
  const int64_t group_bytes =
      n_units * max_len * n_kv_heads / kAttnGroups * head_dim * (kv_fp8 ? 2 : 4);
  return group_bytes <= (kv_fp8 ? 1024 : 256) * 1024 ? PagedAttnForm{1, 2} : PagedAttnForm{2, 1};
}

// ---- draft verification --------------------------------------------------------
// Logits of a call, and tokens of its deciding rows, from which rows are cut coarser.
constexpr int64_t kFineLogits = 1 << 23, kFineCuts = 3 << 20;

struct VerifySizes {
  int chunk, n_chunks;  // tokens of a chunk (a multiple of 1024), chunks of a row
  int cut, n_cuts;      // the same of a deciding row
  int rows;             // target rows, then drafter rows
};
inline VerifySizes verify_sizes(int batch, int n_drafts, bool drafter, int vocab) {
  VerifySizes s;
  s.rows = batch * (n_drafts + 1 + (drafter ? n_drafts : 0));
  // 32 values a thread; few rows are cut finer, so that they meet more work groups.
  s.chunk = (int64_t)s.rows * vocab >= kFineLogits ? 8192 : 2048;
  s.n_chunks = (vocab + s.chunk - 1) / s.chunk;
  // Two passes over one or two rows a sequence, long arithmetic each: cut finer where few
  // cuts of 8192 would leave compute units with one or two groups.  us at cuts of 8192 / 2048,
  // drafter's logits beside the target's: 8 x 128256 33 / 29, 18 x 128256 36 / 33, 50 x 32003
  // 32 / 30, 34 x 128256 70 / 73, 64 x 128256 106 / 123.
  s.cut = (int64_t)batch * vocab >= kFineCuts ? 8192 : 2048;
  s.n_cuts = (vocab + s.cut - 1) / s.cut;
  return s;
}

}  // namespace pdec
