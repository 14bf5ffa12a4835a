// Argument checks that the operators over caller-owned pages share.
#pragma once

#include <stdint.h>

#include "../../include/pdec.h"
#include "status.h"

namespace pdec {

constexpr int64_t kMaxStride = 1 << 22;  // pages of a table row: 2^26 positions
constexpr int64_t kMaxBatch = 1 << 20;

inline int64_t align_up(int64_t v) { return (v + 255) / 256 * 256; }
inline bool aligned(const void* p, int bytes) { return (uintptr_t)p % bytes == 0; }

inline int check_table(int32_t batch, int32_t bt_stride, int64_t n_pages) {
  if (batch < 1 || batch > kMaxBatch || bt_stride < 1 || bt_stride > kMaxStride || n_pages < 1 ||
      n_pages > INT32_MAX)
    return fail(PDEC_INVALID_ARG, "bad batch, bt_stride or n_pages");
  return PDEC_OK;
}

}  // namespace pdec
