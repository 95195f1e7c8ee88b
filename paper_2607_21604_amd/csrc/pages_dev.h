// Device helpers of the kernels over 4-bit pages.
#pragma once
#include "kernels.h"

namespace akvs {

// Rows of request b: [r0, r1), at most rows_max. Values of row_start are clamped into the buffers.
__device__ __forceinline__ void paged_rows(const PagedBatch &s, int b, int &r0, int &r1) {
  if (s.row_start) {
    r0 = min(max(s.row_start[b], 0), s.n_rows);
    r1 = min(max(s.row_start[b + 1], r0), min(s.n_rows, r0 + s.rows_max));
  } else {
    r0 = b * s.rows_max;
    r1 = r0 + s.rows_max;
  }
}

// A request's table and keys: none where its sequence is out of range.
__device__ __forceinline__ const int32_t *paged_keys(const PagedBatch &s, int b, int &len) {
  const int q = s.seq ? s.seq[b] : b;
  if (q < 0 || q >= s.n_seq) {
    len = 0;
    return s.table;
  }
  len = min(max(s.len[q], 0), s.limit);
  return s.table + (size_t)q * s.max_pages;
}

}  // namespace akvs
