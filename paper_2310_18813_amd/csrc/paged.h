// What the operators over a paged cache share: the checks of its description and the device-side reading of a batch.
#pragma once
#include "spec_internal.h"
#include "device_utils.h"

namespace spec {

// spec_paged_cache and spec_paged_batch as the kernels take them
struct PagedArgs {
  unsigned char *k, *v;
  uint32_t page_units, pos_units, head_units;  // strides in units of 16 bytes
  int n_pages, page_shift, n_kv_heads;
  int B, rows, max_rows, max_len;
  const int32_t *row_start, *len, *pages;
  int64_t pages_stride;
};

// A sequence's share of a pass: rows row0 .. row0 + n - 1, row i at position kv - n + i.
struct PagedSeq { int row0, n, kv; };
__device__ __forceinline__ PagedSeq paged_seq(const PagedArgs &a, int b) {
  PagedSeq s;
  if (a.row_start) {  // whatever the device says, rows stay inside the tensors
    s.row0 = min(max(a.row_start[b], 0), a.rows);
    s.n = min(max(a.row_start[b + 1], s.row0), a.rows) - s.row0;
  } else {
    s.n = a.rows / a.B;
    s.row0 = b * s.n;
  }
  s.n = min(s.n, a.max_rows);
  s.kv = min(max(a.len[b], 0), a.max_len);
  return s;
}

// The page of position `pos` (0 <= pos < max_len) of sequence b, -1 if it is absent.
__device__ __forceinline__ int paged_page(const PagedArgs &a, int b, int pos) {
  const int page = a.pages[b * a.pages_stride + (pos >> a.page_shift)];
  return (unsigned)page < (unsigned)a.n_pages ? page : -1;
}

// Byte offset of a position's row of a head: two 32 x 32 + 64 bit products, whatever the sizes of the strides.
__device__ __forceinline__ size_t paged_row(const PagedArgs &a, int page, int pos) {
  return ((uint64_t)(uint32_t)page * a.page_units + (uint64_t)(uint32_t)(pos & ((1 << a.page_shift) - 1)) * a.pos_units) << 4;
}

// Host: checks what both entry points share and fills `out`.  No device call.
int paged_args(const char *who, const spec_paged_cache *cache, const spec_paged_batch *batch, PagedArgs *out);
// a row-wise tensor: `heads` dense heads a row
int paged_rows_check(const char *who, const char *what, const spec_paged_cache *cache, int heads, const void *p, int64_t stride);

}  // namespace spec
