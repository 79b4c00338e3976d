// Device-side view of jn_kv_cache and jn_kv_batch: every index that a kernel forms from
// the caller's device arrays is bounded here.
#pragma once

#include "jn_device.h"
#include "jn_internal.h"

namespace jnx {

// The caller's tables are not written while a kernel reads them, so that what a whole
// wavefront reads of them alike comes by the scalar cache.
typedef const __attribute__((address_space(4))) int32_t* KvTable;
__device__ __forceinline__ KvTable kv_table(const int32_t* p) { return (KvTable)(uintptr_t)p; }

struct KvSeq {
  int32_t past, row0, n;  // cached rows, first new row of the call, new rows
};
__device__ __forceinline__ KvSeq kv_seq(const KvBatch& b, int32_t s) {
  const KvTable cu = kv_table(b.cu) + s;
  const int32_t row0 = min(max(cu[0], 0), b.rows), end = min(cu[1], b.rows);
  return KvSeq{min(max(kv_table(b.past)[s], 0), b.places), row0, min(max(end - row0, 0), b.max_new)};
}

// Sequence of a call's row by all lanes of a wavefront (n_seqs: the row is in none):
// how many sequences end at or before the row, 64 of the ascending ends at a time.
__device__ __forceinline__ int32_t kv_find(const KvBatch& b, int32_t row, int lane) {
  int32_t lo = 0, len = b.n_seqs;
  while (len > 0) {
    const int32_t stride = (len + 63) >> 6, k = (lane + 1) * stride;
    const bool before = k <= len && b.cu[lo + k] <= row;
    const int32_t c = __builtin_popcountll(__ballot(before)) * stride;
    lo += c;
    len = min(len - c, stride - 1);
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

// Page of place t of a sequence with page table `pages`, -1 where there is none.
__device__ __forceinline__ int32_t kv_page(const KvBatch& b, const KvCache& c, const int32_t* pages, int32_t t) {
  if (t < 0 || t >= b.places) return -1;
  const int32_t g = pages[t >> c.page_log2];
  return (uint32_t)g < (uint32_t)c.n_pages ? g : -1;
}
// Element offset of head h's row for place t in page g.
__device__ __forceinline__ int64_t kv_at(const KvCache& c, int32_t g, int32_t h, int32_t t) {
  return g * c.ld_page + (((int64_t)h << c.page_log2) + (t & ((1 << c.page_log2) - 1))) * c.hd;
}

// Parent of row j of a sequence, -1 where that is not an earlier row.
__device__ __forceinline__ int32_t kv_parent(const int32_t* parents, int32_t j) {
  const int32_t p = parents[j];
  return p >= 0 && p < j ? p : -1;
}

}  // namespace jnx
