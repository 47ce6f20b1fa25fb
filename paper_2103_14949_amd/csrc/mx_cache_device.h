// Device-side helpers of the operators around a paged cache: whose a row is, and where its token lies.
#pragma once

#include "mx_cache.h"
#include "mx_device.h"

namespace hago {

// Page of the table that a position lies in.
__device__ __forceinline__ uint32_t cache_page_of(const CacheArgs& c, uint32_t position) {
  return (uint32_t)((uint64_t)position * c.page_factor >> (31 + c.page_shift));
}

// Row of [pages, kv_heads, page] at which a position of a sequence is for a head; -1: it has no place.
__device__ __forceinline__ int64_t cache_place(const CacheArgs& c, int seq, int64_t position, int head) {
  if (position < 0 || position >= c.places) return -1;
  const uint32_t entry = cache_page_of(c, (uint32_t)position);
  const int32_t page = c.table[seq * c.table_stride + entry];
  if ((uint32_t)page >= (uint32_t)c.pages) return -1;
  return ((int64_t)page * c.kv_heads + head) * c.page + (int32_t)((uint32_t)position - entry * (uint32_t)c.page);
}

// The sequence of row t and the position of its token; false: t is in none.  A step of single tokens has row s in sequence s, which
// costs one look; the others halve.
__device__ __forceinline__ bool cache_row(const CacheArgs& c, int64_t t, int& seq, int64_t& position) {
  int low = 0, high = c.seqs;  // offsets[low] <= t < offsets[high], if so at all
  if (t < c.seqs) {
    if (c.offsets[t] <= t && t < c.offsets[t + 1]) low = (int)t, high = (int)t + 1;
  }
  while (high - low > 1) {
    const int mid = low + (high - low) / 2;
    if (c.offsets[mid] <= t) low = mid;
    else high = mid;
  }
  const int32_t first = c.offsets[low], end = c.offsets[low + 1];
  if (t < first || t >= end) return false;
  seq = low;
  position = (int64_t)c.lengths[low] - (end - t);
  return true;
}

}  // namespace hago
