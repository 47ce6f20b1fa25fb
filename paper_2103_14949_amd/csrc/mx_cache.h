// Host-side launch entry points of the operators around a paged cache of keys and values, and of the rotary positions; called only
// from their part of the C ABI (mx_cache_api.hip) after all arguments have been validated.
#pragma once

#include "mx.h"

namespace hago {

constexpr int kCacheMostDim = 256, kRopeMostDim = 4096;
constexpr int64_t kMostRows = 1ll << 27, kMostUnits = 1ll << 22;  // of the attention: T * heads, seqs * kv_heads

// A row of the cache: whole blocks of 32 columns.
constexpr int64_t cache_blocks(int64_t dim) { return (dim + 31) / 32; }
constexpr int64_t cache_row_bytes(int64_t dim, int format) { return cache_blocks(dim) * (format == kMxFp4 ? 16 : 32); }

// The cache, and the tokens that a call is about.
struct CacheArgs {
  uint8_t* k_codes;
  uint8_t* k_scales;
  uint8_t* v_codes;
  uint8_t* v_scales;
  const int32_t* table;
  const int32_t* lengths;
  const int32_t* offsets;
  int64_t table_stride;
  int32_t pages, page, kv_heads, dim, seqs;
  int32_t places;  // positions below it have an entry of the table
  // position / page = position * page_factor >> (31 + page_shift), position < 2^31
  uint32_t page_factor;
  int32_t page_shift;
  int32_t k_format, v_format;
};

// A type's tensor [T, heads, dim] with rows and heads at any distance.
struct HeadsTensor {
  const void* data;
  int64_t row, head;
};

hipError_t launch_mx_cache_write(const CacheArgs& c, const HeadsTensor& k, const HeadsTensor& v, int type, int64_t T, void* k_values, void* v_values, hipStream_t st);
hipError_t launch_mx_cache_read(const CacheArgs& c, int type, int64_t T, void* k, void* v, hipStream_t st);

struct AttentionArgs {
  HeadsTensor q;
  void* out;      // [T, heads, dim]
  float* lse;     // [T, heads] or NULL
  float scale;
  int32_t T, heads, causal, window;  // window 0: none
  int32_t type;
};
int64_t mx_attention_workspace_bytes(int64_t T, int64_t seqs, int64_t heads, int64_t kv_heads, int64_t dim);
hipError_t launch_mx_attention(const CacheArgs& c, const AttentionArgs& a, void* workspace, hipStream_t st);

struct RopeArgs {
  HeadsTensor x;
  void* out;
  int64_t out_row, out_head;
  const int32_t* positions;    // [axes, T]
  const float* frequencies;    // [pairs]
  const int32_t* axis;         // [pairs] or NULL: 0
  int32_t T, heads, dim, pairs, axes, interleaved;
};
hipError_t launch_rope(const RopeArgs& r, int type, hipStream_t st);

}  // namespace hago
