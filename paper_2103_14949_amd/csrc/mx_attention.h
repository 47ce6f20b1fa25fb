// What the kernels of the attention over a paged cache of microscaled keys and values have in common.
//
// Keys and values go into the matrix instructions as bfloat16, which holds every code times its scale (three bits of mantissa, the
// exponents of binary32; below 2^-126 it may be zero); queries and probabilities as one, two or three bfloat16 numbers that add up to
// theirs: bfloat16 queries are held by one, float16 by two, binary32 by three.  Sums are binary32.
#pragma once

#include "mx_cache_device.h"

namespace hago {

typedef __bf16 at_b2 __attribute__((ext_vector_type(2)));
typedef __bf16 at_b8 __attribute__((ext_vector_type(8)));
typedef short at_s4 __attribute__((ext_vector_type(4)));
typedef float at_f4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) at_s4 at_lds_s4;

template <int TYPE>
constexpr int kAttentionPieces = TYPE == kMxBf16 ? 1 : TYPE == kMxF16 ? 2 : 3;

// One sequence's rows and keys in this call.
struct AttentionSpan {
  int32_t first, rows;    // tokens of the call
  int64_t position;       // of the first one
  int32_t low, high;      // keys that any of them can see
};
__device__ __forceinline__ AttentionSpan attention_span(const CacheArgs& c, const AttentionArgs& a, int seq) {
  AttentionSpan s;
  const int32_t b = c.offsets[seq], e = c.offsets[seq + 1], length = c.lengths[seq];
  s.first = b < 0 ? 0 : b;
  const int32_t end = e > a.T ? a.T : e;
  s.rows = end > s.first ? end - s.first : 0;
  s.position = (int64_t)length - ((int64_t)e - s.first);
  s.high = length < 0 ? 0 : length < c.places ? length : c.places;
  const int64_t low = a.window ? s.position - a.window + 1 : 0;
  s.low = low < 0 ? 0 : low < s.high ? (int32_t)low : s.high;
  return s;
}

// Eight codes of a block as bfloat16: dwords `w` (fp8: two, fp4: one), scale 2^(byte - 127).
template <int FORMAT>
__device__ __forceinline__ at_b8 attention_values8(const uint32_t* w, float scale) {
  at_b2 d[4];
  if constexpr (FORMAT == kMxFp4) {
    d[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[0], scale, 0);
    d[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[0], scale, 1);
    d[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[0], scale, 2);
    d[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[0], scale, 3);
  } else {
    d[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[0], scale, false);
    d[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[0], scale, true);
    d[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[1], scale, false);
    d[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[1], scale, true);
  }
  at_b8 v;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = d[i / 2][i % 2];
  return v;
}

// x as PIECES bfloat16 numbers, the largest first.
template <int PIECES>
__device__ __forceinline__ void attention_split(float x, __bf16 (&p)[PIECES]) {
#pragma unroll
  for (int i = 0; i < PIECES; ++i) {
    p[i] = (__bf16)x;
    if (i + 1 < PIECES) x -= (float)p[i];
  }
}

constexpr float kAttentionLog2e = 1.44269504f, kAttentionLn2 = 0.693147181f;

}  // namespace hago
