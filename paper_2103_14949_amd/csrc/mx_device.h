// Device-side helpers of the microscaled operators: elements of the three real types as binary32, and the code of a block.
#pragma once

#include "hago_device.h"
#include "mx.h"

namespace hago {

typedef uint32_t mx_u4 __attribute__((ext_vector_type(4)));
typedef float mx_f2 __attribute__((ext_vector_type(2)));
typedef mx_u4 mx_u4_any __attribute__((aligned(1)));

template <int TYPE>
struct MxElement;
template <>
struct MxElement<kMxF32> {
  using type = float;
};
template <>
struct MxElement<kMxBf16> {
  using type = __bf16;
};
template <>
struct MxElement<kMxF16> {
  using type = _Float16;
};

// Eight consecutive elements at any address of their type's alignment; n of them are inside the row, zeros stand for the others.
// (16 bytes off four cost four passes of the memory pipe instead of one; eight loads of an element each cost eight.)
template <int TYPE>
__device__ __forceinline__ void mx_load8(const typename MxElement<TYPE>::type* p, int n, float (&v)[8]) {
  using T = typename MxElement<TYPE>::type;
  constexpr int kVecs = 8 * sizeof(T) / 16;
  if (n >= 8) {
    union {
      mx_u4 u[kVecs];
      T t[8];
    } b;
#pragma unroll
    for (int i = 0; i < kVecs; ++i) b.u[i] = reinterpret_cast<const mx_u4_any*>(p)[i];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)b.t[i];
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < n ? (float)p[i] : 0.0f;
  }
}

// With the nontemporal hint: values and residuals are read much later than the codes beside them, if at all.  8192 x 4096 bf16 with
// values, us without the hint and with it: the norm 55.5 and 50.6, the quantization to 4 bits 28.3 and 25.1.
template <int TYPE>
__device__ __forceinline__ void mx_store8(typename MxElement<TYPE>::type* p, int n, const float (&v)[8]) {
  using T = typename MxElement<TYPE>::type;
  constexpr int kVecs = 8 * sizeof(T) / 16;
  if (n >= 8) {
    union {
      mx_u4 u[kVecs];
      T t[8];
    } b;
#pragma unroll
    for (int i = 0; i < 8; ++i) b.t[i] = (T)v[i];
#pragma unroll
    for (int i = 0; i < kVecs; ++i) __builtin_nontemporal_store(b.u[i], reinterpret_cast<mx_u4_any*>(p) + i);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) p[i] = (T)v[i];
  }
}

// Largest of a quad of lanes, in all four.
__device__ __forceinline__ uint32_t mx_quad_max(uint32_t m) {
  const uint32_t a = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0xB1, 0xf, 0xf, true);  // quad_perm 1,0,3,2
  m = m > a ? m : a;
  const uint32_t b = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x4E, 0xf, 0xf, true);  // quad_perm 2,3,0,1
  return m > b ? m : b;
}

// Codes of eight elements of a block whose other 24 the other lanes of the quad hold, and the block's scale; v becomes the values
// they stand for.  With m the largest magnitude, the scale is 2^(floor(log2 m) - emax), at least 2^-127, i.e. the exponent field
// of m less emax; dividing by it is exact, rounding to the code (nearest, ties to even) is the only rounding there is.  Magnitudes
// beyond the largest code take it: the scale's rule leaves them up to a quarter above.  A block that holds an infinity or NaN has the scale NaN and
// zero codes.
template <int FORMAT>
__device__ __forceinline__ uint32_t mx_encode8(float (&v)[8], uint32_t (&codes)[2]) {
  constexpr int kEmax = FORMAT == kMxFp4 ? 2 : 8;
  constexpr float kTop = FORMAT == kMxFp4 ? 6.0f : 448.0f;
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t b = __builtin_bit_cast(uint32_t, v[i]) & 0x7fffffffu;
    m = m > b ? m : b;
  }
  m = mx_quad_max(m);
  const bool finite = m < 0x7f800000u;
  const int e = (int)(m >> 23) - kEmax;
  const uint32_t byte = e > 0 ? (uint32_t)e : 0;
  const float inv = __builtin_bit_cast(float, (254 - byte) << 23);  // 2^(127 - byte), byte <= 253
  const float scale = __builtin_bit_cast(float, byte ? byte << 23 : 0x00400000u);
  float s[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) s[i] = __builtin_amdgcn_fmed3f(v[i] * inv, -kTop, kTop);
  codes[0] = codes[1] = 0;
  mx_f2 d[4];
  if constexpr (FORMAT == kMxFp4) {
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, s[0], s[1], 1.0f, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, s[2], s[3], 1.0f, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, s[4], s[5], 1.0f, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, s[6], s[7], 1.0f, 3);
    d[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 0);
    d[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 1);
    d[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 2);
    d[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 3);
    codes[0] = finite ? c : 0;
  } else {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      int c = 0;
      c = __builtin_amdgcn_cvt_pk_fp8_f32(s[4 * i], s[4 * i + 1], c, false);
      c = __builtin_amdgcn_cvt_pk_fp8_f32(s[4 * i + 2], s[4 * i + 3], c, true);
      d[2 * i] = __builtin_amdgcn_cvt_pk_f32_fp8(c, false);
      d[2 * i + 1] = __builtin_amdgcn_cvt_pk_f32_fp8(c, true);
      codes[i] = finite ? (uint32_t)c : 0;
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = finite ? d[i / 2][i % 2] * scale : __builtin_bit_cast(float, 0x7fc00000u);
  return finite ? byte : 255u;
}

// Writes what mx_encode8 gave for columns [col, col + 8) of a row: `row` counts from the tensors' starts.
template <int TYPE, int FORMAT>
__device__ __forceinline__ void mx_put8(const MxOut& out, int64_t row, int cols, int padded, int col, float (&v)[8]) {
  uint32_t codes[2];
  const uint32_t byte = mx_encode8<FORMAT>(v, codes);
  if constexpr (FORMAT == kMxFp4)
    *reinterpret_cast<uint32_t*>(out.codes + row * (padded / 2) + col / 2) = codes[0];
  else
    *reinterpret_cast<uint2*>(out.codes + row * padded + col) = make_uint2(codes[0], codes[1]);
  if ((col & 31) == 0) out.scales[row * (padded / 32) + col / 32] = (uint8_t)byte;
  if (out.values && col < cols)
    mx_store8<TYPE>(static_cast<typename MxElement<TYPE>::type*>(out.values) + row * cols + col, cols - col, v);
}

}  // namespace hago
