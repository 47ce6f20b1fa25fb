// Host-side launch entry points of the microscaled operators; called only from their part of the C ABI (mx_api.hip) after all
// arguments have been validated.
#pragma once

#include "launch.h"

namespace hago {

enum MxFormat : int { kMxFp4 = 0, kMxFp8 = 1 };        // E2M1 and E4M3 in blocks of 32, scales E8M0
enum MxType : int { kMxF32 = 0, kMxBf16 = 1, kMxF16 = 2 };

// Rows are held in whole blocks of 128 columns.
constexpr int64_t mx_padded(int64_t cols) { return (cols + 127) / 128 * 128; }
constexpr int64_t mx_code_bytes(int64_t cols, int format) { return mx_padded(cols) >> (format == kMxFp4 ? 1 : 0); }
constexpr int64_t mx_scale_bytes(int64_t cols) { return mx_padded(cols) / 32; }

// What the row operators write: codes and scales, and the values they stand for unless values is NULL.
struct MxOut {
  uint8_t* codes;
  uint8_t* scales;
  void* values;
  // the same from a later row on; T: the type of values
  template <typename T>
  MxOut from(int64_t row, int64_t cols, int format) const {
    return {codes + row * mx_code_bytes(cols, format), scales + row * mx_scale_bytes(cols), values ? static_cast<T*>(values) + row * cols : nullptr};
  }
};

hipError_t launch_mx_quantize(const void* x, int type, int64_t rows, int64_t cols, int64_t stride, int format, const MxOut& out, hipStream_t st);
hipError_t launch_mx_silu_mul(const void* x, int type, int64_t rows, int64_t cols, int64_t stride, int format, const MxOut& out, hipStream_t st);
hipError_t launch_mx_rmsnorm(const void* x, const void* residual, const void* gamma, int type, int64_t rows, int64_t cols, int64_t stride,
                             float eps, int format, void* residual_out, const MxOut& out, hipStream_t st);

// out[t, n] = bias[n] + sum_k a[row(t), k] w[n, k].  Grouped: T rows of `experts` groups, group e has the rows offsets[e] .. offsets[e + 1]
// and the weights w[e], bias[e]; row(t) = index[t] or t.
struct MxGemmArgs {
  const uint8_t* a;
  const uint8_t* a_scale;
  const uint8_t* w;
  const uint8_t* w_scale;
  const float* bias;       // or NULL
  void* out;
  const int32_t* offsets;  // NULL: one group of all rows
  const int32_t* index;    // or NULL
  int32_t T, N, K, a_rows, experts;
  int32_t type;            // of out
  uint32_t place;          // of the launch: its first tile, or how many workgroups there are where they stay for several tiles
};
// Most tiles of `rows` rows that the groups' rows can make: each has at least one row, each group at most one that is not full.
constexpr int64_t mx_most_tiles(int64_t T, int64_t experts, int64_t rows) {
  const int64_t most = T / rows + experts;
  return most < T ? most : T;
}
hipError_t launch_mx_gemm(const MxGemmArgs& g, int a_format, hipStream_t st);

}  // namespace hago
