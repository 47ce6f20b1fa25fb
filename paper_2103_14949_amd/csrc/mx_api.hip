// C ABI of the microscaled operators: argument validation (host only, before any launch) and dispatch.  See include/hago.h for the
// contract.
#include "../../include/hago.h"

#include <cmath>

#include "mx.h"

namespace {

constexpr int64_t kI32Max = 2147483647ll;

// hago::MxType of a real type, -1: it is none
int real_type(hago_dtype t) { return t == HAGO_F32 ? hago::kMxF32 : t == HAGO_BF16 ? hago::kMxBf16 : t == HAGO_F16 ? hago::kMxF16 : -1; }
bool is_format(hago_mx_format f) { return f == HAGO_MX_FP4 || f == HAGO_MX_FP8; }
hago_status from_hip(hipError_t e) { return e == hipSuccess ? HAGO_OK : HAGO_ERR_DEVICE; }

// What the operators by rows have in common; x has `wide` columns.
hago_status check_rows(const void* x, hago_dtype x_t, int64_t rows, int64_t cols, int64_t wide, int64_t stride, hago_mx_format format, const void* codes,
                       const void* scales, const void* values) {
  if (rows < 0 || cols < 0 || cols > kI32Max - 128 || wide > kI32Max - 128 || stride < wide) return HAGO_ERR_SHAPE;
  if (rows && stride > (1ll << 62) / rows) return HAGO_ERR_SHAPE;
  if (real_type(x_t) < 0) return HAGO_ERR_DTYPE;
  if (!is_format(format)) return HAGO_ERR_PARAM;
  if (rows && cols && (!x || !codes || !scales)) return HAGO_ERR_NULL;
  const size_t size = x_t == HAGO_F32 ? 4 : 2;
  if (!hago::ptr_aligned(x, size) || !hago::ptr_aligned(values, size) || !hago::ptr_aligned(codes, 16) || !hago::ptr_aligned(scales, 4)) return HAGO_ERR_PARAM;
  return HAGO_OK;
}

hago::MxOut out_of(void* codes, void* scales, void* values) { return {static_cast<uint8_t*>(codes), static_cast<uint8_t*>(scales), values}; }

hago_status check_product(const hago::MxGemmArgs& g, int64_t a_rows, int64_t T, int64_t experts, int64_t N, int64_t K, hago_mx_format format, hago_dtype out_t) {
  if (a_rows < 0 || T < 0 || experts < 0 || N < 0 || K < 0 || a_rows > kI32Max || T > kI32Max - 256 || experts > kI32Max - 256 || N > kI32Max - 256 || K > (1 << 22))
    return HAGO_ERR_SHAPE;
  if (real_type(out_t) < 0) return HAGO_ERR_DTYPE;
  if (!is_format(format)) return HAGO_ERR_PARAM;
  if (T == 0 || N == 0 || experts == 0) return HAGO_OK;
  if (a_rows == 0) return HAGO_ERR_SHAPE;
  if (g.index && a_rows * hago::mx_code_bytes(K, format) > kI32Max) return HAGO_ERR_SHAPE;
  // (tiles have 16 rows and 16 columns at least)
  if ((N / 16 + 1) * hago::mx_most_tiles(T, experts, 16) > kI32Max) return HAGO_ERR_SHAPE;
  if (!g.out || (K && (!g.a || !g.a_scale || !g.w || !g.w_scale))) return HAGO_ERR_NULL;
  if (!hago::ptr_aligned(g.a, 16) || !hago::ptr_aligned(g.w, 16) || !hago::ptr_aligned(g.a_scale, 4) || !hago::ptr_aligned(g.w_scale, 4) ||
      !hago::ptr_aligned(g.bias, 4) || !hago::ptr_aligned(g.offsets, 4) || !hago::ptr_aligned(g.index, 4) || !hago::ptr_aligned(g.out, out_t == HAGO_F32 ? 4 : 2))
    return HAGO_ERR_PARAM;
  return HAGO_OK;
}

hago::MxGemmArgs product(const void* a, const void* a_scale, const void* w, const void* w_scale, const float* bias, const int32_t* offsets, const int32_t* index,
                         int64_t a_rows, int64_t T, int64_t experts, int64_t N, int64_t K, hago_dtype out_t, void* out) {
  hago::MxGemmArgs g{};
  g.a = static_cast<const uint8_t*>(a);
  g.a_scale = static_cast<const uint8_t*>(a_scale);
  g.w = static_cast<const uint8_t*>(w);
  g.w_scale = static_cast<const uint8_t*>(w_scale);
  g.bias = bias;
  g.out = out;
  g.offsets = offsets;
  g.index = index;
  g.T = (int32_t)T;
  g.N = (int32_t)N;
  g.K = (int32_t)K;
  g.a_rows = (int32_t)a_rows;
  g.experts = (int32_t)experts;
  g.type = real_type(out_t);
  return g;
}

}  // namespace

extern "C" {

hago_status hago_mx_quantize(const void* x, hago_dtype x_t, int64_t rows, int64_t cols, int64_t row_stride, hago_mx_format format, void* codes, void* scales,
                             void* values, void* stream) {
  const hago_status s = check_rows(x, x_t, rows, cols, cols, row_stride, format, codes, scales, values);
  if (s != HAGO_OK || rows == 0 || cols == 0) return s;
  return from_hip(hago::launch_mx_quantize(x, real_type(x_t), rows, cols, row_stride, format, out_of(codes, scales, values), static_cast<hipStream_t>(stream)));
}

hago_status hago_mx_silu_mul(const void* x, hago_dtype x_t, int64_t rows, int64_t cols, int64_t row_stride, hago_mx_format format, void* codes, void* scales,
                             void* values, void* stream) {
  if (cols < 0 || cols > kI32Max) return HAGO_ERR_SHAPE;
  const hago_status s = check_rows(x, x_t, rows, cols, 2 * cols, row_stride, format, codes, scales, values);
  if (s != HAGO_OK || rows == 0 || cols == 0) return s;
  return from_hip(hago::launch_mx_silu_mul(x, real_type(x_t), rows, cols, row_stride, format, out_of(codes, scales, values), static_cast<hipStream_t>(stream)));
}

hago_status hago_mx_rmsnorm(const void* x, const void* residual, const void* gamma, hago_dtype x_t, int64_t rows, int64_t cols, int64_t row_stride, float eps,
                            hago_mx_format format, void* residual_out, void* codes, void* scales, void* values, void* stream) {
  const hago_status s = check_rows(x, x_t, rows, cols, cols, row_stride, format, codes, scales, values);
  if (s != HAGO_OK) return s;
  const size_t size = x_t == HAGO_F32 ? 4 : 2;
  if (!std::isfinite(eps) || eps < 0) return HAGO_ERR_PARAM;
  if (!hago::ptr_aligned(residual, size) || !hago::ptr_aligned(gamma, size) || !hago::ptr_aligned(residual_out, size)) return HAGO_ERR_PARAM;
  if (residual_out == x && residual_out && row_stride != cols) return HAGO_ERR_PARAM;  // (rows of another distance would be written over)
  if (rows == 0 || cols == 0) return HAGO_OK;
  return from_hip(hago::launch_mx_rmsnorm(x, residual, gamma, real_type(x_t), rows, cols, row_stride, eps, format, residual_out, out_of(codes, scales, values),
                                          static_cast<hipStream_t>(stream)));
}

hago_status hago_mx_dense(const void* a_codes, const void* a_scales, hago_mx_format a_format, const void* w_codes, const void* w_scales, const float* bias,
                          int64_t M, int64_t N, int64_t K, hago_dtype out_t, void* out, void* stream) {
  const hago::MxGemmArgs g = product(a_codes, a_scales, w_codes, w_scales, bias, nullptr, nullptr, M, M, 1, N, K, out_t, out);
  const hago_status s = check_product(g, M, M, 1, N, K, a_format, out_t);
  if (s != HAGO_OK || M == 0 || N == 0) return s;
  return from_hip(hago::launch_mx_gemm(g, a_format, static_cast<hipStream_t>(stream)));
}

hago_status hago_mx_dense_grouped(const void* a_codes, const void* a_scales, hago_mx_format a_format, int64_t a_rows, const int32_t* row_index,
                                  const void* w_codes, const void* w_scales, const float* bias, const int32_t* offsets, int64_t T, int64_t experts, int64_t N,
                                  int64_t K, hago_dtype out_t, void* out, void* stream) {
  const hago::MxGemmArgs g = product(a_codes, a_scales, w_codes, w_scales, bias, offsets, row_index, a_rows, T, experts, N, K, out_t, out);
  const hago_status s = check_product(g, a_rows, T, experts, N, K, a_format, out_t);
  if (s != HAGO_OK || T == 0 || N == 0 || experts == 0) return s;
  if (!offsets) return HAGO_ERR_NULL;
  if (!row_index && a_rows < T) return HAGO_ERR_SHAPE;
  return from_hip(hago::launch_mx_gemm(g, a_format, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
