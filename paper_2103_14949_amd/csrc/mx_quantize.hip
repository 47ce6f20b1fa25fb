// Operators by rows whose result are microscaled codes: the quantization alone, behind a root-mean-square norm (with the residual's
// addition), and behind a gated activation.
//
// A lane takes eight consecutive columns, a quad of lanes a block of 32: the block's largest magnitude takes two lane exchanges, and
// the codes leave as 4 or 8 consecutive bytes per lane.  All three move bytes and little else.
#include "mx_device.h"

namespace hago {

namespace {

// ---- elementwise: codes of x, or of silu(x[:, :cols]) * x[:, cols:2 cols]

constexpr int kThreads = 256, kPerThread = 2;

// g / (1 + e^-g) * u with the exponential and the division rounded as the host's are (the operator waits for memory
// all the same).
__device__ __forceinline__ float silu_mul(float g, float u) { return g / (1.0f + expf(-g)) * u; }

template <int TYPE, int FORMAT, bool GATED>
__global__ __launch_bounds__(kThreads) void mx_quantize_kernel(const void* x, int64_t stride, int64_t rows, int cols, MxOut out) {
  using T = typename MxElement<TYPE>::type;
  const int padded = (cols + 127) & ~127;
  const uint32_t per_row = (uint32_t)padded / 8;
  // the workgroup's first place, in 64 bits; its threads' from there, in 32
  const uint64_t first = (uint64_t)blockIdx.x * (kThreads * kPerThread);
  const uint64_t row0 = first >> 32 ? first / per_row : (uint32_t)first / per_row;
  const uint32_t rest = (uint32_t)(first - row0 * per_row) + threadIdx.x;
  float v[kPerThread][8], u[kPerThread][8];
  int64_t row[kPerThread];
  int col[kPerThread];
#pragma unroll
  for (int i = 0; i < kPerThread; ++i) {
    const uint32_t at = rest + i * kThreads, r = at / per_row;
    row[i] = (int64_t)row0 + r;
    col[i] = (int)(at - r * per_row) * 8;
    if (row[i] >= rows) continue;
    const T* p = static_cast<const T*>(x) + row[i] * stride + col[i];
    mx_load8<TYPE>(p, cols - col[i], v[i]);
    if constexpr (GATED) mx_load8<TYPE>(p + cols, cols - col[i], u[i]);
  }
#pragma unroll
  for (int i = 0; i < kPerThread; ++i) {
    if (row[i] >= rows) continue;  // (whole quads: a row's places are a multiple of 16)
    if constexpr (GATED) {
#pragma unroll
      for (int k = 0; k < 8; ++k) v[i][k] = silu_mul(v[i][k], u[i][k]);
    }
    mx_put8<TYPE, FORMAT>(out, row[i], cols, padded, col[i], v[i]);
  }
}

// ---- norm: h = x + residual, y = h * rsqrt(mean(h^2) + eps) * gamma

struct NormArgs {
  const void *x, *residual, *gamma;
  void* residual_out;
  MxOut out;
  int64_t stride;
  int32_t cols;
  float eps;
};

// The squares' sum over the workgroup's threads, in 64 bits.
__device__ __forceinline__ double block_sum(float mine) {
  __shared__ double parts[16];
  double s = mine;
#pragma unroll
  for (int d = 32; d; d >>= 1) s += __shfl_xor(s, d);
  const int waves = blockDim.x >> 6;
  if (waves == 1) return s;
  if ((threadIdx.x & 63) == 0) parts[threadIdx.x >> 6] = s;
  __syncthreads();
  s = 0;
  for (int w = 0; w < waves; ++w) s += parts[w];
  return s;
}

// One workgroup per row, which stays in registers: VECS places of eight columns per thread.  VECS == 0: rows beyond the registers of a
// workgroup are read twice (the second time mostly from the L2).  A place is read, and its residual written, by one thread, so
// the new residual may lie where the old one, or x, was.
template <int TYPE, int FORMAT, int VECS>
__global__ __launch_bounds__(1024) void mx_rmsnorm_kernel(NormArgs a) {
  using T = typename MxElement<TYPE>::type;
  const int64_t row = blockIdx.x;
  const int cols = a.cols, padded = (cols + 127) & ~127, threads = blockDim.x;
  const T* x = static_cast<const T*>(a.x) + row * a.stride;
  const T* res = a.residual ? static_cast<const T*>(a.residual) + row * cols : nullptr;
  const T* gamma = static_cast<const T*>(a.gamma);
  auto load = [&](int col, float (&h)[8]) {
    mx_load8<TYPE>(x + col, cols - col, h);
    if (res) {
      float r[8];
      mx_load8<TYPE>(res + col, cols - col, r);
#pragma unroll
      for (int k = 0; k < 8; ++k) h[k] += r[k];
    }
  };
  auto square = [](const float (&h)[8], float s) {
#pragma unroll
    for (int k = 0; k < 8; ++k) s = __builtin_fmaf(h[k], h[k], s);
    return s;
  };
  auto finish = [&](int col, float (&h)[8], float factor) {
    if (a.residual_out && col < cols) mx_store8<TYPE>(static_cast<T*>(a.residual_out) + row * cols + col, cols - col, h);
    float g[8];
    if (gamma) mx_load8<TYPE>(gamma + col, cols - col, g);
#pragma unroll
    for (int k = 0; k < 8; ++k) h[k] = gamma ? h[k] * factor * g[k] : h[k] * factor;
    mx_put8<TYPE, FORMAT>(a.out, row, cols, padded, col, h);
  };
  auto factor_of = [&](double sum) { return 1.0f / sqrtf((float)(sum / cols) + a.eps); };
  if constexpr (VECS > 0) {
    float h[VECS][8];
    float sum = 0;
#pragma unroll
    for (int i = 0; i < VECS; ++i) {
      const int col = ((int)threadIdx.x + i * threads) * 8;
      if (col < padded) {
        load(col, h[i]);
        sum = square(h[i], sum);
      }
    }
    const float factor = factor_of(block_sum(sum));
#pragma unroll
    for (int i = 0; i < VECS; ++i) {
      const int col = ((int)threadIdx.x + i * threads) * 8;
      if (col < padded) finish(col, h[i], factor);
    }
  } else {
    float h[8], sum = 0;
    for (int col = (int)threadIdx.x * 8; col < padded; col += threads * 8) {
      load(col, h);
      sum = square(h, sum);
    }
    const float factor = factor_of(block_sum(sum));
    for (int col = (int)threadIdx.x * 8; col < padded; col += threads * 8) {
      load(col, h);
      finish(col, h, factor);
    }
  }
}

// f<TYPE, FORMAT>() for the runtime's two
template <typename F>
hipError_t by_type(int type, int format, const F& f) {
  auto with = [&]<int TYPE>() {
    return format == kMxFp4 ? f.template operator()<TYPE, kMxFp4>() : f.template operator()<TYPE, kMxFp8>();
  };
  switch (type) {
    case kMxF32: return with.template operator()<kMxF32>();
    case kMxBf16: return with.template operator()<kMxBf16>();
    default: return with.template operator()<kMxF16>();
  }
}

template <bool GATED>
hipError_t quantize(const void* x, int type, int64_t rows, int64_t cols, int64_t stride, int format, const MxOut& out, hipStream_t st) {
  // (a launch holds fewer than 2^32 threads)
  const int64_t most = max_blocks(kThreads) * (kThreads * kPerThread) / (mx_padded(cols) / 8);
  for (int64_t row = 0; row < rows; row += most) {
    const int64_t n = rows - row < most ? rows - row : most;
    const hipError_t e = by_type(type, format, [&]<int TYPE, int FORMAT>() {
      using T = typename MxElement<TYPE>::type;
      return launch_kernel(mx_quantize_kernel<TYPE, FORMAT, GATED>, dim3((unsigned)mx_quantize_blocks(n, cols)), dim3(kThreads), 0, st,
                           static_cast<const T*>(x) + row * stride, stride, n, (int)cols, out.from<T>(row, cols, format));
    });
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_mx_quantize(const void* x, int type, int64_t rows, int64_t cols, int64_t stride, int format, const MxOut& out, hipStream_t st) {
  return quantize<false>(x, type, rows, cols, stride, format, out, st);
}

hipError_t launch_mx_silu_mul(const void* x, int type, int64_t rows, int64_t cols, int64_t stride, int format, const MxOut& out, hipStream_t st) {
  return quantize<true>(x, type, rows, cols, stride, format, out, st);
}

hipError_t launch_mx_rmsnorm(const void* x, const void* residual, const void* gamma, int type, int64_t rows, int64_t cols, int64_t stride,
                             float eps, int format, void* residual_out, const MxOut& out, hipStream_t st) {
  const int64_t places = mx_padded(cols) / 8;
  const int vecs = places <= 1024 ? 1 : places <= 2048 ? 2 : places <= 4096 ? 4 : 0;
  const int64_t each = vecs ? (places + vecs - 1) / vecs : 1024;
  const unsigned threads = (unsigned)((each + 63) / 64 * 64);
  const int64_t most = max_blocks((int)threads);
  for (int64_t row = 0; row < rows; row += most) {
    const int64_t n = rows - row < most ? rows - row : most;
    const hipError_t e = by_type(type, format, [&]<int TYPE, int FORMAT>() {
      using T = typename MxElement<TYPE>::type;
      const T* res = residual ? static_cast<const T*>(residual) + row * cols : nullptr;
      T* res_out = residual_out ? static_cast<T*>(residual_out) + row * cols : nullptr;
      const NormArgs a{static_cast<const T*>(x) + row * stride, res, gamma, res_out, out.from<T>(row, cols, format), stride, (int32_t)cols, eps};
      const auto kern = vecs == 1   ? mx_rmsnorm_kernel<TYPE, FORMAT, 1>
                        : vecs == 2 ? mx_rmsnorm_kernel<TYPE, FORMAT, 2>
                        : vecs == 4 ? mx_rmsnorm_kernel<TYPE, FORMAT, 4>
                                    : mx_rmsnorm_kernel<TYPE, FORMAT, 0>;
      return launch_kernel(kern, dim3((unsigned)n), dim3(threads), 0, st, a);
    });
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace hago
