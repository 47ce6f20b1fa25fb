// Operators by rows whose result are microscaled codes: the quantization alone, behind a root-mean-square norm (with the residual's
// addition), and behind a gated activation.
//
// A lane takes eight consecutive columns, a quad of lanes a block of 32: the block's largest magnitude takes two lane exchanges, and
// the codes leave as 4 or 8 consecutive bytes per lane.  All three move bytes and little else: 8192 x 8192 fp32 to 4 bits with values in 99 us, norm
// of 8192 x 4096 bf16 with residual and values in 51, activation of 16384 x 4096 bf16 with values in 82 (5.8, 5.9 and 5.7 TB/s; a copy of 1 GiB by hago_probe_copy 6.3).
#include "mx_device.h"

namespace hago {

namespace {

// ---- elementwise: codes of x, or of silu(x[:, :cols]) * x[:, cols:2 cols]

constexpr int kThreads = 256;

// g / (1 + e^-g) * u within a few units of the last place.  e^-g is 2^t with t = -g log2 e in two parts, the quotient takes one correction.  From -80 on e^-g
// stays below 2^116, so that its reciprocal is a normal number; above 80 the quotient is g.
// (16384 x 4096 bf16 with values: 105 us with expf and the division, rounded once each, 100 with this quotient, 84 with one place per thread and
// hinted stores, 82 since far gates are none of its business.)
constexpr float kLog2e = 1.44269502f, kLog2eRest = 1.92596303e-8f, kLn2 = 0.693147182f, kFarGate = -80.0f;
__device__ __forceinline__ float silu_mul(float g, float u) {
  const float t = g * -kLog2e;
  const float rest = __builtin_fmaf(g, -kLog2e, -t) - g * kLog2eRest;
  const float e = __builtin_amdgcn_exp2f(t);
  const float d = 1.0f + __builtin_fmaf(e, rest * kLn2, e);
  const float r = __builtin_amdgcn_rcpf(d);
  const float q = g * r;
  const float s = __builtin_fmaf(__builtin_fmaf(q, d, -g), -r, q);  // (in these signs -0 stays -0)
  return (g <= 80.0f ? s : g) * u;  // (the comparison fails for a NaN, which is g itself)
}

// The same for gates below -80: g e^g u, to 2^-115 of it.  The quotient alone may be below binary32 where u brings the product back,
// so it is carried in 64 bits.  Of minus infinity the formula, and this, make NaN.
__device__ __forceinline__ float silu_mul_far(float g, float u) {
  const float c = fmaxf(g, -1000.0f), t = c * -kLog2e, n = __builtin_rintf(t);  // (below it the product is 0 for any u)
  const float rest = __builtin_fmaf(c, -kLog2e, -t) - c * kLog2eRest;
  const float e = __builtin_amdgcn_exp2f(n - t);
  const double part = (double)__builtin_fmaf(e, -rest * kLn2, e) * (double)g;
  return (float)(__builtin_amdgcn_ldexp(part, -(int)n) * (double)u);
}

// (One place per thread: two took 0 to 20 % longer, four 10 to 60 % on small tensors.)
template <int TYPE, int FORMAT, bool GATED>
__global__ __launch_bounds__(kThreads) void mx_quantize_kernel(const void* x, int64_t stride, int64_t rows, int cols, uint8_t* codes, uint8_t* scales, void* values) {
  const MxOut out{codes, scales, values};
  using T = typename MxElement<TYPE>::type;
  const int padded = (cols + 127) & ~127;
  const uint32_t per_row = (uint32_t)padded / 8;
  // the workgroup's first place, in 64 bits; its threads' from there, in 32
  const uint64_t first = (uint64_t)blockIdx.x * kThreads;
  const uint64_t row0 = first >> 32 ? first / per_row : (uint32_t)first / per_row;
  const uint32_t at = (uint32_t)(first - row0 * per_row) + threadIdx.x, r = at / per_row;
  const int64_t row = (int64_t)row0 + r;
  const int col = (int)(at - r * per_row) * 8;
  if (row >= rows) return;  // (whole quads: a row's places are a multiple of 16)
  const T* p = static_cast<const T*>(x) + row * stride + col;
  float v[8];
  mx_load8<TYPE>(p, cols - col, v);
  if constexpr (GATED) {
    float u[8];
    mx_load8<TYPE>(p + cols, cols - col, u);
    bool far = false;
    float y[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) far |= v[k] < kFarGate, y[k] = silu_mul(v[k], u[k]);
    if (far) {
#pragma unroll 1
      for (int k = 0; k < 8; ++k) y[k] = v[k] < kFarGate ? silu_mul_far(v[k], u[k]) : y[k];
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = y[k];
  }
  mx_put8<TYPE, FORMAT>(out, row, cols, padded, col, v);
}

// ---- norm: h = x + residual, y = h * rsqrt(mean(h^2) + eps) * gamma

// Sum over LANES consecutive lanes (16, 32 or 64), in all of them.
template <int LANES>
__device__ __forceinline__ double lanes_sum(double v) {
  const auto with = [&](const auto& exchange) {
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint64_t lo = exchange((uint32_t)b), hi = exchange((uint32_t)(b >> 32));
    v += __builtin_bit_cast(double, hi << 32 | lo);
  };
  auto dpp = [&]<int CTRL>() { with([](uint32_t d) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)d, CTRL, 0xf, 0xf, true); }); };
  dpp.template operator()<0xB1>();   // quad_perm 1,0,3,2
  dpp.template operator()<0x4E>();   // quad_perm 2,3,0,1
  dpp.template operator()<0x141>();  // mirrored within eight lanes
  dpp.template operator()<0x140>();  // mirrored within sixteen
  // (of a swap of a register with a copy of it, one of the two results is what the other lanes had)
  const bool odd16 = threadIdx.x & 16, odd32 = threadIdx.x & 32;
  if constexpr (LANES >= 32)
    with([&](uint32_t d) {
      const auto s = __builtin_amdgcn_permlane16_swap(d, d, false, false);
      const uint32_t even = s[0], odd = s[1];
      return odd16 ? even : odd;
    });
  if constexpr (LANES >= 64)
    with([&](uint32_t d) {
      const auto s = __builtin_amdgcn_permlane32_swap(d, d, false, false);
      const uint32_t even = s[0], odd = s[1];
      return odd32 ? even : odd;
    });
  return v;
}

// 1 / sqrt(v) to the last bits of binary64: the hardware's estimate and one step of Newton's.  0 of an infinity.
__device__ __forceinline__ double inverse_root(double v) {
  const double r = __builtin_amdgcn_rsq(v);
  return r == 0.0 ? 0.0 : r * (1.5 - 0.5 * v * r * r);
}

// LANES lanes per row, 16 to 64 (rows of up to 512 columns, 256 / LANES rows per workgroup), or 0: one workgroup per row.  The row stays in registers,
// VECS places of eight columns per thread.  VECS == 0: rows beyond the registers of a
// workgroup are read twice (the second time mostly from the L2).  A place is read, and its residual written, by one thread, so
// the new residual may lie where the old one, or x, was.  gamma is under way while the squares are added up.  The sum and its
// root are in 64 bits, and y is rounded to 32 once, from products in two parts: what y is rounded to next are codes, and an error in front of that moves some of them.
template <int TYPE, int FORMAT, int VECS, int LANES>
__global__ __launch_bounds__(1024) void mx_rmsnorm_kernel(const void* x_, const void* residual, int64_t stride, int cols, float eps, const void* gamma_,
                                                          void* residual_out, uint8_t* codes, uint8_t* scales, void* values, int64_t rows) {
  const MxOut out{codes, scales, values};
  using T = typename MxElement<TYPE>::type;
  const int64_t row = LANES ? (int64_t)blockIdx.x * (256 / (LANES ? LANES : 1)) + threadIdx.x / (LANES ? LANES : 1) : blockIdx.x;
  if (LANES && row >= rows) return;  // (all lanes of a row)
  const int place = LANES ? threadIdx.x % (LANES ? LANES : 1) : threadIdx.x, threads = LANES ? LANES : blockDim.x;
  const int padded = (cols + 127) & ~127;
  const T* x = static_cast<const T*>(x_) + row * stride;
  const T* res = residual ? static_cast<const T*>(residual) + row * cols : nullptr;
  const T* gamma = static_cast<const T*>(gamma_);
  auto load = [&](int col, float (&h)[8]) {
    mx_load8<TYPE>(x + col, cols - col, h);
    if (res) {
      float r[8];
      mx_load8<TYPE>(res + col, cols - col, r);
#pragma unroll
      for (int k = 0; k < 8; ++k) h[k] += r[k];
    }
  };
  auto square = [](const float (&h)[8], double s) {
#pragma unroll
    for (int k = 0; k < 8; ++k) s = __builtin_fma((double)h[k], (double)h[k], s);
    return s;
  };
  auto finish = [&](int col, float (&h)[8], double factor, const float (&g)[8]) {
    if (residual_out && col < cols) mx_store8<TYPE>(static_cast<T*>(residual_out) + row * cols + col, cols - col, h);
    if (factor > 0x1p-100 && factor < 0x1p100) {
      const float f = (float)factor, rest = (float)(factor - f);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        // (what is left of the products with its sign turned: so -0 stays -0)
        const float p = h[k] * f, e = __builtin_fmaf(-h[k], rest, __builtin_fmaf(-h[k], f, p));
        const float y = p * g[k];
        h[k] = gamma ? y - __builtin_fmaf(e, g[k], __builtin_fmaf(-p, g[k], y)) : p - e;
      }
    } else {  // (rows at the ends of binary32, where the factor or its second part is no normal number of it, and rows that have no factor)
#pragma unroll
      for (int k = 0; k < 8; ++k) h[k] = col + k < cols ? (float)((double)h[k] * factor * (gamma ? (double)g[k] : 1.0)) : 0.0f;
    }
    mx_put8<TYPE, FORMAT>(out, row, cols, padded, col, h);
  };
  auto factor_of = [&](double mine) {
    double sum;
    if constexpr (LANES != 0) {
      sum = lanes_sum<LANES>(mine);
    } else {
      __shared__ double parts[16];
      const int lane = threadIdx.x & 63, waves = blockDim.x >> 6;
      sum = lanes_sum<64>(mine);
      if (waves > 1) {
        if (lane == 0) parts[threadIdx.x >> 6] = sum;
        __syncthreads();
        sum = lanes_sum<16>((lane & 15) < waves ? parts[lane & 15] : 0.0);
      }
    }
    return inverse_root(sum / (double)cols + (double)eps);
  };
  if constexpr (VECS > 0) {
    float h[VECS][8], g[VECS][8];
    double sum = 0;
#pragma unroll
    for (int i = 0; i < VECS; ++i) {
      const int col = (place + i * threads) * 8;
      if (col < padded) load(col, h[i]);
    }
    if (gamma) {
#pragma unroll
      for (int i = 0; i < VECS; ++i) {
        const int col = (place + i * threads) * 8;
        if (col < padded) mx_load8<TYPE>(gamma + col, cols - col, g[i]);
      }
    }
#pragma unroll
    for (int i = 0; i < VECS; ++i)
      if ((place + i * threads) * 8 < padded) sum = square(h[i], sum);
    const double factor = factor_of(sum);
#pragma unroll
    for (int i = 0; i < VECS; ++i) {
      const int col = (place + i * threads) * 8;
      if (col < padded) finish(col, h[i], factor, g[i]);
    }
  } else {
    float h[8], g[8];
    double sum = 0;
    const uint32_t end = padded;  // (a place behind the last one may lie beyond 2^31)
    for (uint32_t at = place * 8; at < end; at += threads * 8) {
      load((int)at, h);
      sum = square(h, sum);
    }
    const double factor = factor_of(sum);
    for (uint32_t at = place * 8; at < end; at += threads * 8) {
      const int col = (int)at;
      load(col, h);
      if (gamma) mx_load8<TYPE>(gamma + col, cols - col, g);
      finish(col, h, factor, g);
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
  const int64_t most = max_blocks(kThreads) * kThreads / (mx_padded(cols) / 8);
  for (int64_t row = 0; row < rows; row += most) {
    const int64_t n = rows - row < most ? rows - row : most;
    const hipError_t e = by_type(type, format, [&]<int TYPE, int FORMAT>() {
      using T = typename MxElement<TYPE>::type;
      const MxOut to = out.from<T>(row, cols, format);
      const int64_t blocks = (n * (mx_padded(cols) / 8) + kThreads - 1) / kThreads;
      return launch_kernel(mx_quantize_kernel<TYPE, FORMAT, GATED>, dim3((unsigned)blocks), dim3(kThreads), 0, st,
                           static_cast<const T*>(x) + row * stride, stride, n, (int)cols, to.codes, to.scales, to.values);
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
  const int lanes = places <= 16 ? 16 : places <= 32 ? 32 : places <= 64 ? 64 : 0;
  const int vecs = places <= 1024 ? 1 : places <= 2048 ? 2 : places <= 4096 ? 4 : 0;
  const int64_t each = vecs ? (places + vecs - 1) / vecs : 1024;
  const unsigned threads = lanes ? 256 : (unsigned)((each + 63) / 64 * 64), per_block = lanes ? 256 / lanes : 1;
  const int64_t most = max_blocks((int)threads) * per_block;
  for (int64_t row = 0; row < rows; row += most) {
    const int64_t n = rows - row < most ? rows - row : most;
    const hipError_t e = by_type(type, format, [&]<int TYPE, int FORMAT>() {
      using T = typename MxElement<TYPE>::type;
      const T* res = residual ? static_cast<const T*>(residual) + row * cols : nullptr;
      T* res_out = residual_out ? static_cast<T*>(residual_out) + row * cols : nullptr;
      const MxOut to = out.from<T>(row, cols, format);
      const auto kern = lanes == 16   ? mx_rmsnorm_kernel<TYPE, FORMAT, 1, 16>
                        : lanes == 32 ? mx_rmsnorm_kernel<TYPE, FORMAT, 1, 32>
                        : lanes == 64 ? mx_rmsnorm_kernel<TYPE, FORMAT, 1, 64>
                        : vecs == 1   ? mx_rmsnorm_kernel<TYPE, FORMAT, 1, 0>
                        : vecs == 2   ? mx_rmsnorm_kernel<TYPE, FORMAT, 2, 0>
                        : vecs == 4   ? mx_rmsnorm_kernel<TYPE, FORMAT, 4, 0>
                                      : mx_rmsnorm_kernel<TYPE, FORMAT, 0, 0>;
      return launch_kernel(kern, dim3((unsigned)((n + per_block - 1) / per_block)), dim3(threads), 0, st, static_cast<const T*>(x) + row * stride, res, stride, (int)cols, eps, gamma,
                           res_out, to.codes, to.scales, to.values, n);
    });
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace hago
