// Rotary positions: pairs of columns turned by position * frequency, each pair by the position on its own axis.
//
// Bytes bound it (a read and a write of the tensor), so the angles must not: a workgroup takes all the heads of a few tokens, or as
// many as give every thread something, works out each token's cosines and sines once (one pair a thread), and keeps them in LDS.  An
// angle far from the origin loses its fraction in 32 bits: position * frequency, its turns and their fraction are 64 bits, the
// polynomials behind them 32.
#include "mx_cache.h"
#include "mx_device.h"

namespace hago {

namespace {

constexpr int kThreads = 256;
constexpr int kRopeAngles = 2048;  // cosines of a workgroup, and as many sines

// cos and sin of 2 pi t.  t less its nearest quarter is at most 1/8, the angle pi/4: their series in eleven and ten terms of x are below
// 2^-28 off there.
__device__ __forceinline__ void cos_sin_turns(double t, float& c, float& s) {
  const double frac = t - __builtin_rint(t);
  const double quarter = __builtin_rint(frac * 4.0);
  const float x = (float)((frac - quarter * 0.25) * 6.283185307179586);
  const float z = x * x;
  float p = -2.50521084e-8f;  // -1/11!
  p = __builtin_fmaf(p, z, 2.75573192e-6f);
  p = __builtin_fmaf(p, z, -1.98412698e-4f);
  p = __builtin_fmaf(p, z, 8.33333333e-3f);
  p = __builtin_fmaf(p, z, -1.66666667e-1f);
  const float sn = __builtin_fmaf(p * z, x, x);
  float q = -2.75573192e-7f;  // -1/10!
  q = __builtin_fmaf(q, z, 2.48015873e-5f);
  q = __builtin_fmaf(q, z, -1.38888889e-3f);
  q = __builtin_fmaf(q, z, 4.16666667e-2f);
  q = __builtin_fmaf(q, z, -0.5f);
  const float cs = __builtin_fmaf(q, z, 1.0f);
  const int k = (int)quarter & 3;
  c = k & 1 ? sn : cs;
  s = k & 1 ? cs : sn;
  if (k == 1 || k == 2) c = -c;
  if (k >= 2) s = -s;
}

// Units of eight pairs (16 columns); behind them, units of 16 columns that stay as they are.
template <int TYPE, bool INTERLEAVED>
__global__ __launch_bounds__(kThreads) void rope_kernel(RopeArgs r, int tokens, int heads_each, int head_groups, int64_t tiles) {
  using T = typename MxElement<TYPE>::type;
  __shared__ __align__(16) float cosines[kRopeAngles];
  __shared__ __align__(16) float sines[kRopeAngles];
  const int pairs = r.pairs, padded = (pairs + 7) & ~7;
  const int turned = padded / 8, rest = r.dim - 2 * pairs;
  const bool in_place = r.out == r.x.data;
  const int units = turned + (in_place ? 0 : (rest + 15) / 16);
  for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    const int64_t t0 = tile / head_groups * tokens;
    const int h0 = (int)(tile % head_groups) * heads_each;
    const int nt = r.T - t0 < tokens ? (int)(r.T - t0) : tokens, nh = r.heads - h0 < heads_each ? r.heads - h0 : heads_each;
    if (tile != blockIdx.x) __syncthreads();
    for (int i = threadIdx.x; i < nt * padded; i += kThreads) {
      const int t = i / padded, j = i - t * padded;
      float c = 0.0f, s = 0.0f;
      if (j < pairs) {
        const int axis = r.axis ? r.axis[j] : 0;
        const int pos = axis >= 0 && axis < r.axes ? r.positions[(int64_t)axis * r.T + t0 + t] : 0;
        cos_sin_turns((double)pos * (double)r.frequencies[j] * 0.15915494309189535, c, s);
      }
      cosines[i] = c;
      sines[i] = s;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < nt * nh * units; i += kThreads) {
      const int u = i % units, th = i / units, h = th % nh, t = th / nh;
      const T* x = static_cast<const T*>(r.x.data) + (t0 + t) * r.x.row + (int64_t)(h0 + h) * r.x.head;
      T* y = static_cast<T*>(r.out) + (t0 + t) * r.out_row + (int64_t)(h0 + h) * r.out_head;
      float a[8], b[8];
      if (u >= turned) {
        const int col = 2 * pairs + (u - turned) * 16, n = r.dim - col;
        mx_load8<TYPE>(x + col, n, a);
        if (n > 8) mx_load8<TYPE>(x + col + 8, n - 8, b);
        mx_store8<TYPE>(y + col, n, a);
        if (n > 8) mx_store8<TYPE>(y + col + 8, n - 8, b);
        continue;
      }
      const int j = u * 8, n = pairs - j;
      float c[8], s[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) c[k] = cosines[t * padded + j + k], s[k] = sines[t * padded + j + k];
      if constexpr (INTERLEAVED) {
        mx_load8<TYPE>(x + 2 * j, 2 * n, a);
        if (n > 4) mx_load8<TYPE>(x + 2 * j + 8, 2 * n - 8, b);
        float ya[8], yb[8];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          ya[2 * k] = __builtin_fmaf(a[2 * k], c[k], -(a[2 * k + 1] * s[k]));
          ya[2 * k + 1] = __builtin_fmaf(a[2 * k + 1], c[k], a[2 * k] * s[k]);
          yb[2 * k] = __builtin_fmaf(b[2 * k], c[k + 4], -(b[2 * k + 1] * s[k + 4]));
          yb[2 * k + 1] = __builtin_fmaf(b[2 * k + 1], c[k + 4], b[2 * k] * s[k + 4]);
        }
        mx_store8<TYPE>(y + 2 * j, 2 * n, ya);
        if (n > 4) mx_store8<TYPE>(y + 2 * j + 8, 2 * n - 8, yb);
      } else {
        mx_load8<TYPE>(x + j, n, a);
        mx_load8<TYPE>(x + pairs + j, n, b);
        float ya[8], yb[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          ya[k] = __builtin_fmaf(a[k], c[k], -(b[k] * s[k]));
          yb[k] = __builtin_fmaf(b[k], c[k], a[k] * s[k]);
        }
        mx_store8<TYPE>(y + j, n, ya);
        mx_store8<TYPE>(y + pairs + j, n, yb);
      }
    }
  }
}

template <int TYPE>
hipError_t launch(const RopeArgs& r, hipStream_t st) {
  const int padded = (r.pairs + 7) & ~7;
  const int64_t units = padded / 8 + (r.dim - 2 * r.pairs + 15) / 16;
  // Four tokens a workgroup share nothing but the launch; fewer where the grid would not fill the GPU, and then fewer heads.
  int tokens = 4;
  while (tokens > 1 && ((int64_t)tokens * padded > kRopeAngles || r.T / tokens < 1024)) tokens /= 2;
  int heads_each = r.heads;
  while (heads_each > 1 && (int64_t)heads_each * tokens * units > kThreads && ((int64_t)r.T + tokens - 1) / tokens * ((r.heads + heads_each - 1) / heads_each) < 1024)
    heads_each = (heads_each + 1) / 2;
  const int groups = (r.heads + heads_each - 1) / heads_each;
  const int64_t tiles = ((int64_t)r.T + tokens - 1) / tokens * groups, most = max_blocks(kThreads);
  const dim3 grid((uint32_t)(tiles < most ? tiles : most));
  return launch_kernel(r.interleaved ? rope_kernel<TYPE, true> : rope_kernel<TYPE, false>, grid, dim3(kThreads), 0, st, r, tokens, heads_each, groups, tiles);
}

}  // namespace

hipError_t launch_rope(const RopeArgs& r, int type, hipStream_t st) {
  return type == kMxF32 ? launch<kMxF32>(r, st) : type == kMxBf16 ? launch<kMxBf16>(r, st) : launch<kMxF16>(r, st);
}

}  // namespace hago
