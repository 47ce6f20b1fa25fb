// Rotary positions: pairs of columns turned by position * frequency, each pair by the position on its own axis.
//
// Bytes bound it (a read and a write of the tensor), so the angles must not: a workgroup takes all the heads of a few tokens, or as
// many as give every thread something, works out each token's cosines and sines once (one pair a thread), and keeps them in LDS.  An
// angle far from the origin loses its fraction in 32 bits: position * frequency, its turns and their fraction are 64 bits, the
// polynomials behind them 32.
//
// 8192 x 40 heads x 128 columns, bf16, from a strided tensor: 32.5 us, 5.2 TB/s (a copy has 5.9); 4001 x 20 x 80 f16 on three axes 9.3 us (13.5 with loads of single elements at the ends of the
// pairs); one token 4.4 us, the host's.
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

// i / d for i < 2^31: i * factor >> (31 + shift).
struct Divisor {
  uint32_t d, factor;
  int shift;
  explicit Divisor(uint32_t n) : d(n), factor(0), shift(0) {
    while ((1ll << shift) < n) ++shift;
    factor = (uint32_t)((1ull << (31 + shift)) / n + 1);
  }
  __device__ __forceinline__ uint32_t divide(uint32_t i) const { return (uint32_t)((uint64_t)i * factor >> (31 + shift)); }
};

// Units of eight pairs (16 columns).  Neighbours: the columns behind the last pair are in such units too, and pass; halves: they have units of their own.  Loads
// reach to the end of a row where they may, which is eight columns at once.  A thread's next unit is under way while it turns one, its
// first while the angles are worked out.
template <int TYPE, bool INTERLEAVED>
__global__ __launch_bounds__(kThreads) void rope_kernel(RopeArgs r, int tokens, Divisor heads_each, Divisor units, uint32_t head_groups, int64_t tiles) {
  using T = typename MxElement<TYPE>::type;
  __shared__ __align__(16) float cosines[kRopeAngles];
  __shared__ __align__(16) float sines[kRopeAngles];
  const int pairs = r.pairs, padded = (pairs + 7) & ~7, turned = padded / 8;
  for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    const int64_t unit_tile = tile / head_groups, t0 = unit_tile * tokens;
    const int h0 = (int)(tile - unit_tile * head_groups) * (int)heads_each.d;
    const int nt = r.T - t0 < tokens ? (int)(r.T - t0) : tokens;
    const uint32_t all = nt * heads_each.d * units.d;
    float a[8], b[8];
    // unit i: its part of a row, and the row (heads behind the last: none)
    const auto place = [&](uint32_t i, int& u, int& t, int& h) {
      const uint32_t th = units.divide(i);
      t = (int)heads_each.divide(th);
      u = (int)(i - th * units.d), h = h0 + (int)(th - t * heads_each.d);
      return i < all && h < r.heads;
    };
    const auto load = [&](uint32_t i) {
      int u, t, h;
      if (!place(i, u, t, h)) return;
      const T* x = static_cast<const T*>(r.x.data) + (t0 + t) * r.x.row + (int64_t)h * r.x.head;
      const int j = u * 8, first = INTERLEAVED ? 2 * j : u < turned ? j : 2 * pairs + 16 * (u - turned), second = !INTERLEAVED && u < turned ? pairs + j : first + 8;
      mx_load8<TYPE>(x + first, r.dim - first, a);
      if (second < r.dim) mx_load8<TYPE>(x + second, r.dim - second, b);
    };
    load(threadIdx.x);
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
    for (uint32_t i = threadIdx.x; i < all; i += kThreads) {
      float ya[8], yb[8];
      int u, t, h;
      const bool there = place(i, u, t, h);
      T* y = static_cast<T*>(r.out) + (t0 + t) * r.out_row + (int64_t)h * r.out_head;
      const int j = u * 8, n = pairs - j;
#pragma unroll
      for (int k = 0; k < 8; ++k) ya[k] = a[k], yb[k] = b[k];
      if (u < turned) {
        float c[8], s[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) c[k] = cosines[t * padded + j + k], s[k] = sines[t * padded + j + k];
        if constexpr (INTERLEAVED) {
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            if (k < n) {
              ya[2 * k] = __builtin_fmaf(a[2 * k], c[k], -(a[2 * k + 1] * s[k]));
              ya[2 * k + 1] = __builtin_fmaf(a[2 * k + 1], c[k], a[2 * k] * s[k]);
            }
            if (k + 4 < n) {
              yb[2 * k] = __builtin_fmaf(b[2 * k], c[k + 4], -(b[2 * k + 1] * s[k + 4]));
              yb[2 * k + 1] = __builtin_fmaf(b[2 * k + 1], c[k + 4], b[2 * k] * s[k + 4]);
            }
          }
        } else {
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            ya[k] = __builtin_fmaf(a[k], c[k], -(b[k] * s[k]));
            yb[k] = __builtin_fmaf(b[k], c[k], a[k] * s[k]);
          }
        }
      }
      load(i + kThreads);
      if (!there) continue;
      if (!INTERLEAVED && u < turned) {
        mx_store8<TYPE>(y + j, n, ya);
        mx_store8<TYPE>(y + pairs + j, n, yb);
      } else {
        const int first = INTERLEAVED ? 2 * j : 2 * pairs + 16 * (u - turned);
        mx_store8<TYPE>(y + first, r.dim - first, ya);
        if (first + 8 < r.dim) mx_store8<TYPE>(y + first + 8, r.dim - first - 8, yb);
      }
    }
  }
}

template <int TYPE>
hipError_t launch(const RopeArgs& r, hipStream_t st) {
  const int padded = (r.pairs + 7) & ~7;
  // (in place, what is not turned is where it belongs)
  const bool in_place = r.out == r.x.data;
  const int64_t units = r.interleaved ? (in_place ? padded / 8 : (r.dim + 15) / 16) : padded / 8 + (in_place ? 0 : (r.dim - 2 * r.pairs + 15) / 16);
  if (!units) return hipSuccess;
  // Two tokens a workgroup (8192 x 40 x 128 bf16: 32.5 us, with four 33.2, with eight 35.2); one, and then fewer heads, where the grid would not fill the GPU.
  int tokens = 2;
  while (tokens > 1 && ((int64_t)tokens * padded > kRopeAngles || r.T / tokens < 1024)) tokens /= 2;
  int heads_each = r.heads;
  while (heads_each > 1 && (int64_t)heads_each * tokens * units > kThreads && ((int64_t)r.T + tokens - 1) / tokens * ((r.heads + heads_each - 1) / heads_each) < 1024)
    heads_each = (heads_each + 1) / 2;
  const int groups = (r.heads + heads_each - 1) / heads_each;
  const int64_t tiles = ((int64_t)r.T + tokens - 1) / tokens * groups, most = max_blocks(kThreads);
  const dim3 grid((uint32_t)(tiles < most ? tiles : most));
  return launch_kernel(r.interleaved ? rope_kernel<TYPE, true> : rope_kernel<TYPE, false>, grid, dim3(kThreads), 0, st, r, tokens, Divisor((uint32_t)heads_each),
                       Divisor((uint32_t)units), (uint32_t)groups, tiles);
}

}  // namespace

hipError_t launch_rope(const RopeArgs& r, int type, hipStream_t st) {
  return type == kMxF32 ? launch<kMxF32>(r, st) : type == kMxBf16 ? launch<kMxBf16>(r, st) : launch<kMxF16>(r, st);
}

}  // namespace hago
