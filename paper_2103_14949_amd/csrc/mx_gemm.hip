// Microscaled matrix products, dense and grouped by expert: D[i][j] = sum_k P[i][k] Q[j][k], P = weights (E2M1), Q = activations
// (E2M1 or E4M3), on the scaled matrix instructions, which multiply 32 k of a row by its scale before they add.
//
// Operand layout of v_mfma_scale_f32_32x32x64_f8f6f4, measured: lane l has row l % 32 of either operand; of 4-bit codes the 16 bytes
// of k = 32 (l / 32) on, of 8-bit codes the 16 bytes of k = 16 (l / 32) on and those of k = 32 + 16 (l / 32) on; the scale that lane l
// gives is the one of k = 32 (l / 32) on of its row.  Products of two 4-bit codes are added exactly (2e-8 of the terms' sum against 64
// bits).  Of 8-bit codes the instruction adds terms aligned to the largest one, and what lies some 2^-17 below it is cut off.
#include "mx_gemm.h"

namespace hago {

namespace {

// One wavefront per 32 x 32 tile, operands straight from memory.
template <int FA>
__global__ __launch_bounds__(64) void mx_gemm_simple_kernel(MxGemmArgs g) {
  const int lane = threadIdx.x, half = lane >> 5;
  const int tiles_p = (g.N + 31) / 32;
  const int tile_p = (int)(blockIdx.x % (uint32_t)tiles_p), tile_q = (int)(blockIdx.x / (uint32_t)tiles_p);
  MxRows rows;
  if (!mx_find_rows<32>(g, [&](int) { return tile_q; }, rows)) return;
  const int padded = (g.K + 127) & ~127;
  const int t = rows.row + (lane & 31);
  const int64_t ra = mx_row_of(g, min(t, rows.end - 1));
  const int64_t rw = (int64_t)rows.expert * g.N + min(tile_p * 32 + (lane & 31), g.N - 1);
  const uint8_t* a = g.a + ra * (FA == kMxFp4 ? padded / 2 : padded) + half * 16;
  const uint8_t* w = g.w + rw * (padded / 2) + half * 16;
  const uint8_t* as = g.a_scale + ra * (padded / 32) + half;
  const uint8_t* ws = g.w_scale + rw * (padded / 32) + half;
  mx_v16f acc = {};
  for (int k = 0; k < padded; k += 64) {
    mx_v8i p = {}, q = {};
    const mx_v4i wv = *reinterpret_cast<const mx_v4i*>(w + k / 2);
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = wv[i];
    const mx_v4i lo = *reinterpret_cast<const mx_v4i*>(a + (FA == kMxFp4 ? k / 2 : k));
#pragma unroll
    for (int i = 0; i < 4; ++i) q[i] = lo[i];
    if constexpr (FA == kMxFp8) {
      const mx_v4i hi = *reinterpret_cast<const mx_v4i*>(a + k + 32);
#pragma unroll
      for (int i = 0; i < 4; ++i) q[4 + i] = hi[i];
    }
    acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(p, q, acc, kMxMfmaFormat<kMxFp4>, kMxMfmaFormat<FA>, 0, ws[k / 32], 0, as[k / 32]);
  }
  if (t >= rows.end) return;
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    const int n = tile_p * 32 + 8 * (r / 4) + 4 * half + r % 4;
    if (n < g.N) mx_store_one(g.out, g.type, (int64_t)t * g.N + n, g.bias ? acc[r] + g.bias[(int64_t)rows.expert * g.N + n] : acc[r]);
  }
}

}  // namespace

hipError_t launch_mx_gemm(const MxGemmArgs& g, int a_format, hipStream_t st) {
  const int64_t tiles = (int64_t)((g.N + 31) / 32) * (g.offsets ? mx_most_tiles(g.T, g.experts, 32) : (g.T + 31) / 32);
  return launch_kernel(a_format == kMxFp4 ? mx_gemm_simple_kernel<kMxFp4> : mx_gemm_simple_kernel<kMxFp8>, dim3((unsigned)tiles), dim3(64), 0, st, g);
}

}  // namespace hago
