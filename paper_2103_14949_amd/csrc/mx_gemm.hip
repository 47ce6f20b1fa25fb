// Microscaled matrix products, dense and grouped by expert: D[i][j] = sum_k P[i][k] Q[j][k], P = weights (E2M1), Q = activations
// (E2M1 or E4M3), on the scaled matrix instructions, which multiply 32 k of a row by its scale before they add.
//
// Operand layout of v_mfma_scale_f32_32x32x64_f8f6f4, measured: lane l has row l % 32 of either operand; of 4-bit codes the 16 bytes
// of k = 32 (l / 32) on, of 8-bit codes the 16 bytes of k = 16 (l / 32) on and those of k = 32 + 16 (l / 32) on; the scale that lane l
// gives is the one of k = 32 (l / 32) on of its row.  Products of two 4-bit codes are added exactly (2e-8 of the terms' sum against 64
// bits).  Of 8-bit codes the instruction adds terms aligned to the largest one, and what lies some 2^-17 below it is cut off.
#include "mx_tile.h"

namespace hago {

namespace {

// Tiles BP x BQ (features x rows) by number, the largest one first.
template <int FA>
hipError_t launch_shape(const MxGemmArgs& g, int shape, hipStream_t st) {
  switch (shape) {
    case 0: return FA == kMxFp4 ? launch_tile<kMxFp4, 2, 4, 4, 2>(g, st) : launch_tile<kMxFp8, 4, 2, 2, 2>(g, st);  // 256 x 256, 256 x 128
    case 1: return launch_tile<FA, 2, 2, 2, 2>(g, st);                                                             // 128 x 128
    default: return launch_tile<FA, 2, 2, 1, 1>(g, st);                                                            // 64 x 64
  }
}

int64_t count_tiles(const MxGemmArgs& g, int bp, int bq) {
  return (int64_t)((g.N + bp - 1) / bp) * (g.offsets ? mx_most_tiles(g.T, g.experts, bq) : (g.T + bq - 1) / bq);
}

}  // namespace

hipError_t launch_mx_gemm(const MxGemmArgs& g, int a_format, hipStream_t st) {
  int shape = test_hook(kHookMxKernel);
  if (shape < 0) shape = count_tiles(g, 256, a_format == kMxFp4 ? 256 : 128) >= 256 ? 0 : count_tiles(g, 128, 128) >= 256 ? 1 : 2;
  return a_format == kMxFp4 ? launch_shape<kMxFp4>(g, shape, st) : launch_shape<kMxFp8>(g, shape, st);
}

}  // namespace hago
