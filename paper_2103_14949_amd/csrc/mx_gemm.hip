// Microscaled matrix products, dense and grouped by expert: D[i][j] = sum_k P[i][k] Q[j][k], P = weights (E2M1), Q = activations
// (E2M1 or E4M3), on the scaled matrix instructions, which multiply 32 k of a row by its scale before they add.
//
// Operand layout of v_mfma_scale_f32_32x32x64_f8f6f4, measured: lane l has row l % 32 of either operand; of 4-bit codes the 16 bytes
// of k = 32 (l / 32) on, of 8-bit codes the 16 bytes of k = 16 (l / 32) on and those of k = 32 + 16 (l / 32) on; the scale that lane l
// gives is the one of k = 32 (l / 32) on of its row.  Products of two 4-bit codes are added exactly (2e-8 of the terms' sum against 64
// bits).  Of 8-bit codes the instruction adds terms aligned to the largest one, and what lies some 2^-17 below it is cut off.
#include <algorithm>
#include <cmath>

#include "mx_few.h"
#include "mx_tile.h"

namespace hago {

namespace {

// What a call would take in a kernel, in us, from what this chip measured over a thousand dense and grouped products of 1 to 16384 rows,
// 64 to 8192 features and k (the kernel it picks is 3 % slower than the fastest one on the average, 17 % in one of twenty).  A tile's time is `each` and
// `step` per stage of 256 k, workgroups of a round on a CU share it, and alone it takes `alone` per stage, for it waits for its loads.
struct MxShape {
  int bp, bq;      // features and rows of a tile
  int waves;       // of a workgroup with few rows; 0: operands through LDS
  float fixed, each, alone, step;
  float step_row;  // few rows: more per stage (of 512 k there) for the activations of 16 rows
};
constexpr int kShapes = 13;
constexpr MxShape kMxShapes[2][kShapes] = {
    {{256, 256, 0, 0.00f, 6.23f, 0.82f, 1.21f, 0}, {128, 128, 0, 3.62f, 1.74f, 0.48f, 0.56f, 0}, {128, 64, 0, 3.66f, 0.93f, 0.54f, 0.42f, 0},
     {64, 64, 0, 2.72f, 0.56f, 0.34f, 0.28f, 0}, {64, 32, 0, 2.86f, 0.74f, 0.29f, 0.21f, 0}, {16, 16, 4, 2.602f, 0.101f, 0.313f, 0.197f, 0.015f},
     {16, 16, 8, 2.509f, 0.302f, 0.494f, 0.183f, 0.009f}, {32, 16, 2, 3.202f, 0.000f, 0.153f, 0.342f, 0.050f}, {32, 16, 4, 2.789f, 0.196f, 0.139f, 0.292f, 0.052f},
     {32, 16, 8, 2.332f, 0.609f, 0.984f, 0.294f, 0.015f}, {32, 32, 16, 1.024f, 3.031f, 3.269f, 0.192f, 0.081f}, {16, 16, 16, 1.996f, 0.866f, 0.300f, 0.184f, 0.000f},
     {32, 16, 16, 1.628f, 1.577f, 0.773f, 0.266f, 0.042f}},
    {{256, 128, 0, 0.29f, 5.61f, 0.46f, 1.23f, 0}, {128, 128, 0, 1.69f, 3.96f, 0.31f, 0.82f, 0}, {128, 64, 0, 3.56f, 1.19f, 0.70f, 0.52f, 0},
     {64, 64, 0, 2.65f, 0.75f, 0.47f, 0.34f, 0}, {64, 32, 0, 2.60f, 1.16f, 0.39f, 0.27f, 0}, {16, 16, 4, 2.657f, 0.028f, 0.302f, 0.239f, 0.093f},
     {16, 16, 8, 2.526f, 0.252f, 0.565f, 0.223f, 0.090f}, {32, 16, 2, 3.043f, 0.000f, 0.300f, 0.383f, 0.112f}, {32, 16, 4, 2.858f, 0.136f, 0.462f, 0.345f, 0.108f},
     {32, 16, 8, 2.458f, 0.559f, 0.910f, 0.337f, 0.073f}, {32, 32, 16, 0.760f, 3.036f, 3.549f, 0.301f, 0.146f}, {16, 16, 16, 2.056f, 0.844f, 0.696f, 0.230f, 0.054f},
     {32, 16, 16, 1.591f, 1.627f, 1.162f, 0.310f, 0.112f}}};

int pick_shape(const MxGemmArgs& g, int a_format) {
  const double k = (double)mx_padded(g.K);
  // groups that have a row, where rows fall to them by chance, and the rows of one
  const double used = g.offsets ? g.experts * -std::expm1(-(double)g.T / g.experts) : 1, rows = g.T / used;
  int best = 0;
  double least = 1e300;
  for (int i = 0; i < kShapes; ++i) {
    const MxShape& s = kMxShapes[a_format][i];
    const double per_group = g.offsets ? (rows > s.bq / 2 ? rows / s.bq + 0.5 : 1.0) : std::ceil(rows / s.bq);
    const double tiles = std::ceil((double)g.N / s.bp) * used * per_group / 256;  // per CU
    double t;
    if (s.waves) {
      const double chunks = std::ceil(k / 512);
      t = s.fixed + std::max(std::ceil(chunks / s.waves) * s.alone, std::max(1.0, tiles) * (s.each + chunks * (s.step + s.step_row * std::min(rows, (double)s.bq) / 16)));
    } else {
      const double stages = std::ceil(k / 256);
      t = s.fixed + std::max(stages * s.alone, std::ceil(tiles) * (s.each + stages * s.step));
    }
    if (t < least) least = t, best = i;
  }
  return best;
}

template <int FA>
hipError_t launch_shape(const MxGemmArgs& g, int shape, hipStream_t st) {
  switch (shape) {
    case 0: return FA == kMxFp4 ? launch_tile<kMxFp4, 2, 4, 4, 2, 2>(g, st) : launch_tile<kMxFp8, 4, 2, 2, 2, 2>(g, st);
    case 1: return launch_tile<FA, 2, 2, 2, 2, 2>(g, st);
    case 2: return launch_tile<FA, 2, 2, 2, 1, 2>(g, st);
    case 3: return launch_tile<FA, 2, 2, 1, 1, 2>(g, st);
    case 4: return launch_tile<FA, 2, 1, 1, 1, 4>(g, st);
    case 5: case 6: case 11: return launch_few<FA, 1, 1>(g, kMxShapes[FA][shape].waves, st);
    case 10: return launch_few<FA, 2, 2>(g, kMxShapes[FA][shape].waves, st);
    default: return launch_few<FA, 2, 1>(g, kMxShapes[FA][shape].waves, st);
  }
}

}  // namespace

hipError_t launch_mx_gemm(const MxGemmArgs& g, int a_format, hipStream_t st) {
  int shape = test_hook(kHookMxKernel);
  if (shape < 0 || shape >= kShapes) shape = pick_shape(g, a_format);
  return a_format == kMxFp4 ? launch_shape<kMxFp4>(g, shape, st) : launch_shape<kMxFp8>(g, shape, st);
}

}  // namespace hago
