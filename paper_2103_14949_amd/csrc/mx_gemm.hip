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
constexpr int kShapes = 11;
constexpr MxShape kMxShapes[2][kShapes] = {
    {{256, 256, 0, 0.00f, 6.32f, 0.30f, 1.24f, 0}, {128, 128, 0, 2.46f, 2.17f, 0.66f, 0.54f, 0}, {128, 64, 0, 2.83f, 1.04f, 0.47f, 0.43f, 0},
     {64, 64, 0, 2.85f, 0.58f, 0.34f, 0.28f, 0}, {64, 32, 0, 2.90f, 0.77f, 0.28f, 0.21f, 0},
     {16, 16, 4, 2.59f, 0.11f, 0.32f, 0.195f, 0.013f}, {16, 16, 8, 2.49f, 0.33f, 0.27f, 0.185f, 0.0f}, {32, 16, 2, 2.99f, 0.0f, 0.09f, 0.366f, 0.041f},
     {32, 16, 4, 2.65f, 0.23f, 0.22f, 0.307f, 0.044f}, {32, 16, 8, 2.32f, 0.58f, 0.88f, 0.301f, 0.010f}, {32, 32, 16, 1.04f, 3.07f, 2.69f, 0.174f, 0.092f}},
    {{256, 128, 0, 0.00f, 4.91f, 1.00f, 1.28f, 0}, {128, 128, 0, 0.22f, 4.78f, 0.55f, 0.82f, 0}, {128, 64, 0, 2.63f, 1.42f, 0.65f, 0.55f, 0},
     {64, 64, 0, 2.80f, 0.80f, 0.47f, 0.34f, 0}, {64, 32, 0, 2.75f, 1.21f, 0.34f, 0.27f, 0},
     {16, 16, 4, 2.65f, 0.02f, 0.29f, 0.240f, 0.096f}, {16, 16, 8, 2.55f, 0.23f, 0.50f, 0.228f, 0.090f}, {32, 16, 2, 3.00f, 0.0f, 0.30f, 0.383f, 0.119f},
     {32, 16, 4, 2.75f, 0.15f, 0.38f, 0.372f, 0.094f}, {32, 16, 8, 2.39f, 0.48f, 0.56f, 0.361f, 0.064f}, {32, 32, 16, 0.77f, 3.05f, 3.54f, 0.315f, 0.134f}}};

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
    case 5: case 6: return launch_few<FA, 1, 1>(g, kMxShapes[FA][shape].waves, st);
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
