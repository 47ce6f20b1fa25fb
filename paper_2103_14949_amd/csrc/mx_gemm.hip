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
    {{256, 256, 0, 0.00f, 6.25f, 0.81f, 1.21f, 0}, {128, 128, 0, 3.65f, 1.73f, 0.63f, 0.56f, 0}, {128, 64, 0, 3.66f, 0.94f, 0.53f, 0.42f, 0},
     {64, 64, 0, 2.72f, 0.56f, 0.33f, 0.28f, 0}, {64, 32, 0, 2.86f, 0.75f, 0.29f, 0.21f, 0},
     {16, 16, 4, 2.615f, 0.100f, 0.343f, 0.195f, 0.017f}, {16, 16, 8, 2.527f, 0.303f, 0.553f, 0.184f, 0.007f}, {32, 16, 2, 3.148f, 0.000f, 0.295f, 0.366f, 0.029f},
     {32, 16, 4, 2.807f, 0.195f, 0.271f, 0.294f, 0.049f}, {32, 16, 8, 2.392f, 0.607f, 0.776f, 0.291f, 0.015f}, {32, 32, 16, 1.057f, 3.026f, 2.788f, 0.193f, 0.080f}},
    {{256, 128, 0, 0.33f, 5.60f, 0.93f, 1.23f, 0}, {128, 128, 0, 1.73f, 3.93f, 0.87f, 0.82f, 0}, {128, 64, 0, 3.58f, 1.19f, 0.69f, 0.51f, 0},
     {64, 64, 0, 2.65f, 0.75f, 0.47f, 0.34f, 0}, {64, 32, 0, 2.61f, 1.16f, 0.39f, 0.27f, 0},
     {16, 16, 4, 2.666f, 0.028f, 0.336f, 0.237f, 0.095f}, {16, 16, 8, 2.572f, 0.251f, 0.577f, 0.218f, 0.095f}, {32, 16, 2, 3.063f, 0.000f, 0.300f, 0.390f, 0.104f},
     {32, 16, 4, 2.891f, 0.136f, 0.478f, 0.338f, 0.112f}, {32, 16, 8, 2.484f, 0.559f, 0.333f, 0.335f, 0.073f}, {32, 32, 16, 0.769f, 3.041f, 3.558f, 0.301f, 0.144f}}};

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
