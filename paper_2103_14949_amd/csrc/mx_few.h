// Microscaled products of few rows: the weights are read once, straight into registers, and that is the work.
//
// A wavefront has 16 TP features and 16 TQ rows and every W-th chunk of 512 k of them, W the wavefronts of a workgroup, whose
// sums meet in LDS and are added in the wavefronts' order.  Operands of v_mfma_scale_f32_16x16x128_f8f6f4, measured: lane l has row l % 16; of 4-bit codes
// the 16 bytes of k = 32 (l / 16) on, of 8-bit codes the 16 bytes of k = 16 (l / 16) on and of k = 64 + 16 (l / 16) on; its scale is the one of
// k = 32 (l / 16) on.  The loads of a chunk go out together: four pieces of 64 bytes of a row (two lines), 16 bytes of its scales.
//
// What bounds it: the weights' bytes, and how many of them are under way.  Where there is a workgroup for every CU and no more, 16 wavefronts each have 4 or 8 KB of a
// chunk so; weights not in the last-level cache, us with 8 and with 16: a row through 8192 x 8192 12.3, 11.1 (3.2 TB/s; 8.5 out of the cache), 8 rows through 4096
// features of 14336 k 12.7, 11.3.  The next chunk's loads behind the ones of this chunk give as much there (11.4, 10.9), and their registers cost more
// where there are many workgroups (16 rows of 60 experts 31 us, 44 so).  Nontemporal loads of the weights took longer (30, 36).
#pragma once

#include "mx_gemm.h"

namespace hago {

namespace {

constexpr int kMostFewWaves = 16;

// SPLIT: 8-bit rows in two parts (mx_split8), for 32-bit results.
template <int FA, int TP, int TQ, bool SPLIT>
__global__ __launch_bounds__(64 * kMostFewWaves) void mx_few_kernel(HAGO_MX_GEMM_PARAMETERS) {
  const MxGemmArgs g = HAGO_MX_GEMM_STRUCT;
  constexpr int BP = 16 * TP, BQ = 16 * TQ, PLANES = FA == kMxFp8 ? 2 : 1, STEPS = 4;
  extern __shared__ __attribute__((aligned(16))) float sums[];
  const int lane = threadIdx.x & 63, part = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
  const int tiles_p = (g.N + BP - 1) / BP;
  const uint32_t tile = g.place + blockIdx.x;
  const int tile_q = (int)(tile / (uint32_t)tiles_p), p0 = (int)(tile % (uint32_t)tiles_p) * BP;
  const MxGroups<BQ> groups(g);
  if (tile_q >= groups.tiles) return;
  const MxRows rows = groups.rows(g, tile_q);
  const int nq = min(rows.end - rows.row, BQ);
  const int padded = (g.K + 127) & ~127, steps = padded / 128;
  const int wbytes = padded / 2, abytes = FA == kMxFp4 ? wbytes : padded, sbytes = padded / 32;

  const uint8_t *wr[TP], *wsr[TP], *ar[TQ], *asr[TQ];  // the lane's rows
#pragma unroll
  for (int i = 0; i < TP; ++i) {
    const int64_t r = (int64_t)rows.expert * g.N + min(p0 + 16 * i + (lane & 15), g.N - 1);
    wr[i] = g.w + r * wbytes + part * 16;
    wsr[i] = g.w_scale + r * sbytes;
  }
#pragma unroll
  for (int j = 0; j < TQ; ++j) {
    const int64_t r = mx_row_of(g, rows.row + min(16 * j + (lane & 15), nq - 1));
    ar[j] = g.a + r * abytes + part * 16;
    asr[j] = g.a_scale + r * sbytes;
  }
  mx_v4f acc[TP][TQ];
#pragma unroll
  for (int i = 0; i < TP; ++i)
#pragma unroll
    for (int j = 0; j < TQ; ++j) acc[i][j] = mx_v4f{0, 0, 0, 0};

  typedef uint32_t v4u __attribute__((ext_vector_type(4)));
  typedef v4u v4u_4 __attribute__((aligned(4)));
  const uint32_t shift = 8 * part;
  // the scales of four steps, this lane's in the low byte of each
  auto scales = [&](const uint8_t* row, int step, bool whole) {
    v4u s;
    if (whole) {
      s = *reinterpret_cast<const v4u_4*>(row + 4 * step);
    } else {
#pragma unroll
      for (int u = 0; u < STEPS; ++u) s[u] = *reinterpret_cast<const uint32_t*>(row + 4 * min(step + u, steps - 1));
    }
    return s;
  };
  for (int step = wave * STEPS; step < steps; step += waves * STEPS) {
    const bool whole = step + STEPS <= steps;
    mx_v4i wf[STEPS][TP], af[STEPS][TQ * PLANES];
    v4u wsf[TP], asf[TQ];
#pragma unroll
    for (int u = 0; u < STEPS; ++u) {
      const int at = whole ? step + u : min(step + u, steps - 1);
#pragma unroll
      for (int i = 0; i < TP; ++i) wf[u][i] = *reinterpret_cast<const mx_v4i*>(wr[i] + at * 64);
    }
#pragma unroll
    for (int i = 0; i < TP; ++i) wsf[i] = scales(wsr[i], step, whole);
#pragma unroll
    for (int j = 0; j < TQ; ++j) asf[j] = scales(asr[j], step, whole);
#pragma unroll
    for (int u = 0; u < STEPS; ++u) {
      const int at = whole ? step + u : min(step + u, steps - 1);
#pragma unroll
      for (int j = 0; j < TQ; ++j)
#pragma unroll
        for (int h = 0; h < PLANES; ++h) af[u][j * PLANES + h] = *reinterpret_cast<const mx_v4i*>(ar[j] + at * 64 * PLANES + h * 64);
    }
#pragma unroll
    for (int u = 0; u < STEPS; ++u) {
      if (step + u >= steps) break;
#pragma unroll
      for (int j = 0; j < TQ; ++j) {
        const mx_v4i lo = af[u][j * PLANES], hi = af[u][j * PLANES + PLANES - 1];
        mx_v8i q, low;
        if constexpr (FA == kMxFp4) q = __builtin_shufflevector(lo, lo, 0, 1, 2, 3, -1, -1, -1, -1);
        else q = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        if constexpr (SPLIT) mx_split8(q, q, low);
#pragma unroll
        for (int i = 0; i < TP; ++i) {
          const mx_v8i p = __builtin_shufflevector(wf[u][i], wf[u][i], 0, 1, 2, 3, -1, -1, -1, -1);
          const auto add = [&](const mx_v8i& part) {
            acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(p, part, acc[i][j], kMxMfmaFormat<kMxFp4>, kMxMfmaFormat<FA>, 0, (int)(wsf[i][u] >> shift), 0,
                                                                         (int)(asf[j][u] >> shift));
          };
          add(q);
          if constexpr (SPLIT) add(low);
        }
      }
    }
  }

  // sums[wave][row][feature]: lane l has features 4 (l / 16) on of row l % 16
#pragma unroll
  for (int i = 0; i < TP; ++i)
#pragma unroll
    for (int j = 0; j < TQ; ++j)
      *reinterpret_cast<mx_v4f*>(sums + (wave * BQ + 16 * j + (lane & 15)) * BP + 16 * i + 4 * part) = acc[i][j];
  __syncthreads();
  for (int o = threadIdx.x; o < nq * BP; o += blockDim.x) {
    const int n = p0 + o % BP;
    if (n >= g.N) continue;
    float v = sums[o];
    for (int k = 1; k < waves; ++k) v += sums[k * BQ * BP + o];
    if (g.bias) v += g.bias[(int64_t)rows.expert * g.N + n];
    mx_store_one(g.out, g.type, (int64_t)(rows.row + o / BP) * g.N + n, v);
  }
}

template <int FA, int TP, int TQ, bool SPLIT>
hipError_t launch_few(const MxGemmArgs& g, int waves, hipStream_t st) {
  constexpr int BP = 16 * TP, BQ = 16 * TQ;
  static_assert(kMostFewWaves * BP * BQ * sizeof(float) <= 65536, "LDS without a raised limit");
  const int64_t tiles_q = g.offsets ? mx_most_tiles(g.T, g.experts, BQ) : (g.T + BQ - 1) / BQ;
  const int64_t tiles = (int64_t)((g.N + BP - 1) / BP) * tiles_q;
  return launch_mx_tiles(mx_few_kernel<FA, TP, TQ, SPLIT>, tiles, 64 * waves, waves * BP * BQ * sizeof(float), st, g);
}

}  // namespace

}  // namespace hago
