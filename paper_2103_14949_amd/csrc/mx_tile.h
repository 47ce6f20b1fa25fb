// Microscaled products on tiles whose operands stream from memory straight into LDS.
//
// D[i][j] = sum_k P[i][k] Q[j][k], P = weights (i = feature, contiguous in the result), Q = activations.  A stage is 256 k of a tile's
// rows: 128 bytes of a row of 4-bit codes (whole lines), two planes of 128 bytes of one of 8-bit codes, and 8 scale bytes a row.
// SLOTS slots of LDS hold a stage each.  A stage has four groups of 64 k, one matrix instruction per 32 x 32 block each; fragments
// are double-buffered by groups, so that before its last group a stage has been read completely: there lies the one barrier of a stage,
// behind it the loads of a later stage go out into the slot just read, and the next group's fragments come from the next slot.
//
// LDS.  A load of a wavefront fills 1 KB: 8 rows of 128 bytes, the 16-byte chunks of a row permuted by bits 1 to 3 of the row
// (swz in qgemm_stream.h), on the global side, so that fragments are read at the full rate.  Scales lie as [row][8 bytes]; a lane takes both dwords of its row and shifts
// its half's byte of either pair down, so that one instruction's byte select serves both halves of the wavefront.
//
// Out of range.  Loads go through descriptors of the tile's own rows (64-bit base, so tensors have any size), and lanes whose row or k
// lies outside get an offset beyond: zeros, code and scale, whose products are zero.
#pragma once

#include "mx_gemm.h"
#include "qgemm_stream.h"

namespace hago {

namespace {

__device__ __forceinline__ void mx_dma4(v4i rsrc, uint32_t lds_addr, uint32_t voff, uint32_t soff) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, %3 offen lds"
               :
               : "s"(lds_addr), "v"(voff), "s"(rsrc), "s"(soff)
               : "memory", "m0");
}

template <int FA, int WP, int WQ, int TP, int TQ, int SLOTS>
struct MxTile {
  static constexpr int NW = WP * WQ, NT = 64 * NW;
  static constexpr int BP = WP * TP * 32, BQ = WQ * TQ * 32;
  static constexpr int PLANES = FA == kMxFp8 ? 2 : 1;
  static constexpr int DATA = (BP + PLANES * BQ) * 128, STAGE = DATA + (BP + BQ) * 8;
  static constexpr int PITCH = TP * 128 + 16;  // bytes of a result row in LDS, at most
  static constexpr int LDS = SLOTS * STAGE > NW * 32 * PITCH ? SLOTS * STAGE : NW * 32 * PITCH;
};

template <int FA, int WP, int WQ, int TP, int TQ, int SLOTS>
__global__ __launch_bounds__(64 * WP * WQ, 1) void mx_tile_kernel(MxGemmArgs g) {
  using Tile = MxTile<FA, WP, WQ, TP, TQ, SLOTS>;
  constexpr int NW = Tile::NW, BP = Tile::BP, BQ = Tile::BQ, PLANES = Tile::PLANES, DATA = Tile::DATA, STAGE = Tile::STAGE;
  constexpr int GP = BP / 8, G = GP + PLANES * BQ / 8;   // loads of a stage: of P, in all
  constexpr int L = G / NW;                              // a wavefront issues loads wave, wave + NW, ...
  static_assert(GP % NW == 0 && G % NW == 0 && NW % 2 == 0, "a load's operand is the same in every wavefront");
  constexpr int GS = (BP + BQ) / 32, LS = (GS + NW - 1) / NW;  // loads of scales (some twice where NW does not divide them)
  constexpr int NM = TP * TQ;

  extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
  const int t = threadIdx.x, lane = t & 63, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int wp = wave % WP, wq = wave / WP;

  const int tiles_p = (g.N + BP - 1) / BP;
  int tile_p = 0;
  MxRows rows;
  const bool any = mx_find_rows<BQ>(g, [&](int tiles_q) {
    const uint32_t count = (uint32_t)tiles_p * (uint32_t)tiles_q;
    if (blockIdx.x >= count) return -1;
    int tile_q;
    panel_tile((int)xcd_run(blockIdx.x, count), tiles_p, tiles_q, tile_p, tile_q);
    return tile_q;
  }, rows);
  if (!any) return;
  const int p0 = tile_p * BP;
  const int np = min(g.N - p0, BP), nq = min(rows.end - rows.row, BQ);

  const int padded = (g.K + 127) & ~127;
  const uint32_t wbytes = (uint32_t)padded / 2, abytes = FA == kMxFp4 ? wbytes : (uint32_t)padded, sbytes = (uint32_t)padded / 32;
  const int64_t wrow = (int64_t)rows.expert * g.N + p0, arow = g.index ? 0 : rows.row;
  const uint32_t arows = g.index ? (uint32_t)g.a_rows : (uint32_t)nq;
  const v4i rs_w = make_rsrc(g.w + wrow * wbytes, (uint32_t)np * wbytes), rs_ws = make_rsrc(g.w_scale + wrow * sbytes, (uint32_t)np * sbytes);
  const v4i rs_a = make_rsrc(g.a + arow * abytes, arows * abytes), rs_as = make_rsrc(g.a_scale + arow * sbytes, arows * sbytes);
  const uint32_t lds0 = (uint32_t)(size_t)(__attribute__((address_space(3))) uint8_t*)smem;

  // row r of the tile's activations -> its row among those the descriptors begin with; negative: none
  auto a_row = [&](int r) { return r < nq ? (g.index ? mx_row_of(g, rows.row + r) : r) : -1; };

  // the lane's byte offset of every load: its row's start and its chunk of a stage (the chunk is the same in every load, since
  // every load of a wavefront has the wavefront's parity)
  const int lrow = lane / 8;
  const uint32_t lck = (uint32_t)(((lane % 8) ^ swz<128>((wave & 1) * 8 + lrow)) * 16);
  uint32_t voff[L];
#pragma unroll
  for (int d = 0; d < L; ++d) {
    const bool isq = d >= GP / NW;
    if (!isq) {
      const int r = (wave + NW * d) * 8 + lrow;
      voff[d] = r < np ? (uint32_t)r * wbytes + lck : kOob;
    } else {
      const int v = (wave + NW * d - GP) * 8 + lrow, r = a_row(v % BQ);
      voff[d] = r >= 0 ? (uint32_t)r * abytes + lck + (uint32_t)(v / BQ) * 128 : kOob;
    }
  }
  uint32_t soff[LS];
  uint32_t sdst[LS];
  bool sisq[LS];
#pragma unroll
  for (int d = 0; d < LS; ++d) {
    const int grp = (wave + NW * d) % GS;
    const int v = grp * 32 + lane / 2;
    sisq[d] = grp >= BP / 32;
    const int r = sisq[d] ? a_row(v - BP) : v < np ? v : -1;
    soff[d] = r >= 0 ? (uint32_t)r * sbytes + (uint32_t)(lane % 2) * 4 : kOob;
    sdst[d] = lds0 + (uint32_t)(DATA + grp * 256);
  }
  // the sums start from the bias (of features beyond the last one, which nobody stores: the last one's)
  mx_v16f acc[TP][TQ];
  if (g.bias) {
    const float* bias = g.bias + (int64_t)rows.expert * g.N;
#pragma unroll
    for (int i = 0; i < TP; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float b = bias[min(p0 + (wp * TP + i) * 32 + 8 * (r / 4) + 4 * half + r % 4, g.N - 1)];
#pragma unroll
        for (int j = 0; j < TQ; ++j) acc[i][j][r] = b;
      }
  } else {
#pragma unroll
    for (int i = 0; i < TP; ++i)
#pragma unroll
      for (int j = 0; j < TQ; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[i][j][r] = 0;
  }
  const int KT = (padded + 255) / 256;
  constexpr int ISSUES = L + LS;
  // loads lo .. hi - 1 of a stage
  auto issue = [&](int stage, auto slot, auto lo, auto hi) {
    constexpr int base = decltype(slot)::value * STAGE;
    const uint32_t kp = (uint32_t)stage * 128, kq = kp * PLANES, ks = (uint32_t)stage * 8;
    const bool there = stage < KT;
    [&]<int... I>(std::integer_sequence<int, I...>) {
      ([&] {
        constexpr int d = decltype(lo)::value + I;
        if constexpr (d < L) {
          constexpr bool isq = d >= GP / NW;
          constexpr int plane = isq ? ((NW * d - GP) * 8) / BQ : 0;  // (BQ rows are whole rounds of loads, or all of a round)
          const uint32_t at = (isq ? kq + plane * 128 : kp) + lck, end = isq ? abytes : wbytes;
          dma16s(isq ? rs_a : rs_w, lds0 + (uint32_t)(base + NW * d * 1024) + (uint32_t)wave * 1024, at < end ? voff[d] : kOob, there ? (isq ? kq : kp) : 0);
        } else {
          constexpr int s = d - L;
          mx_dma4(sisq[s] ? rs_as : rs_ws, sdst[s] + base, ks + (uint32_t)(lane % 2) * 4 < sbytes ? soff[s] : kOob, there ? ks : 0);
        }
      }(), ...);
    }(std::make_integer_sequence<int, decltype(hi)::value - decltype(lo)::value>{});
  };
  static_assert(PLANES == 1 || (BQ / 8) % NW == 0, "a load's plane is the same in every wavefront");
  template_int<0> i0;
  [&]<int... I>(std::integer_sequence<int, I...>) { (issue(I, template_int<I>{}, i0, template_int<ISSUES>{}), ...); }(std::make_integer_sequence<int, SLOTS>{});

  // fragment addresses inside a stage
  const int frow = lane & 31;
  auto chunk_at = [&](int c) { return (c ^ swz<128>(frow & 15)) * 16; };
  const int prow = wp * TP * 32 + frow, qrow = wq * TQ * 32 + frow;
  int pa[4], qa[PLANES * 4];
#pragma unroll
  for (int h = 0; h < 4; ++h) {
    pa[h] = prow * 128 + chunk_at(2 * h + half);
    if constexpr (FA == kMxFp4) {
      qa[h] = (BP + qrow) * 128 + chunk_at(2 * h + half);
    } else {
      qa[2 * h] = (BP + (h / 2) * BQ + qrow) * 128 + chunk_at(4 * (h % 2) + half);
      qa[2 * h + 1] = (BP + (h / 2) * BQ + qrow) * 128 + chunk_at(4 * (h % 2) + 2 + half);
    }
  }
  const int psa = DATA + prow * 8, qsa = DATA + (BP + qrow) * 8, shift = 8 * half;
  constexpr int kFrag = 32 * 128;
  typedef uint32_t v2u __attribute__((ext_vector_type(2)));
  mx_v4i pf[2][TP], qf[2][TQ * PLANES];
  v2u sc[2][TP + TQ];
  // read r of the NR of a group's operands, activations first
  constexpr int NR = TQ * PLANES + TP;
  auto read = [&](const uint8_t* base, auto set, auto group, int r) {
    constexpr int S = decltype(set)::value, H = decltype(group)::value;
    if (r < TQ * PLANES) qf[S][r] = *reinterpret_cast<const mx_v4i*>(base + qa[PLANES * H + r % PLANES] + (r / PLANES) * kFrag);
    else pf[S][r - TQ * PLANES] = *reinterpret_cast<const mx_v4i*>(base + pa[H] + (r - TQ * PLANES) * kFrag);
  };
  auto read_scale = [&](const uint8_t* base, auto set, int r) {
    constexpr int S = decltype(set)::value;
    sc[S][r] = *reinterpret_cast<const v2u*>(base + (r < TP ? psa + r * 256 : qsa + (r - TP) * 256));
  };
  auto shift_scales = [&](auto set) {
    constexpr int S = decltype(set)::value;
#pragma unroll
    for (int r = 0; r < TP + TQ; ++r) sc[S][r] = sc[S][r] >> (uint32_t)shift;
  };
  // Group H of a stage in slot R: multiply its set of fragments, behind the instructions go the reads of the next group's set (from `next`) and,
  // in the last group, of the next stage's scales, and the loads of stage `dma_stage`.
  auto multiply = [&](auto hconst, auto ring, const uint8_t* next, int dma_stage) {
    constexpr int H = decltype(hconst)::value, S = H & 1, R = decltype(ring)::value & 1;
    constexpr int reads = NR + (H == 3 ? TP + TQ : 0), each = (reads + NM - 1) / NM > 2 ? (reads + NM - 1) / NM : 2;
    [&]<int... Mi>(std::integer_sequence<int, Mi...>) {
      ([&] {
        constexpr int m = Mi, j = m / TP, i = m % TP;
        const mx_v4i p4 = pf[S][i], q4 = qf[S][j * PLANES], q5 = qf[S][j * PLANES + PLANES - 1];
        const mx_v8i p = __builtin_shufflevector(p4, p4, 0, 1, 2, 3, -1, -1, -1, -1);
        mx_v8i q;
        if constexpr (FA == kMxFp4) q = __builtin_shufflevector(q4, q4, 0, 1, 2, 3, -1, -1, -1, -1);
        else q = __builtin_shufflevector(q4, q5, 0, 1, 2, 3, 4, 5, 6, 7);
        acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(p, q, acc[i][j], kMxMfmaFormat<kMxFp4>, kMxMfmaFormat<FA>, 2 * (H % 2), (int)sc[R][i][H / 2],
                                                                    2 * (H % 2), (int)sc[R][TP + j][H / 2]);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int r = each * m; r < each * m + each && r < reads; ++r) {
          if (r < NR) read(next, template_int<(S ^ 1)>{}, template_int<(H + 1) % 4>{}, r);
          else read_scale(next, template_int<(R ^ 1)>{}, r - NR);
        }
        if constexpr (H == 3) issue(dma_stage, ring, template_int<m * ISSUES / NM>{}, template_int<(m + 1) * ISSUES / NM>{});
        __builtin_amdgcn_sched_barrier(0);
      }(), ...);
    }(std::make_integer_sequence<int, NM>{});
    if constexpr (H == 3) shift_scales(template_int<(R ^ 1)>{});
  };
  auto stage_body = [&](int kt, auto ring) {
    constexpr int R = decltype(ring)::value;
    const uint8_t* here = smem + R * STAGE;
    const uint8_t* other = smem + (R + 1) % SLOTS * STAGE;
    multiply(template_int<0>{}, ring, here, 0);
    multiply(template_int<1>{}, ring, here, 0);
    multiply(template_int<2>{}, ring, here, 0);
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((SLOTS - 2) * ISSUES) : "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    multiply(template_int<3>{}, ring, other, kt + SLOTS);
  };

  asm volatile("s_waitcnt vmcnt(%0)" ::"n"((SLOTS - 1) * ISSUES) : "memory");  // stage 0
  __syncthreads();
#pragma unroll
  for (int r = 0; r < NR; ++r) read(smem, i0, i0, r);
#pragma unroll
  for (int r = 0; r < TP + TQ; ++r) read_scale(smem, i0, r);
  shift_scales(i0);
  static_assert(SLOTS % 2 == 0 && SLOTS * ISSUES <= 63, "sets of scales by the slot's parity; loads that can be counted");
  for (int kt = 0; kt < KT; kt += SLOTS) {
    [&]<int... I>(std::integer_sequence<int, I...>) {
      ([&] {
        if (I == 0 || kt + I < KT) stage_body(kt + I, template_int<I>{});
      }(), ...);
    }(std::make_integer_sequence<int, SLOTS>{});
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // (the stages beyond K; before LDS is reused)
  __syncthreads();

  // Results: 32 rows of a wavefront's features at a time go through its own piece of LDS and leave by whole rows.
  uint8_t* mine = smem + wave * 32 * Tile::PITCH;
  const int n0 = p0 + wp * TP * 32;
  auto leave = [&]<int TYPE>() {
    using T = typename MxElement<TYPE>::type;
    constexpr int kPitch = TP * 32 * sizeof(T) + 16, kVec = 16 / sizeof(T), kLanes = TP * 32 / kVec;
#pragma unroll
    for (int j = 0; j < TQ; ++j) {
#pragma unroll
      for (int i = 0; i < TP; ++i)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
          const int n = i * 32 + 2 * r + 4 * half;
          T v[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) v[k] = (T)acc[i][j][r + k];
          __builtin_memcpy(mine + frow * kPitch + n * sizeof(T), v, sizeof(v));
        }
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
      const int q = wq * TQ * 32 + j * 32;
#pragma unroll 4
      for (int it = 0; it < kLanes / 2; ++it) {
        const int r = (lane + 64 * it) / kLanes, c = (lane + 64 * it) % kLanes, n = n0 + c * kVec;
        if (q + r >= nq || n >= g.N) continue;
        const uint8_t* src = mine + r * kPitch + c * 16;
        T* dst = static_cast<T*>(g.out) + (int64_t)(rows.row + q + r) * g.N + n;
        if (n + kVec <= g.N) {
          __builtin_nontemporal_store(*reinterpret_cast<const mx_u4*>(src), reinterpret_cast<mx_u4_any*>(dst));
        } else {
#pragma unroll 1
          for (int k = 0; n + k < g.N; ++k) dst[k] = reinterpret_cast<const T*>(src)[k];
        }
      }
      __builtin_amdgcn_wave_barrier();
    }
  };
  if (g.type == kMxF32) leave.template operator()<kMxF32>();
  else if (g.type == kMxBf16) leave.template operator()<kMxBf16>();
  else leave.template operator()<kMxF16>();
}

template <int FA, int WP, int WQ, int TP, int TQ, int SLOTS>
hipError_t launch_tile(const MxGemmArgs& g, hipStream_t st) {
  using Tile = MxTile<FA, WP, WQ, TP, TQ, SLOTS>;
  const auto kern = mx_tile_kernel<FA, WP, WQ, TP, TQ, SLOTS>;
  static std::atomic<uint64_t> attr_set{0};  // the devices whose dynamic-LDS limit is raised
  const hipError_t e = raise_lds_limit(reinterpret_cast<const void*>(kern), Tile::LDS, attr_set);
  if (e != hipSuccess) return e;
  const int64_t tiles_q = g.offsets ? mx_most_tiles(g.T, g.experts, Tile::BQ) : (g.T + Tile::BQ - 1) / Tile::BQ;
  const int64_t tiles = (int64_t)((g.N + Tile::BP - 1) / Tile::BP) * tiles_q;
  return launch_kernel(kern, dim3((unsigned)tiles), dim3(Tile::NT), Tile::LDS, st, g);
}

}  // namespace

}  // namespace hago
