// Microscaled products on tiles whose operands stream from memory straight into LDS.
//
// D[i][j] = sum_k P[i][k] Q[j][k], P = weights (i = feature, contiguous in the result), Q = activations.  A stage is KB = 256 or 128 k of a
// tile's rows: KB / 2 bytes of a row of 4-bit codes (256: whole lines), planes of 128 bytes of one of 8-bit codes, and KB / 32 scale bytes a
// row.  SLOTS slots of LDS hold a stage each.  A stage has groups of 64 k, one matrix instruction per 32 x 32 block each; fragments
// are double-buffered by groups, so that before its last group a stage has been read completely: there lies the one barrier of a stage,
// behind it the loads of a later stage go out into the slot just read, and the next group's fragments come from the next slot.
//
// What bounds it.  The matrix instructions alone run at 6800 (4-bit rows) and 4200 TFLOP/s (8-bit rows) on such codes; 8192 rows through
// 8192 x 8192 take 265 us (4150) and 390 us (2820).  The matrix unit is busy for 56 % and 74 % of the cycles, at 1.6 GHz of 2.4: power sets the
// clock.  The tile is 256 x 256 by eight wavefronts of 128 x 64, 0.75 KB of LDS per instruction; four of 128 x 128, with
// 0.5 KB, take 283 us against 260 with 4-bit rows, so those bytes are not all of the rest.  The 6.4 M cycles of bank conflicts counted with 4-bit rows are
// the reads of scales, of which a stage of 256 k has 8 bytes a row (one of 128 k has 4, and none).  8-bit rows leave no room for two stages of 256 k of it (197 KB); three of 128 k fit (150 KB): 390 us, and 453 with
// 256 x 128 tiles of two stages of 256 k.  4-bit rows with stages of 128 k in four slots take 331 us instead of 276, 128 x 128 tiles 512 instead of 356:
// a row's half line is fetched twice and there are twice the barriers.  A higher priority for wavefronts in matrix instructions made no difference.
//
// A workgroup stays for several tiles where the loads of the next one's first stages fit behind the last one's (Tile::STAYS).  Results leave
// from the registers by pieces of whole 64 bytes that quads of lanes exchange, and by LDS where a wavefront has one 32-feature block only.
//
// LDS.  A load of a wavefront fills 1 KB: 8 rows of 128 bytes or 16 of 64, the 16-byte chunks of a row permuted by bits of the row
// (swz in qgemm_stream.h), on the global side, so that fragments are read at the full rate.  Scales lie as [row][KB / 32 bytes]; a lane takes a
// dword for 128 k and shifts its half's byte of either pair down, so that one byte select serves both halves of the wavefront.
//
// Out of range.  Loads go through descriptors of the tile's own rows (64-bit base, so tensors have any size), and lanes whose row or k
// lies outside get an offset beyond: zeros, code and scale, whose products are zero.
#pragma once

#include "mx_gemm.h"
#include "qgemm_stream.h"

namespace hago {

namespace {

// Loads into the LDS (qgemm_stream.h) at a constant distance behind a scalar address: what lies in scalar registers for every load of every
// slot is missing elsewhere.
template <int AT>
__device__ __forceinline__ void mx_dma16(v4i rsrc, uint32_t lds_addr, uint32_t voff, uint32_t soff) {
  asm volatile("s_add_u32 m0, %0, %4\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
               :
               : "s"(lds_addr), "v"(voff), "s"(rsrc), "s"(soff), "n"(AT)
               : "memory", "m0", "scc");
}
template <int AT>
__device__ __forceinline__ void mx_dma4(v4i rsrc, uint32_t lds_addr, uint32_t voff, uint32_t soff) {
  asm volatile("s_add_u32 m0, %0, %4\n\ts_nop 0\n\tbuffer_load_dword %1, %2, %3 offen lds"
               :
               : "s"(lds_addr), "v"(voff), "s"(rsrc), "s"(soff), "n"(AT)
               : "memory", "m0", "scc");
}

template <int FA, int WP, int WQ, int TP, int TQ, int SLOTS, int KB>
struct MxTile {
  static constexpr int NW = WP * WQ, NT = 64 * NW;
  static constexpr int BP = WP * TP * 32, BQ = WQ * TQ * 32;
  static constexpr int PB = KB / 2, SB = KB / 32;  // bytes of a row of weights and of scales in a stage
  static constexpr int QB = FA == kMxFp8 ? 128 : PB, PLANES = FA == kMxFp8 ? KB / 128 : 1;  // of a plane's row of activations
  static constexpr int DATA = BP * PB + PLANES * BQ * QB, STAGE = DATA + (BP + BQ) * SB;
  // rows leave from the registers where a wavefront has pairs of 32-feature blocks, by LDS otherwise
  static constexpr bool BY_LDS = TP % 2 != 0;
  static constexpr int PITCH = TP * 128 + 16;  // bytes of a result row in LDS, at most
  static constexpr int LDS = !BY_LDS || SLOTS * STAGE > NW * 32 * PITCH ? SLOTS * STAGE : NW * 32 * PITCH;
  // A workgroup goes from tile to tile; the next one's first stages are under way while a tile's results leave.
  static constexpr bool STAYS = !BY_LDS && SLOTS == 2 && TP * TQ < 8;
  static constexpr int RESIDENT = 160 * 1024 / LDS < 16 / NW ? 160 * 1024 / LDS : 16 / NW;  // workgroups that a CU holds
};

// 32 rows of a wavefront's features at a time go through its own piece of LDS and leave by whole rows.
template <int TYPE, int TP, int TQ>
__device__ __forceinline__ void leave_by_lds(const MxGemmArgs& g, const mx_v16f (&acc)[TP][TQ], int row, int q0, int nq, int n0, int lane, uint8_t* mine) {
  using T = typename MxElement<TYPE>::type;
  constexpr int kPitch = TP * 32 * sizeof(T) + 16, kVec = 16 / sizeof(T), kLanes = TP * 32 / kVec;
  const int half = lane >> 5;
#pragma unroll
  for (int j = 0; j < TQ; ++j) {
#pragma unroll
    for (int i = 0; i < TP; ++i)
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        T v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = (T)acc[i][j][r + k];
        __builtin_memcpy(mine + (lane & 31) * kPitch + (i * 32 + 2 * r + 4 * half) * sizeof(T), v, sizeof(v));
      }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
#pragma unroll 4
    for (int it = 0; it < kLanes / 2; ++it) {
      const int r = q0 + j * 32 + (lane + 64 * it) / kLanes, c = (lane + 64 * it) % kLanes, n = n0 + c * kVec;
      if (r >= nq || n >= g.N) continue;
      const uint8_t* src = mine + (lane + 64 * it) / kLanes * kPitch + c * 16;
      T* dst = static_cast<T*>(g.out) + (int64_t)(row + r) * g.N + n;
      if (n + kVec <= g.N) {
        __builtin_nontemporal_store(*reinterpret_cast<const mx_u4*>(src), reinterpret_cast<mx_u4_any*>(dst));
      } else {
#pragma unroll 1
        for (int k = 0; n + k < g.N; ++k) dst[k] = reinterpret_cast<const T*>(src)[k];
      }
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// Straight from the registers.  A lane has 4 features in every 8 of its row; the halves of the wavefront exchange theirs between two blocks of 32
// features, so that either has whole rows of one, and the lanes of a quad exchange 16-byte pieces, so that a quad stores 64
// consecutive bytes of a row at a time.
template <int TYPE, int TP, int TQ>
__device__ __forceinline__ void leave_by_quads(const MxGemmArgs& g, const mx_v16f (&acc)[TP][TQ], int row, int q0, int nq, int n0, int lane) {
  using T = typename MxElement<TYPE>::type;
  constexpr int kVec = 16 / sizeof(T), D = sizeof(T), kSets = sizeof(T) / 2;  // dwords of 4 features / 2, sets of 64 bytes in 32 features
  const int half = lane >> 5;
#pragma unroll
  for (int j = 0; j < TQ; ++j)
#pragma unroll
    for (int i = 0; i < TP; i += 2) {
      uint32_t piece[4 * kSets][4];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        T a[4], b[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) a[k] = (T)acc[i][j][4 * q + k], b[k] = (T)acc[i + 1][j][4 * q + k];
        uint32_t x[D], y[D];
        __builtin_memcpy(x, a, sizeof(a));
        __builtin_memcpy(y, b, sizeof(b));
#pragma unroll
        for (int d = 0; d < D; ++d) {
          const auto s = __builtin_amdgcn_permlane32_swap(x[d], y[d], false, false);
          // (this lane's block: features 8 q + 0 .. 3 and 8 q + 4 .. 7)
          if constexpr (D == 2) piece[q][d] = s[0], piece[q][2 + d] = s[1];
          else piece[2 * q][d] = s[0], piece[2 * q + 1][d] = s[1];
        }
      }
#pragma unroll
      for (int set = 0; set < kSets; ++set) {
        uint32_t(&p)[4][4] = *reinterpret_cast<uint32_t(*)[4][4]>(&piece[4 * set]);
        quad_transpose<4>(p, lane);
        const int n = n0 + (i + half) * 32 + set * 4 * kVec + (lane & 3) * kVec;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const int r = q0 + j * 32 + (lane & 28) + t;
          if (r >= nq || n >= g.N) continue;
          T* dst = static_cast<T*>(g.out) + (int64_t)(row + r) * g.N + n;
          const mx_u4 v = {p[t][0], p[t][1], p[t][2], p[t][3]};
          if (n + kVec <= g.N) {
            __builtin_nontemporal_store(v, reinterpret_cast<mx_u4_any*>(dst));
          } else {
            T e[kVec];
            __builtin_memcpy(e, &v, 16);
#pragma unroll
            for (int k = 0; k < kVec - 1; ++k)
              if (n + k < g.N) dst[k] = e[k];
          }
        }
      }
    }
}

// SPLIT: 8-bit rows in two parts (mx_split8), for 32-bit results.
template <int FA, int WP, int WQ, int TP, int TQ, int SLOTS, int KB, bool SPLIT>
__global__ __launch_bounds__(64 * WP * WQ, 1) void mx_tile_kernel(HAGO_MX_GEMM_PARAMETERS) {
  const MxGemmArgs g = HAGO_MX_GEMM_STRUCT;
  using Tile = MxTile<FA, WP, WQ, TP, TQ, SLOTS, KB>;
  constexpr int NW = Tile::NW, BP = Tile::BP, BQ = Tile::BQ, PLANES = Tile::PLANES, DATA = Tile::DATA, STAGE = Tile::STAGE;
  constexpr int PB = Tile::PB, QB = Tile::QB, SB = Tile::SB;
  constexpr int RP = 1024 / PB, RQ = 1024 / QB, RS = 256 / SB;   // rows of a load
  constexpr int GP = BP / RP, G = GP + PLANES * BQ / RQ;         // loads of a stage: of P, in all
  constexpr int L = G / NW;                                      // a wavefront issues loads wave, wave + NW, ...
  static_assert(GP % NW == 0 && G % NW == 0 && NW % 2 == 0 && BP % RS == 0, "a load's operand is the same in every wavefront");
  constexpr int GS = (BP + BQ) / RS, LS = (GS + NW - 1) / NW;    // loads of scales (some twice where NW does not divide them)
  constexpr int NM = TP * TQ, GROUPS = KB / 64;

  extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
  const int t = threadIdx.x, lane = t & 63, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int wp = wave % WP, wq = wave / WP;

  const int padded = (g.K + 127) & ~127;
  const uint32_t wbytes = (uint32_t)padded / 2, abytes = FA == kMxFp4 ? wbytes : (uint32_t)padded, sbytes = (uint32_t)padded / 32;
  const uint32_t lds0 = (uint32_t)(size_t)(__attribute__((address_space(3))) uint8_t*)smem, wave_lds = lds0 + (uint32_t)wave * 1024;
  // (of a workgroup that stays, whole rounds of the slots: its last stage may hold nothing)
  const int KT = (padded + KB - 1) / KB, stages = Tile::STAYS ? (KT + SLOTS - 1) / SLOTS * SLOTS : KT;

  const int tiles_p = (g.N + BP - 1) / BP;
  const MxGroups<BQ> groups(g);
  const uint32_t count = (uint32_t)tiles_p * (uint32_t)groups.tiles;
  uint32_t id = Tile::STAYS ? blockIdx.x : g.place + blockIdx.x;
  if (id >= count) return;
  struct Place {
    MxRows rows;
    int p0;
  };
  auto place_of = [&](uint32_t id) {
    int tile_p, tile_q;
    panel_tile((int)xcd_run(id, count), tiles_p, groups.tiles, tile_p, tile_q);
    return Place{groups.rows(g, tile_q), tile_p * BP};
  };

  // The rows of a tile's activations that this lane loads, of those the descriptors begin with; negative: none.  Both planes of a row are the same
  // lane's, so one of PLANES loads stands for all.
  constexpr int LQ = (G - GP) / NW / PLANES;
  const int prow_of = lane / (PB / 16), qrow_of = lane / (QB / 16);  // the lane's row of a load
  struct Picked {
    int q[LQ], s[LS];
  };
  auto pick_rows = [&](const Place& at) {
    const int nq = min(at.rows.end - at.rows.row, BQ);
    auto row_of = [&](int r) { return r < nq ? (g.index ? mx_row_of(g, at.rows.row + r) : r) : -1; };
    Picked p;
#pragma unroll
    for (int d = 0; d < LQ; ++d) p.q[d] = row_of((wave + NW * d) * RQ + qrow_of);
#pragma unroll
    for (int d = 0; d < LS; ++d) {
      const int v = (wave + NW * d) % GS * RS + lane / (SB / 4);
      p.s[d] = v >= BP ? row_of(v - BP) : at.p0 + v < g.N ? v : -1;
    }
    return p;
  };

  // A tile's descriptors, and the lane's byte offset of every load: its row's start and its chunk of a stage (the chunk is the same in
  // every load, since every load of a wavefront has the wavefront's parity).
  auto chunk_of = [&](auto bytes, int row) {
    constexpr int B = decltype(bytes)::value;
    return (uint32_t)(((lane % (B / 16)) ^ swz<B>(B == 128 ? (wave & 1) * 8 + row : row)) * 16);
  };
  const uint32_t pck = chunk_of(template_int<PB>{}, prow_of), qck = chunk_of(template_int<QB>{}, qrow_of), sck = (uint32_t)(lane % (SB / 4)) * 4;
  v4i rs_w, rs_ws, rs_a, rs_as;
  uint32_t voff[L], soff[LS];
  auto bind = [&](const Place& at, const Picked& picked) {
    const int np = min(g.N - at.p0, BP), nq = min(at.rows.end - at.rows.row, BQ);
    const int64_t wrow = (int64_t)at.rows.expert * g.N + at.p0, arow = g.index ? 0 : at.rows.row;
    const uint32_t arows = g.index ? (uint32_t)g.a_rows : (uint32_t)nq;
    rs_w = make_rsrc(g.w + wrow * wbytes, (uint32_t)np * wbytes), rs_ws = make_rsrc(g.w_scale + wrow * sbytes, (uint32_t)np * sbytes);
    rs_a = make_rsrc(g.a + arow * abytes, arows * abytes), rs_as = make_rsrc(g.a_scale + arow * sbytes, arows * sbytes);
#pragma unroll
    for (int d = 0; d < L; ++d) {
      if (d < GP / NW) {
        const int r = (wave + NW * d) * RP + prow_of;
        voff[d] = r < np ? (uint32_t)r * wbytes + pck : kOob;
      } else {
        constexpr int kPlane = LQ;  // loads of a plane
        const int e = d - GP / NW, plane = e / kPlane, r = picked.q[e % kPlane];
        voff[d] = r >= 0 ? (uint32_t)r * abytes + qck + (uint32_t)plane * QB : kOob;
      }
    }
#pragma unroll
    for (int d = 0; d < LS; ++d) soff[d] = picked.s[d] >= 0 ? (uint32_t)picked.s[d] * sbytes + sck : kOob;
  };
  constexpr int ISSUES = L + LS;
  // loads lo .. hi - 1 of a stage
  auto issue = [&](int stage, auto slot, auto lo, auto hi) {
    constexpr int base = decltype(slot)::value * STAGE;
    const uint32_t kp = (uint32_t)stage * PB, kq = (uint32_t)stage * (QB * PLANES), ks = (uint32_t)stage * SB;
    const bool there = stage < KT;
    [&]<int... I>(std::integer_sequence<int, I...>) {
      ([&] {
        constexpr int d = decltype(lo)::value + I;
        if constexpr (d < L) {
          constexpr bool isq = d >= GP / NW;
          constexpr int plane = isq && PLANES > 1 ? (d - GP / NW) / LQ : 0;
          const uint32_t at = isq ? kq + plane * QB + qck : kp + pck, end = isq ? abytes : wbytes;
          mx_dma16<base + NW * d * 1024>(isq ? rs_a : rs_w, wave_lds, at < end ? voff[d] : kOob, there ? (isq ? kq : kp) : 0);
        } else {
          constexpr int s = d - L;
          const int grp = (wave + NW * s) % GS;
          mx_dma4<base + DATA>(grp >= BP / RS ? rs_as : rs_ws, lds0 + (uint32_t)grp * 256, ks + sck < sbytes ? soff[s] : kOob, there ? ks : 0);
        }
      }(), ...);
    }(std::make_integer_sequence<int, decltype(hi)::value - decltype(lo)::value>{});
  };
  static_assert(PLANES == 1 || (BQ / RQ) % NW == 0, "a load's plane is the same in every wavefront");
  template_int<0> i0;

  // fragment addresses inside a stage
  const int frow = lane & 31;
  auto chunk_at = [&](auto bytes, int c) { return (c ^ swz<decltype(bytes)::value>(frow & 15)) * 16; };
  template_int<PB> pb;
  template_int<QB> qb;
  const int prow = wp * TP * 32 + frow, qrow = wq * TQ * 32 + frow;
  constexpr int PIECES = FA == kMxFp8 ? 2 : 1;  // 16-byte pieces of a fragment of activations
  int pa[GROUPS], qa[PIECES * GROUPS];
#pragma unroll
  for (int h = 0; h < GROUPS; ++h) {
    pa[h] = prow * PB + chunk_at(pb, 2 * h + half);
    if constexpr (FA == kMxFp4) {
      qa[h] = BP * PB + qrow * QB + chunk_at(qb, 2 * h + half);
    } else {
      qa[2 * h] = BP * PB + ((h / 2) * BQ + qrow) * QB + chunk_at(qb, 4 * (h % 2) + half);
      qa[2 * h + 1] = BP * PB + ((h / 2) * BQ + qrow) * QB + chunk_at(qb, 4 * (h % 2) + 2 + half);
    }
  }
  const int psa = DATA + prow * SB, qsa = DATA + (BP + qrow) * SB, shift = 8 * half;
  mx_v4i pf[2][TP], qf[2][TQ * PIECES];
  uint32_t sc[TP + TQ], sc_next[TP + TQ];  // scales of 128 k; the next ones as they are read
  // read r of the NR of a group's operands, activations first
  constexpr int NR = TQ * PIECES + TP;
  auto read = [&](const uint8_t* base, auto set, auto group, int r) {
    constexpr int S = decltype(set)::value, H = decltype(group)::value;
    if (r < TQ * PIECES) qf[S][r] = *reinterpret_cast<const mx_v4i*>(base + qa[PIECES * H + r % PIECES] + (r / PIECES) * 32 * QB);
    else pf[S][r - TQ * PIECES] = *reinterpret_cast<const mx_v4i*>(base + pa[H] + (r - TQ * PIECES) * 32 * PB);
  };
  auto read_scale = [&](const uint8_t* base, int part, int r) {
    sc_next[r] = *reinterpret_cast<const uint32_t*>(base + (r < TP ? psa + r * 32 * SB : qsa + (r - TP) * 32 * SB) + 4 * part);
  };
  auto shift_scales = [&] {
#pragma unroll
    for (int r = 0; r < TP + TQ; ++r) sc[r] = sc_next[r] >> shift;
  };
  // Group H of a stage: multiply its set of fragments, behind the instructions go the reads of the next group's set (from `next`) and of
  // the next 128 k's scales in front of them, and in the last group the loads of stage `dma_stage`.
  auto multiply = [&](mx_v16f (&acc)[TP][TQ], auto hconst, const uint8_t* next, int dma_stage, auto ring) {
    constexpr int H = decltype(hconst)::value, S = H & 1;
    mx_v8i q_high, q_low;
    constexpr int reads = NR + (H % 2 ? TP + TQ : 0), each = (reads + NM - 1) / NM > 2 ? (reads + NM - 1) / NM : 2;
    [&]<int... Mi>(std::integer_sequence<int, Mi...>) {
      ([&] {
        constexpr int m = Mi, j = m / TP, i = m % TP;
        const mx_v4i p4 = pf[S][i], q4 = qf[S][j * PIECES], q5 = qf[S][j * PIECES + PIECES - 1];
        const mx_v8i p = __builtin_shufflevector(p4, p4, 0, 1, 2, 3, -1, -1, -1, -1);
        mx_v8i q;
        if constexpr (FA == kMxFp4) q = __builtin_shufflevector(q4, q4, 0, 1, 2, 3, -1, -1, -1, -1);
        else q = __builtin_shufflevector(q4, q5, 0, 1, 2, 3, 4, 5, 6, 7);
        if constexpr (SPLIT) {
          if constexpr (i == 0) mx_split8(q, q_high, q_low);
          q = q_high;
        }
        const auto add = [&](const mx_v8i& part) {
          acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(p, part, acc[i][j], kMxMfmaFormat<kMxFp4>, kMxMfmaFormat<FA>, 2 * (H % 2), (int)sc[i],
                                                                      2 * (H % 2), (int)sc[TP + j]);
        };
        add(q);
        if constexpr (SPLIT) add(q_low);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int r = each * m; r < each * m + each && r < reads; ++r) {
          if (r < NR) read(next, template_int<(S ^ 1)>{}, template_int<(H + 1) % GROUPS>{}, r);
          else read_scale(next, (H + 1) % GROUPS / 2, r - NR);
        }
        if constexpr (H == GROUPS - 1) issue(dma_stage, ring, template_int<m * ISSUES / NM>{}, template_int<(m + 1) * ISSUES / NM>{});
        __builtin_amdgcn_sched_barrier(0);
      }(), ...);
    }(std::make_integer_sequence<int, NM>{});
    if constexpr (H % 2 != 0) shift_scales();
  };
  constexpr int kStores16 = TQ * TP / 2 * 4, kStores32 = 2 * kStores16;
  int stores = 0;  // of the last tile's results, behind the loads of this one's first two stages
  bool first = true, more = false;
  // Before a stage's last group: the next stage has landed (the stores behind it need not have), and every wavefront is done with this one's slot.
  auto meet = [&](int kt) {
    if (Tile::STAYS && kt == 0 && stores == kStores16) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kStores16) : "memory");
    else if (Tile::STAYS && kt == 0 && stores == kStores32) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kStores32) : "memory");
    else asm volatile("s_waitcnt vmcnt(%0)" ::"n"((SLOTS - 2) * ISSUES) : "memory");
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  // the stage that goes into a stage's slot behind it (stages behind the last one are the next tile's)
  auto fetched = [&](int kt) { return Tile::STAYS && more && kt + SLOTS >= stages ? kt + SLOTS - stages : kt + SLOTS; };
  auto stage_body = [&](mx_v16f (&acc)[TP][TQ], int kt, auto ring) {
    constexpr int R = decltype(ring)::value;
    const uint8_t* here = smem + R * STAGE;
    const uint8_t* other = smem + (R + 1) % SLOTS * STAGE;
    [&]<int... H>(std::integer_sequence<int, H...>) { (multiply(acc, template_int<H>{}, here, 0, ring), ...); }(std::make_integer_sequence<int, GROUPS - 1>{});
    meet(kt);
    multiply(acc, template_int<GROUPS - 1>{}, other, fetched(kt), ring);
  };
  // a stage of which nothing is this wavefront's
  auto idle_stage = [&](int kt, auto ring) {
    meet(kt);
    issue(fetched(kt), ring, i0, template_int<ISSUES>{});
  };

  auto by_type = [&](const auto& f) {
    if constexpr (SPLIT) f.template operator()<kMxF32>();
    else if (FA == kMxFp4 && g.type == kMxF32) f.template operator()<kMxF32>();
    else if (g.type == kMxBf16) f.template operator()<kMxBf16>();
    else f.template operator()<kMxF16>();
  };

  Place here = place_of(id);
  bind(here, pick_rows(here));
  [&]<int... I>(std::integer_sequence<int, I...>) { (issue(I, template_int<I>{}, i0, template_int<ISSUES>{}), ...); }(std::make_integer_sequence<int, SLOTS>{});
  static_assert(SLOTS * ISSUES <= 63, "loads that can be counted");
  for (;;) {
    // the next tile's rows are looked up now and used when this one's loads have all gone out
    more = Tile::STAYS && id + g.place < count;
    Place next = here;
    Picked picked;
    if (more) next = place_of(id + g.place);
    if (more) picked = pick_rows(next);
    auto bind_next = [&](int kt) {
      if (more && kt + SLOTS >= stages) bind(next, picked);
    };
    auto start = [&] {
      if (first) asm volatile("s_waitcnt vmcnt(%0)" ::"n"((SLOTS - 1) * ISSUES) : "memory");  // stage 0 (of a later tile: waited for in the last stage)
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
    };
    auto drain = [&] {  // (the stages beyond K have to land before the slots are used for something else)
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();
    };
    auto round = [&](int kt, int end, const auto& body) {  // stages kt .. end - 1, at most one a slot
      [&]<int... I>(std::integer_sequence<int, I...>) {
        ([&] {
          if (I == 0 || kt + I < end) body(kt + I, template_int<I>{});
        }(), ...);
      }(std::make_integer_sequence<int, SLOTS>{});
    };
    const int n0 = here.p0 + wp * TP * 32, nq = min(here.rows.end - here.rows.row, BQ);
    // A wavefront that has none of a ragged tile's rows or features loads and waits with the others, no more.  (Its way and the others' part
    // before there are sums: where they meet with sums in registers, the compiler keeps two sets of them.)
    if (wq * TQ * 32 >= nq || n0 >= g.N) {
      start();
      for (int kt = 0; kt < stages; kt += SLOTS) {
        bind_next(kt);
        round(kt, stages, idle_stage);
      }
      if (Tile::BY_LDS) drain();
    } else {
      // the sums start from the bias (of features beyond the last one, which nobody stores: the last one's)
      mx_v16f acc[TP][TQ];
      if (g.bias) {
        const float* bias = g.bias + (int64_t)here.rows.expert * g.N;
#pragma unroll
        for (int i = 0; i < TP; ++i)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const float b = bias[min(n0 + i * 32 + 8 * (r / 4) + 4 * half + r % 4, g.N - 1)];
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
      start();
#pragma unroll
      for (int r = 0; r < NR; ++r) read(smem, i0, i0, r);
#pragma unroll
      for (int r = 0; r < TP + TQ; ++r) read_scale(smem, 0, r);
      shift_scales();
      auto work = [&](int kt, auto ring) { stage_body(acc, kt, ring); };
      for (int kt = 0; kt < KT; kt += SLOTS) {
        bind_next(kt);
        round(kt, KT, work);
      }
      if constexpr (Tile::BY_LDS) {
        drain();
        uint8_t* mine = smem + wave * 32 * Tile::PITCH;
        by_type([&]<int TYPE>() { leave_by_lds<TYPE, TP, TQ>(g, acc, here.rows.row, wq * TQ * 32, nq, n0, lane, mine); });
      } else {
        if (KT < stages) idle_stage(KT, template_int<1>{});
        by_type([&]<int TYPE>() { leave_by_quads<TYPE, TP, TQ>(g, acc, here.rows.row, wq * TQ * 32, nq, n0, lane); });
      }
    }
    if (!more) break;
    // (every lane of a whole tile stores, so that the stores can be counted)
    stores = nq == BQ && n0 + TP * 32 <= g.N ? (g.type == kMxF32 ? kStores32 : kStores16) : 0;
    first = false;
    id += g.place;
    here = next;
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // (nothing may be on its way into LDS that is given back)
}

template <int FA, int WP, int WQ, int TP, int TQ, int SLOTS, int KB, bool SPLIT>
hipError_t launch_tile(const MxGemmArgs& g, hipStream_t st) {
  using Tile = MxTile<FA, WP, WQ, TP, TQ, SLOTS, KB>;
  const auto kern = mx_tile_kernel<FA, WP, WQ, TP, TQ, SLOTS, KB, SPLIT>;
  static std::atomic<uint64_t> attr_set{0};  // the devices whose dynamic-LDS limit is raised
  const hipError_t e = raise_lds_limit(reinterpret_cast<const void*>(kern), Tile::LDS, attr_set);
  if (e != hipSuccess) return e;
  const int64_t tiles_q = g.offsets ? mx_most_tiles(g.T, g.experts, Tile::BQ) : (g.T + Tile::BQ - 1) / Tile::BQ;
  const int64_t tiles = (int64_t)((g.N + Tile::BP - 1) / Tile::BP) * tiles_q;
  const int64_t resident = tiles < 256 * Tile::RESIDENT ? tiles : 256 * Tile::RESIDENT;
  if (Tile::STAYS) return launch_mx_at(kern, resident, (uint32_t)resident, Tile::NT, Tile::LDS, st, g);
  return launch_mx_tiles(kern, tiles, Tile::NT, Tile::LDS, st, g);
}

}  // namespace

}  // namespace hago
