// What the kernels of the attention over a paged cache of microscaled keys and values have in common.
//
// Keys and values go into the matrix instructions as bfloat16, which holds every code times its scale (three bits of mantissa, the
// exponents of binary32; below 2^-126 it may be zero); queries and probabilities as one, two or three bfloat16 numbers that add up to
// theirs: bfloat16 queries are held by one, float16 by two, binary32 by three.  Sums are binary32.
#pragma once

#include "mx_cache_device.h"

namespace hago {

typedef __bf16 at_b2 __attribute__((ext_vector_type(2)));
typedef __bf16 at_b8 __attribute__((ext_vector_type(8)));
typedef short at_s4 __attribute__((ext_vector_type(4)));
typedef float at_f4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) at_s4 at_lds_s4;

template <int TYPE>
constexpr int kAttentionPieces = TYPE == kMxBf16 ? 1 : TYPE == kMxF16 ? 2 : 3;

// One sequence's rows and keys in this call.
struct AttentionSpan {
  int32_t first, rows;    // tokens of the call
  int64_t position;       // of the first one
  int32_t low, high;      // keys that any of them can see
};
__device__ __forceinline__ AttentionSpan attention_span(const CacheArgs& c, const AttentionArgs& a, int seq) {
  AttentionSpan s;
  const int32_t b = c.offsets[seq], e = c.offsets[seq + 1], length = c.lengths[seq];
  s.first = b < 0 ? 0 : b;
  const int32_t end = e > a.T ? a.T : e;
  s.rows = end > s.first ? end - s.first : 0;
  s.position = (int64_t)length - ((int64_t)e - s.first);
  s.high = length < 0 ? 0 : length < c.places ? length : c.places;
  const int64_t low = a.window ? s.position - a.window + 1 : 0;
  s.low = low < 0 ? 0 : low < s.high ? (int32_t)low : s.high;
  return s;
}

// Eight codes of a block as bfloat16: dwords `w` (fp8: two, fp4: one), scale 2^(byte - 127).
template <int FORMAT>
__device__ __forceinline__ at_b8 attention_values8(const uint32_t* w, float scale) {
  at_b2 d[4];
  if constexpr (FORMAT == kMxFp4) {
    d[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[0], scale, 0);
    d[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[0], scale, 1);
    d[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[0], scale, 2);
    d[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[0], scale, 3);
  } else {
    d[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[0], scale, false);
    d[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[0], scale, true);
    d[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[1], scale, false);
    d[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[1], scale, true);
  }
  at_b8 v;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = d[i / 2][i % 2];
  return v;
}

// x as PIECES bfloat16 numbers, the largest first.
template <int PIECES>
__device__ __forceinline__ void attention_split(float x, __bf16 (&p)[PIECES]) {
#pragma unroll
  for (int i = 0; i < PIECES; ++i) {
    p[i] = (__bf16)x;
    if (i + 1 < PIECES) x -= (float)p[i];
  }
}

struct AttentionWork {
  float* partial;   // [slots][rows of a tile][32 DB]
  float2* stats;    // [slots][rows of a tile]: maximum and sum
  int2* joins;      // [T][heads]: the row of the first of its partials, number of partials
};

template <int WAVES>
__device__ __forceinline__ int64_t attention_scan(int64_t v, int64_t* totals, int64_t& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x / 64;
  int64_t sum = v;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int64_t other = __shfl_up(sum, d);
    if (lane >= d) sum += other;
  }
  if (lane == 63) totals[wave] = sum;
  __syncthreads();
  total = 0;
  int64_t before = 0;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    if (w < wave) before += totals[w];
    total += totals[w];
  }
  __syncthreads();
  return before + sum - v;
}

// A workgroup's run of keys.
struct AttentionRun {
  int seq, local, runs, slot;  // place among the sequence's runs, runs of a unit, first partial of the sequence (-1: none)
};

// Units are (ROWS rows, head); each is cut into ceil(blocks / share) runs, a block being BLOCK keys, such that there are about `share_of` of them: at most
// that many and as many as units, and of those of units that are cut at most twice as many.
template <int THREADS, int ROWS, int BLOCK>
__device__ __forceinline__ bool attention_run(const CacheArgs& c, const AttentionArgs& a, int group, int share_of, int64_t id, AttentionRun& run) {
  __shared__ int64_t totals[THREADS / 64];
  __shared__ AttentionRun found;
  const int tid = threadIdx.x;
  const auto sizes = [&](int s, int64_t& units, int64_t& blocks) {
    units = 0, blocks = 0;
    if (s >= c.seqs) return;
    const AttentionSpan span = attention_span(c, a, s);
    units = ((int64_t)span.rows * group + ROWS - 1) / ROWS * c.kv_heads;
    blocks = span.high > span.low ? (span.high - (span.low & ~15) + BLOCK - 1) / BLOCK : 1;
  };
  int64_t units, blocks, all = 0;
  for (int s = 0; s < c.seqs; s += THREADS) {
    int64_t total;
    sizes(s + tid, units, blocks);
    attention_scan<THREADS / 64>(units * blocks, totals, total);
    all += total;
  }
  const int64_t share = all > share_of ? (all + share_of - 1) / share_of : 1;
  if (tid == 0) found.seq = -1;
  int64_t before = 0, slots_before = 0;
  for (int s = 0; s < c.seqs; s += THREADS) {
    if (c.seqs > THREADS) sizes(s + tid, units, blocks);
    const int64_t runs = (blocks + share - 1) / share;
    // (both counts below 2^31)
    int64_t total;
    const int64_t at = attention_scan<THREADS / 64>(units * runs << 32 | (runs > 1 ? units * runs : 0), totals, total);
    const int64_t first = before + (at >> 32);
    if (id >= first && id < first + units * runs)
      found = AttentionRun{s + tid, (int)(id - first), (int)runs, runs > 1 ? (int)(slots_before + (at & 0xffffffff)) : -1};
    before += total >> 32;
    slots_before += total & 0xffffffff;
    if (before > id) break;
  }
  __syncthreads();
  run = found;
  // (the same in all lanes, which the compiler does not know of what lies in LDS)
  run.seq = __builtin_amdgcn_readfirstlane(run.seq);
  run.local = __builtin_amdgcn_readfirstlane(run.local);
  run.runs = __builtin_amdgcn_readfirstlane(run.runs);
  run.slot = __builtin_amdgcn_readfirstlane(run.slot);
  return run.seq >= 0;
}

// A lane's part of a key or value: 8 DB codes.
template <int FORMAT, int DB>
struct AttentionChunk {
  static constexpr int kWords = FORMAT == kMxFp4 ? DB : 2 * DB;
  static constexpr int kScales = DB == 8 ? 2 : 1;
  static constexpr int kRowWords = FORMAT == kMxFp4 ? 4 : 8;  // of a block
  static constexpr int kPiece = kWords < 4 ? kWords : 4;      // of a load
  uint32_t w[kWords];
  uint32_t scale[kScales];

  // Of any row that there is.  Where a row has fewer blocks than DB, the pieces behind its end are others of its own: queries are zero there, and
  // results are not kept.
  __device__ __forceinline__ void load(const uint8_t* codes, const uint8_t* scales, int64_t place, int blocks, int part) {
    typedef uint32_t piece __attribute__((ext_vector_type(kPiece)));
    const uint32_t* row = reinterpret_cast<const uint32_t*>(codes) + place * (blocks * kRowWords);
#pragma unroll
    for (int i = 0; i < kWords; i += kPiece) {
      const int at = part * kWords + i, most = blocks * kRowWords - kPiece;
      const piece p = *reinterpret_cast<const piece*>(row + (at < most ? at : most));
#pragma unroll
      for (int k = 0; k < kPiece; ++k) w[i + k] = p[k];
    }
#pragma unroll
    for (int i = 0; i < kScales; ++i) {
      const int block = part * DB / 4 + i;
      scale[i] = scales[place * blocks + (block < blocks ? block : blocks - 1)];
    }
  }
  // eight codes of step st
  __device__ __forceinline__ at_b8 values(int st) const {
    return attention_values8<FORMAT>(w + st * (FORMAT == kMxFp4 ? 1 : 2), __builtin_bit_cast(float, scale[st / 4 % kScales] << 23));
  }
};

// Host side: blocks of 32 columns that the kernels are made for, and what the kernel for many rows has of rows and runs.
constexpr int attention_blocks(int64_t dim) { return dim <= 64 ? 2 : dim <= 128 ? 4 : 8; }
template <int DB>
constexpr int kManyWaves = DB == 8 ? 4 : 8;
constexpr int attention_many_rows(int db) { return 32 * (db == 2 ? kManyWaves<2> : db == 4 ? kManyWaves<4> : kManyWaves<8>); }
constexpr int kAttentionManyRuns = 256;
hipError_t launch_attention_many(const CacheArgs& c, const AttentionArgs& a, const AttentionWork& work, hipStream_t st);

constexpr float kAttentionLog2e = 1.44269504f, kAttentionLn2 = 0.693147181f;

}  // namespace hago
