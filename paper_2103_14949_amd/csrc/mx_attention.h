// What the kernels of the attention over a paged cache of microscaled keys and values have in common.
//
// Keys and values go into the matrix instructions as bfloat16 (values as float16 where the kernel for many rows says so), which holds every code times its scale (three bits of mantissa, the
// exponents of binary32; below 2^-126 it may be zero); queries as one, two or three bfloat16 numbers that add up to theirs (bfloat16, float16, binary32), and probabilities
// as each kernel says.  Sums are binary32.
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
  uint32_t* plan;   // NULL, or [seqs + 1][2]: keys of a run in blocks, then runs and partials of all sequences up to each
};

// Sums over the lanes up to each.
__device__ __forceinline__ uint32_t attention_scan(uint32_t v) {
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x111, 0xf, 0xf, true);   // row_shr:1
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x112, 0xf, 0xf, true);   // row_shr:2
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x114, 0xf, 0xf, true);   // row_shr:4
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x118, 0xf, 0xf, true);   // row_shr:8
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x142, 0xa, 0xf, false);  // row_bcast:15, into the odd rows
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x143, 0xc, 0xf, false);  // row_bcast:31, into the last two
  return v;
}

// A workgroup's run of keys.
struct AttentionRun {
  int seq, local, runs, slot;  // place among the sequence's runs, runs of a unit, first partial of the sequence (-1: none)
};

// A sequence's units (ROWS rows, head) and their keys in blocks of BLOCK; none behind the last sequence.
template <int ROWS, int BLOCK>
__device__ __forceinline__ void attention_units(const CacheArgs& c, const AttentionArgs& a, uint32_t group, int seq, AttentionSpan& span, uint32_t& units, uint32_t& blocks) {
  units = 0, blocks = 1;
  if (seq >= c.seqs) return;
  span = attention_span(c, a, seq);
  units = ((uint32_t)span.rows * group + ROWS - 1) / ROWS * c.kv_heads;
  if (span.high > span.low) blocks = (uint32_t)(span.high - (span.low & ~15) + BLOCK - 1) / BLOCK;
}
template <int SHARES>
__device__ __forceinline__ uint32_t attention_share(uint64_t all) {
  static_assert((SHARES & (SHARES - 1)) == 0);
  const uint64_t wide = (all + SHARES - 1) / SHARES;
  return __builtin_amdgcn_readfirstlane(wide > 0x7fffffffu ? 0x7fffffffu : wide ? (uint32_t)wide : 1);
}

// Units are cut into ceil(blocks / share) runs, such that there are about SHARES of them: at most
// that many and as many as units, and of those of units that are cut at most twice as many.  Every wavefront finds the run for itself, 64 sequences
// at a time, or in the plan that a launch in front has made of many sequences; the sequence's rows and keys come with it.  (Offsets that break the
// contract can make counts wrap: what is found then is still inside its sequence.)
template <int ROWS, int BLOCK, int SHARES>
__device__ __forceinline__ bool attention_run(const CacheArgs& c, const AttentionArgs& a, const AttentionWork& work, uint32_t group, uint32_t id, AttentionRun& run,
                                              AttentionSpan& span) {
  const int lane = threadIdx.x & 63;
  if (work.plan) {
    const uint32_t* const ends = work.plan + 2;
    int low = 0, high = c.seqs;  // the first sequence whose runs end behind id is among them, if it is any
    while (high - low > 1) {
      const int step = (high - low + 63) / 64, at = low + (lane + 1) * step - 1 < high ? low + (lane + 1) * step - 1 : high - 1;
      const uint64_t behind = __ballot(ends[2 * (int64_t)at] > id);
      if (!behind) return false;
      const int first = __builtin_ctzll(behind), from = low + first * step;
      high = from + step < high ? from + step : high;
      low = from;
    }
    low = __builtin_amdgcn_readfirstlane(low);
    const uint32_t before = low ? ends[2 * (int64_t)low - 2] : 0, slots_before = low ? ends[2 * (int64_t)low - 1] : 0, share = work.plan[0];
    uint32_t units, blocks;
    AttentionSpan found;
    attention_units<ROWS, BLOCK>(c, a, group, low, found, units, blocks);
    const uint32_t runs = blocks > share ? (blocks + share - 1) / share : 1, local = id - before;
    if (__builtin_amdgcn_readfirstlane(local >= units * runs)) return false;
    run.seq = low;
    run.local = (int)__builtin_amdgcn_readfirstlane(local);
    run.runs = (int)__builtin_amdgcn_readfirstlane(runs);
    run.slot = run.runs > 1 ? (int)__builtin_amdgcn_readfirstlane(slots_before) : -1;
    span.first = __builtin_amdgcn_readfirstlane(found.first);
    span.rows = __builtin_amdgcn_readfirstlane(found.rows);
    span.low = __builtin_amdgcn_readfirstlane(found.low);
    span.high = __builtin_amdgcn_readfirstlane(found.high);
    const uint32_t below = __builtin_amdgcn_readfirstlane((uint32_t)found.position), above = __builtin_amdgcn_readfirstlane((uint32_t)((uint64_t)found.position >> 32));
    span.position = (int64_t)((uint64_t)above << 32 | below);
    return true;
  }
  AttentionSpan mine{};  // of this lane's sequence
  uint32_t units = 0, blocks = 1;
  uint64_t all = 0;
  for (int s = 0; s < c.seqs; s += 64) {
    attention_units<ROWS, BLOCK>(c, a, group, s + lane, mine, units, blocks);
    all += (uint64_t)units * blocks;
  }
  if (c.seqs > 1)
#pragma unroll
    for (int d = 1; d < 64; d *= 2) all += __shfl_xor(all, d);
  const uint32_t share = attention_share<SHARES>(all);
  uint32_t before = 0, slots_before = 0;
  for (int s = 0; s < c.seqs; s += 64) {
    if (c.seqs > 64) attention_units<ROWS, BLOCK>(c, a, group, s + lane, mine, units, blocks);
    const uint32_t runs = blocks > share ? (blocks + share - 1) / share : 1, count = units * runs, cut = runs > 1 ? count : 0;
    const uint32_t upto = attention_scan(count), slots_upto = attention_scan(cut);
    const uint64_t found = __ballot(id - before - (upto - count) < count);
    if (found) {
      const int at = __builtin_ctzll(found);
      run.seq = s + at;
      run.local = (int)(id - before - __builtin_amdgcn_readlane(upto - count, at));
      run.runs = (int)__builtin_amdgcn_readlane(runs, at);
      run.slot = run.runs > 1 ? (int)(slots_before + __builtin_amdgcn_readlane(slots_upto - cut, at)) : -1;
      span.first = __builtin_amdgcn_readlane(mine.first, at);
      span.rows = __builtin_amdgcn_readlane(mine.rows, at);
      span.low = __builtin_amdgcn_readlane(mine.low, at);
      span.high = __builtin_amdgcn_readlane(mine.high, at);
      const uint32_t below = __builtin_amdgcn_readlane((uint32_t)mine.position, at), above = __builtin_amdgcn_readlane((uint32_t)((uint64_t)mine.position >> 32), at);
      span.position = (int64_t)((uint64_t)above << 32 | below);
      return true;
    }
    before += __builtin_amdgcn_readlane(upto, 63);
    slots_before += __builtin_amdgcn_readlane(slots_upto, 63);
  }
  return false;
}

namespace {  // (a kernel of its own in every file)

// The plan of more sequences than every wavefront should look at, by one workgroup.
constexpr int kPlanThreads = 1024;
template <int ROWS, int BLOCK, int SHARES>
__global__ __launch_bounds__(kPlanThreads) void plan_kernel(CacheArgs c, AttentionArgs a, uint32_t* plan, uint32_t group) {
  constexpr int kPlanWaves = kPlanThreads / 64;
  __shared__ uint64_t totals[kPlanWaves];
  __shared__ uint2 counts[kPlanWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid / 64;
  AttentionSpan span;
  uint32_t units, blocks;
  uint64_t all = 0;
  for (int64_t s = tid; s < c.seqs; s += kPlanThreads) {
    attention_units<ROWS, BLOCK>(c, a, group, (int)s, span, units, blocks);
    all += (uint64_t)units * blocks;
  }
#pragma unroll
  for (int d = 1; d < 64; d *= 2) all += __shfl_xor(all, d);
  if (lane == 0) totals[wave] = all;
  __syncthreads();
  all = 0;
  for (int w = 0; w < kPlanWaves; ++w) all += totals[w];
  const uint32_t share = attention_share<SHARES>(all);
  if (tid == 0) plan[0] = share;
  uint32_t before = 0, slots_before = 0;
  for (int64_t base = 0; base < c.seqs; base += kPlanThreads) {
    const int64_t s = base + tid;
    attention_units<ROWS, BLOCK>(c, a, group, s < c.seqs ? (int)s : c.seqs, span, units, blocks);
    const uint32_t runs = blocks > share ? (blocks + share - 1) / share : 1, count = units * runs, cut = runs > 1 ? count : 0;
    const uint32_t upto = attention_scan(count), slots_upto = attention_scan(cut);
    if (lane == 63) counts[wave] = make_uint2(upto, slots_upto);
    __syncthreads();
    uint32_t earlier = before, slots_earlier = slots_before;
    for (int w = 0; w < kPlanWaves; ++w) {
      const uint2 n = counts[w];
      if (w < wave) earlier += n.x, slots_earlier += n.y;
      before += n.x, slots_before += n.y;
    }
    if (s < c.seqs) plan[2 + 2 * s] = earlier + upto, plan[3 + 2 * s] = slots_earlier + slots_upto;
    __syncthreads();
  }
}
template <int ROWS, int BLOCK, int SHARES>
hipError_t launch_plan(const CacheArgs& c, const AttentionArgs& a, const AttentionWork& work, hipStream_t st) {
  if (!work.plan) return hipSuccess;
  return launch_kernel(plan_kernel<ROWS, BLOCK, SHARES>, dim3(1), dim3(kPlanThreads), 0, st, c, a, work.plan, (uint32_t)(a.heads / c.kv_heads));
}

}  // namespace

// A lane's part of a key or value: 8 DB codes.
template <int FORMAT, int DB>
struct AttentionChunk {
  static constexpr int kWords = FORMAT == kMxFp4 ? DB : 2 * DB;
  static constexpr int kScales = DB == 8 ? 2 : 1;
  static constexpr int kRowWords = FORMAT == kMxFp4 ? 4 : 8;  // of a block
  static constexpr int kPiece = kWords < 4 ? kWords : 4;      // of a load
  uint32_t w[kWords];
  uint32_t scale[kScales];

  // Bytes from a row's first code, and block from its first, of load i.  Where a row has fewer blocks than the kernel is made for, those behind its end are
  // others of its own: queries are zero there, and results are not kept.
  static __device__ __forceinline__ uint32_t code_at(int blocks, int part, int i) {
    const int at = part * kWords + i * kPiece, most = blocks * kRowWords - kPiece;
    return 4 * (at < most ? at : most);
  }
  static __device__ __forceinline__ uint32_t scale_at(int blocks, int part, int i) {
    const int block = part * DB / 4 + i;
    return block < blocks ? block : blocks - 1;
  }
  static constexpr int kLoads = kWords / kPiece;
  // codes and scales of a row (any that there is), `code` and `scale_of` as above.  WORDS: scale_of are those of the words that the scales lie in; each is one only
  // after `unpack` with its place there.  (A byte of a loop's next round is extended, and waited for, where it is loaded.)
  template <bool WORDS>
  __device__ __forceinline__ void load(const uint8_t* codes, const uint8_t* scales, const uint32_t (&code)[kLoads], const uint32_t (&scale_of)[kScales]) {
    typedef uint32_t piece __attribute__((ext_vector_type(kPiece)));
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const piece p = *reinterpret_cast<const piece*>(codes + code[i]);
#pragma unroll
      for (int k = 0; k < kPiece; ++k) w[i * kPiece + k] = p[k];
    }
#pragma unroll
    for (int i = 0; i < kScales; ++i) scale[i] = WORDS ? *reinterpret_cast<const uint32_t*>(scales + scale_of[i]) : scales[scale_of[i]];
  }
  __device__ __forceinline__ void unpack(const uint32_t (&shift)[kScales]) {
#pragma unroll
    for (int i = 0; i < kScales; ++i) scale[i] = scale[i] >> shift[i] & 255;
  }
  // eight codes of step st, and 2^up times their scale
  __device__ __forceinline__ const uint32_t* words(int st) const { return w + st * (FORMAT == kMxFp4 ? 1 : 2); }
  __device__ __forceinline__ float scale_of(int st, int up) const { return __builtin_bit_cast(float, (scale[st / 4 % kScales] + up) << 23); }
  __device__ __forceinline__ at_b8 values(int st) const { return attention_values8<FORMAT>(words(st), scale_of(st, 0)); }
};

// Host side: blocks of 32 columns that the kernels are made for, and what the kernel for many rows has of rows and runs.
constexpr int attention_blocks(int64_t dim) { return dim <= 64 ? 2 : dim <= 128 ? 4 : 8; }
// (two wavefronts a SIMD where 256 registers do)
constexpr int attention_many_waves(int type, int db) { return type == kMxBf16 && db != 8 ? 8 : 4; }
constexpr int attention_many_rows(int type, int db) { return 32 * attention_many_waves(type, db); }
constexpr int kAttentionManyRuns = 256;
// Whether a wavefront's `keys` neighbours, the first at a multiple of their number, lie in one page, and their scales in words of 32 bits that are the cache's.
inline bool attention_even(const CacheArgs& c, int keys) { return c.page % keys == 0 && ptr_aligned(c.k_scales, 4) && ptr_aligned(c.v_scales, 4); }
hipError_t launch_attention_many_bf16(const CacheArgs& c, const AttentionArgs& a, const AttentionWork& work, hipStream_t st);
hipError_t launch_attention_many_f16(const CacheArgs& c, const AttentionArgs& a, const AttentionWork& work, hipStream_t st);

constexpr float kAttentionLog2e = 1.44269504f, kAttentionLn2 = 0.693147181f;

}  // namespace hago
