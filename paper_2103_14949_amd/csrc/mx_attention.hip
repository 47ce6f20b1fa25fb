// Attention over a paged cache of microscaled keys and values, few rows a sequence: the form for single tokens, and the one that is
// right for every call.
//
// out = softmax(scale * q k^T) v in one pass over the keys with the running maximum and sum.  The cache's bytes bound it, so a
// workgroup is one (sequence, 16 rows, head of the cache) and a run of keys, its rows the queries of all heads that share those keys;
// the runs are as long as makes all workgroups' work alike, whatever the lengths, and a second launch joins the sequences that were cut.
// Lengths stay on the device: every workgroup finds its run by a scan over the sequences.
//
// A wavefront goes its own way through 32 keys at a time, with no barrier.  S^T = K Q^T: a lane (key r = lane % 16, part h = lane / 16)
// loads part h of key r, which is whole in one block of 32 (or two) and becomes the operand by eight conversions.  Its results are keys
// 4 h .. 4 h + 3 of query r, which is the operand of O^T = V^T P^T as it stands, if V^T's lanes hold the same keys; they read them so from
// LDS, 4 x 16 elements at a time transposed.
#include "mx_attention.h"

namespace hago {

namespace {

constexpr int kThreads = 256, kWaves = 4, kKeys = 32, kBlock = kWaves * kKeys;
// Workgroups that share the keys, by blocks of a row: as many as are resident.
template <int DB>
constexpr int kRuns = DB == 8 ? 512 : 1024;
constexpr int kMostRuns = 1024;

struct AttentionWork {
  float* partial;   // [2 kRuns][16][32 DB]
  float2* stats;    // [2 kRuns][16]: maximum and sum
  int2* joins;      // [T][heads]: 16 * first partial + row, number of partials
};

__device__ __forceinline__ int64_t scan_within_block(int64_t v, int64_t* totals, int64_t& total) {
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
  for (int w = 0; w < kWaves; ++w) {
    if (w < wave) before += totals[w];
    total += totals[w];
  }
  __syncthreads();
  return before + sum - v;
}

// A workgroup's run.
struct Run {
  int seq, local, runs, slot;  // place among the sequence's runs, runs of a unit, first partial of the sequence (-1: none)
};

// Units are (16 rows, head); each is cut into ceil(blocks / share) runs.
__device__ __forceinline__ bool find_run(const CacheArgs& c, const AttentionArgs& a, int group, int share_of, int64_t id, Run& run) {
  __shared__ int64_t totals[kWaves];
  __shared__ Run found;
  const int tid = threadIdx.x;
  const auto sizes = [&](int s, int64_t& units, int64_t& blocks) {
    units = 0, blocks = 0;
    if (s >= c.seqs) return;
    const AttentionSpan span = attention_span(c, a, s);
    units = ((int64_t)span.rows * group + 15) / 16 * c.kv_heads;
    blocks = span.high > span.low ? (span.high - (span.low & ~15) + kBlock - 1) / kBlock : 1;
  };
  int64_t units, blocks, all = 0;
  for (int s = 0; s < c.seqs; s += kThreads) {
    int64_t total;
    sizes(s + tid, units, blocks);
    scan_within_block(units * blocks, totals, total);
    all += total;
  }
  const int64_t share = all > share_of ? (all + share_of - 1) / share_of : 1;
  if (tid == 0) found.seq = -1;
  int64_t before = 0, slots_before = 0;
  for (int s = 0; s < c.seqs; s += kThreads) {
    if (c.seqs > kThreads) sizes(s + tid, units, blocks);
    const int64_t runs = (blocks + share - 1) / share;
    // (both counts below 2^31)
    int64_t total;
    const int64_t at = scan_within_block(units * runs << 32 | (runs > 1 ? units * runs : 0), totals, total);
    const int64_t first = before + (at >> 32);
    if (id >= first && id < first + units * runs)
      found = Run{s + tid, (int)(id - first), (int)runs, runs > 1 ? (int)(slots_before + (at & 0xffffffff)) : -1};
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
struct Chunk {
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

__device__ __forceinline__ float max_of_parts(float v) {
  v = fmaxf(v, __shfl_xor(v, 16));
  return fmaxf(v, __shfl_xor(v, 32));
}
__device__ __forceinline__ float sum_of_parts(float v) {
  v += __shfl_xor(v, 16);
  return v + __shfl_xor(v, 32);
}

template <int TYPE, int KF, int VF, int DB>
__global__ __launch_bounds__(kThreads, TYPE != kMxBf16 && DB == 8 ? 1 : 2) void attention_kernel(CacheArgs c, AttentionArgs a, AttentionWork work, int group) {
  using E = typename MxElement<TYPE>::type;
  constexpr int PIECES = kAttentionPieces<TYPE>, D = 32 * DB;
  constexpr int kRow = 2 * D + 32;                          // bytes of a row of values in LDS: 4 x 16 elements of it fall on different banks
  constexpr int kSums = D + 4;                              // floats of a row of results there
  constexpr int kRegion = kKeys * kRow;                     // of a wavefront
  static_assert(16 * kSums * 4 + 128 <= kRegion);
  __shared__ __align__(16) uint8_t lds[kWaves * kRegion];

  Run run;
  if (!find_run(c, a, group, kRuns<DB>, blockIdx.x, run)) return;
  const AttentionSpan span = attention_span(c, a, run.seq);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), r = lane & 15, part = lane / 16;
  const int tiles = (int)(((int64_t)span.rows * group + 15) / 16);
  const int head = run.local % c.kv_heads, tile = run.local / c.kv_heads % tiles, split = run.local / c.kv_heads / tiles;
  const int blocks = (c.dim + 31) / 32;
  const float factor = a.scale * kAttentionLog2e;

  // this lane's query: its row of the call, and the keys it sees
  const int64_t index = (int64_t)tile * 16 + r;
  const bool row_there = index < (int64_t)span.rows * group;
  const int token = row_there ? (int)(index / group) : 0;
  const int64_t t = span.first + token;
  const int q_head = head * group + (int)(index - (int64_t)token * group);
  const auto end_of = [&](int i) {
    const int64_t p = span.position + i + 1;
    return !a.causal || p > span.high ? span.high : p < 0 ? 0 : (int)p;
  };
  const auto low_of = [&](int i) {
    const int64_t p = a.window ? span.position + i - a.window + 1 : 0;
    return p < 0 ? 0 : p < span.high ? (int)p : span.high;
  };
  const int end = row_there ? end_of(token) : 0, low = row_there ? low_of(token) : 0;
  at_b8 q[PIECES][DB];
#pragma unroll
  for (int st = 0; st < DB; ++st) {
    const int col = part * 8 * DB + 8 * st;
    float x[8];
    if (row_there && col < c.dim)
      mx_load8<TYPE>(static_cast<const E*>(a.q.data) + t * a.q.row + (int64_t)q_head * a.q.head + col, c.dim - col, x);
    else
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      __bf16 p[PIECES];
      attention_split<PIECES>(x[i], p);
#pragma unroll
      for (int k = 0; k < PIECES; ++k) q[k][st][i] = p[k];
    }
  }

  // the keys of this run that any of the tile's rows sees
  const int64_t last_row = ((int64_t)tile + 1) * 16 < (int64_t)span.rows * group ? ((int64_t)tile + 1) * 16 - 1 : (int64_t)span.rows * group - 1;
  const int start = span.low & ~15, all_blocks = span.high > span.low ? (span.high - start + kBlock - 1) / kBlock : 1;
  const int each = (all_blocks + run.runs - 1) / run.runs;
  // (positions stay 2^16 below 2^31; of the runs' ends only what is below `high` counts)
  const int64_t run_first = start + (int64_t)split * each * kBlock, run_end = run_first + (int64_t)each * kBlock;
  int k0 = run_first < span.high ? (int)run_first : span.high, k1 = run_end < span.high ? (int)run_end : span.high;
  const int tile_low = low_of((int)((int64_t)tile * 16 / group)) & ~15, tile_end = end_of((int)(last_row / group));
  if (k0 < tile_low) k0 = tile_low;
  if (k1 > tile_end) k1 = tile_end;

  uint8_t* mine = lds + wave * kRegion;
  float m = -INFINITY, l = 0.0f;
  at_f4 o[2 * DB] = {};
  Chunk<KF, DB> kc[2];
  Chunk<VF, DB> vc[2];
  bool there[2];  // the key has a place
  const auto load = [&](int base) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int key = base + 16 * i + r;
      int64_t place = key < k1 ? cache_place(c, run.seq, key, head) : -1;
      there[i] = place >= 0;
      if (place < 0) place = 0;
      kc[i].load(c.k_codes, c.k_scales, place, blocks, part);
      vc[i].load(c.v_codes, c.v_scales, place, blocks, part);
    }
  };
  int base = k0 + wave * kKeys;
  if (base < k1) load(base);
  for (; base < k1; base += kBlock) {
    // S^T, values into LDS
    at_f4 s[2] = {};
    uint64_t none[2][Chunk<VF, DB>::kScales];  // lanes whose blocks of a value stand for NaN
    uint32_t seen = ((uint32_t)__ballot(there[0]) & 0xffff) | (uint32_t)__ballot(there[1]) << 16;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
#pragma unroll
      for (int st = 0; st < DB; ++st) {
        const at_b8 k = kc[i].values(st);
#pragma unroll
        for (int p = PIECES - 1; p >= 0; --p) s[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, q[p][st], s[i], 0, 0, 0);
      }
      // (what has no place, and what is NaN, is zero here: a probability of zero does not take a NaN away)
      constexpr int kScales = Chunk<VF, DB>::kScales, kEach = Chunk<VF, DB>::kWords / kScales;
#pragma unroll
      for (int b = 0; b < kScales; ++b) {
        const bool nan = vc[i].scale[b] == 255, zero = nan || !there[i];
        none[i][b] = __ballot(nan && there[i]);
        if (zero) vc[i].scale[b] = 0;
#pragma unroll
        for (int w = 0; w < kEach; ++w) vc[i].w[b * kEach + w] = zero ? 0 : vc[i].w[b * kEach + w];
      }
#pragma unroll
      for (int st = 0; st < DB; ++st) *reinterpret_cast<at_b8*>(mine + (16 * i + r) * kRow + part * 16 * DB + 16 * st) = vc[i].values(st);
    }
    // the next keys and values on their way
    if (base + kBlock < k1) load(base + kBlock);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    // softmax: this lane's are keys base + 16 i + 4 part + j of query r
    const int from = low - base, to = end - base;
    seen &= from >= 32 || to <= 0 || from >= to ? 0 : (from <= 0 ? ~0u : ~0u << from) & (to >= 32 ? ~0u : ~(~0u << to));
    float x[2][4], most = m;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        x[i][j] = seen >> (16 * i + 4 * part + j) & 1 ? s[i][j] * factor : -INFINITY;
        most = fmaxf(most, x[i][j]);
      }
    most = max_of_parts(most);
    const float zero = most == -INFINITY ? 0.0f : most;
    const float fade = __builtin_amdgcn_exp2f(m - zero);
    m = most;
    l *= fade;
    at_b8 pr[PIECES];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float p = __builtin_amdgcn_exp2f(x[i][j] - zero);
        l += p;
        __bf16 piece[PIECES];
        attention_split<PIECES>(p, piece);
#pragma unroll
        for (int k = 0; k < PIECES; ++k) pr[k][4 * i + j] = piece[k];
      }
    // O^T
#pragma unroll
    for (int d = 0; d < 2 * DB; ++d) {
#pragma unroll
      for (int j = 0; j < 4; ++j) o[d][j] *= fade;
      union {
        at_s4 half[2];
        at_b8 whole;
      } v;
#pragma unroll
      for (int i = 0; i < 2; ++i)
        v.half[i] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((at_lds_s4*)(mine + (16 * i + 4 * part + r / 4) * kRow + 32 * d + 8 * (r % 4)));
#pragma unroll
      for (int p = PIECES - 1; p >= 0; --p) o[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v.whole, pr[p], o[d], 0, 0, 0);
    }
    uint64_t any = 0;
#pragma unroll
    for (int b = 0; b < Chunk<VF, DB>::kScales; ++b) any |= none[0][b] | none[1][b];
    if (any) {
      // NaN for the queries that see such a value, and for no other: tile d is columns 16 d on, which part 2 d / DB holds
#pragma unroll
      for (int d = 0; d < 2 * DB; ++d) {
        const int of = 2 * d / DB, b = DB == 8 ? d / 2 % 2 : 0;
        const uint32_t keys = ((uint32_t)(none[0][b] >> (16 * of)) & 0xffff) | (uint32_t)(none[1][b] >> (16 * of)) << 16;
#pragma unroll
        for (int j = 0; j < 4; ++j) o[d][j] = seen & keys ? NAN : o[d][j];
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }

  // the wavefronts' results together
  l = sum_of_parts(l);
  float* sums = reinterpret_cast<float*>(mine);
  float2* stats = reinterpret_cast<float2*>(mine + 16 * kSums * 4);
#pragma unroll
  for (int d = 0; d < 2 * DB; ++d) *reinterpret_cast<at_f4*>(sums + r * kSums + 16 * d + 4 * part) = o[d];
  if (part == 0) stats[r] = make_float2(m, l);
  __syncthreads();
  const int row = threadIdx.x / 16, col = threadIdx.x % 16 * (2 * DB);
  float most = -INFINITY, weight[kWaves], sum = 0.0f;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) most = fmaxf(most, reinterpret_cast<const float2*>(lds + w * kRegion + 16 * kSums * 4)[row].x);
  const float zero = most == -INFINITY ? 0.0f : most;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    const float2 s = reinterpret_cast<const float2*>(lds + w * kRegion + 16 * kSums * 4)[row];
    weight[w] = __builtin_amdgcn_exp2f(s.x - zero);
    sum = __builtin_fmaf(s.y, weight[w], sum);
  }
  float y[2 * DB];
#pragma unroll
  for (int i = 0; i < 2 * DB; ++i) {
    y[i] = 0.0f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) y[i] = __builtin_fmaf(reinterpret_cast<const float*>(lds + w * kRegion)[row * kSums + col + i], weight[w], y[i]);
  }
  const int64_t out_index = (int64_t)tile * 16 + row;
  if (out_index >= (int64_t)span.rows * group) return;
  const int64_t out_row = (span.first + out_index / group) * a.heads + head * group + out_index % group;
  if (run.runs == 1) {
    const float inverse = sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f;
#pragma unroll
    for (int i = 0; i < 2 * DB; ++i)
      if (col + i < c.dim) static_cast<E*>(a.out)[out_row * c.dim + col + i] = (E)(y[i] * inverse);
    if (col == 0) {
      if (a.lse) a.lse[out_row] = sum == 0.0f ? -INFINITY : (most + __builtin_amdgcn_logf(sum)) * kAttentionLn2;
      work.joins[out_row] = make_int2(0, 1);
    }
    return;
  }
  const int64_t first = run.slot + ((int64_t)tile * c.kv_heads + head) * run.runs, slot = first + split;
  if (slot < 0 || slot >= 2 * kRuns<DB>) return;  // (only offsets that break the contract)
#pragma unroll
  for (int i = 0; i < 2 * DB; ++i) work.partial[(slot * 16 + row) * D + col + i] = y[i];
  if (col == 0) {
    work.stats[slot * 16 + row] = make_float2(most, sum);
    if (split == 0) work.joins[out_row] = make_int2((int)(first * 16 + row), run.runs);
  }
}

// Joins the runs of a row.  Four columns a thread, the runs by turns; the order of the sums is the runs'.
template <int TYPE, int DB>
__global__ __launch_bounds__(kThreads) void join_kernel(CacheArgs c, AttentionArgs a, AttentionWork work, int64_t rows) {
  using E = typename MxElement<TYPE>::type;
  constexpr int D = 32 * DB, kColumns = D / 4, kTurns = kThreads / kColumns;
  __shared__ float weights[kMostRuns];
  __shared__ float shared[kWaves][2];
  __shared__ at_f4 sums[kTurns][kColumns];
  const int tid = threadIdx.x;
  for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
    const int64_t t = row / a.heads;
    if (t < c.offsets[0] || t >= c.offsets[c.seqs]) continue;
    const int2 join = work.joins[row];
    const int runs = join.y;
    // (what no sequence wrote may be anything)
    if (runs < 2 || runs > kRuns<DB> || join.x < 0 || (int64_t)join.x + 16 * (runs - 1) >= 32 * kRuns<DB>) continue;
    float most = -INFINITY, sum = 0.0f;
    for (int i = tid; i < runs; i += kThreads) most = fmaxf(most, work.stats[join.x + 16 * i].x);
#pragma unroll
    for (int d = 1; d < 64; d *= 2) most = fmaxf(most, __shfl_xor(most, d));
    __syncthreads();
    if ((tid & 63) == 0) shared[tid / 64][0] = most;
    __syncthreads();
    most = fmaxf(fmaxf(shared[0][0], shared[1][0]), fmaxf(shared[2][0], shared[3][0]));
    const float zero = most == -INFINITY ? 0.0f : most;
    for (int i = tid; i < runs; i += kThreads) {
      const float2 s = work.stats[join.x + 16 * i];
      const float w = __builtin_amdgcn_exp2f(s.x - zero);
      weights[i] = w;
      sum = __builtin_fmaf(s.y, w, sum);
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
    if ((tid & 63) == 0) shared[tid / 64][1] = sum;
    __syncthreads();
    sum = (shared[0][1] + shared[1][1]) + (shared[2][1] + shared[3][1]);
    const int col = tid % kColumns, turn = tid / kColumns;
    at_f4 y = {};
    for (int i = turn; i < runs; i += kTurns) {
      const at_f4 p = *reinterpret_cast<const at_f4*>(work.partial + ((int64_t)join.x + 16 * i) * D + 4 * col);
#pragma unroll
      for (int k = 0; k < 4; ++k) y[k] = __builtin_fmaf(p[k], weights[i], y[k]);
    }
    sums[turn][col] = y;
    __syncthreads();
    if (turn == 0) {
#pragma unroll
      for (int i = 1; i < kTurns; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k) y[k] += sums[i][col][k];
      const float inverse = sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f;
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (4 * col + k < c.dim) static_cast<E*>(a.out)[row * c.dim + 4 * col + k] = (E)(y[k] * inverse);
      if (a.lse && col == 0) a.lse[row] = sum == 0.0f ? -INFINITY : (most + __builtin_amdgcn_logf(sum)) * kAttentionLn2;
    }
    __syncthreads();
  }
}

constexpr int64_t padded16(int64_t n) { return (n + 15) / 16 * 16; }
int blocks_of(int64_t dim) { return dim <= 64 ? 2 : dim <= 128 ? 4 : 8; }
int64_t partial_floats(int db) { return 2ll * (db == 8 ? kRuns<8> : kRuns<4>) * 16 * 32 * db; }
int64_t stats_bytes(int db) { return 2ll * (db == 8 ? kRuns<8> : kRuns<4>) * 16 * (int64_t)sizeof(float2); }

template <int TYPE, int KF, int VF, int DB>
hipError_t launch(const CacheArgs& c, const AttentionArgs& a, const AttentionWork& work, hipStream_t st) {
  const int group = a.heads / c.kv_heads;
  const int64_t units = ((int64_t)a.T * group / 16 + (c.seqs < a.T ? c.seqs : a.T)) * c.kv_heads;
  const hipError_t e = launch_kernel(attention_kernel<TYPE, KF, VF, DB>, dim3((uint32_t)(units + kRuns<DB>)), dim3(kThreads), 0, st, c, a, work, group);
  if (e != hipSuccess) return e;
  const int64_t rows = (int64_t)a.T * a.heads, most = max_blocks(kThreads);
  return launch_kernel(join_kernel<TYPE, DB>, dim3((uint32_t)(rows < most ? rows : most)), dim3(kThreads), 0, st, c, a, work, rows);
}
template <int TYPE, int KF, int VF>
hipError_t with_dim(const CacheArgs& c, const AttentionArgs& a, const AttentionWork& work, hipStream_t st) {
  switch (blocks_of(c.dim)) {
    case 2: return launch<TYPE, KF, VF, 2>(c, a, work, st);
    case 4: return launch<TYPE, KF, VF, 4>(c, a, work, st);
  }
  return launch<TYPE, KF, VF, 8>(c, a, work, st);
}
template <int TYPE>
hipError_t with_formats(const CacheArgs& c, const AttentionArgs& a, const AttentionWork& work, hipStream_t st) {
  if (c.k_format == kMxFp4) return c.v_format == kMxFp4 ? with_dim<TYPE, kMxFp4, kMxFp4>(c, a, work, st) : with_dim<TYPE, kMxFp4, kMxFp8>(c, a, work, st);
  return c.v_format == kMxFp4 ? with_dim<TYPE, kMxFp8, kMxFp4>(c, a, work, st) : with_dim<TYPE, kMxFp8, kMxFp8>(c, a, work, st);
}

}  // namespace

int64_t mx_attention_workspace_bytes(int64_t T, int64_t heads, int64_t kv_heads, int64_t dim) {
  const int db = blocks_of(dim);
  return partial_floats(db) * 4 + stats_bytes(db) + padded16(T * heads * (int64_t)sizeof(int2));
}

hipError_t launch_mx_attention(const CacheArgs& c, const AttentionArgs& a, void* workspace, hipStream_t st) {
  const int db = blocks_of(c.dim);
  uint8_t* w = static_cast<uint8_t*>(workspace);
  AttentionWork work;
  work.partial = reinterpret_cast<float*>(w);
  work.stats = reinterpret_cast<float2*>(w + partial_floats(db) * 4);
  work.joins = reinterpret_cast<int2*>(w + partial_floats(db) * 4 + stats_bytes(db));
  return a.type == kMxF32 ? with_formats<kMxF32>(c, a, work, st) : a.type == kMxBf16 ? with_formats<kMxBf16>(c, a, work, st) : with_formats<kMxF16>(c, a, work, st);
}

}  // namespace hago
