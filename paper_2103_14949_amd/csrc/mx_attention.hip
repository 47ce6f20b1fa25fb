// Attention over a paged cache of microscaled keys and values, few rows a sequence: the form for single tokens, and the one that is
// right for every call.
//
// out = softmax(scale * q k^T) v in one pass over the keys with the running maximum and sum.  The cache's bytes bound it, so a
// workgroup is one (sequence, 16 rows, head of the cache) and a run of keys, its rows the queries of all heads that share those keys;
// the runs are as long as makes all workgroups' work alike, whatever the lengths, and a second launch joins the sequences that were cut.
// Lengths stay on the device: every wavefront finds its run by a scan over the sequences.
//
// A wavefront goes its own way through 32 keys at a time, with no barrier.  S^T = K Q^T: a lane (key r = lane % 16, part h = lane / 16)
// loads part h of key r, which is whole in one block of 32 (or two) and becomes the operand by conversions.  Its results are keys
// 4 h .. 4 h + 3 of query r, which is the operand of O^T = V^T P^T as it stands, if V^T's lanes hold the same keys; they read them so from
// LDS, 4 x 16 elements at a time transposed.  Codes are an iteration ahead, the pages that they are in two.  Probabilities are two
// bfloat16 numbers for bfloat16 queries too: one would be 2^-8 off, as much as the result's own rounding, and the second costs 0 to 2.5 % where bytes bound the kernel
// (the 64 sequences below 148.1 and 148.6 us, their 4-bit codes 89.1 and 91.5).
//
// 64 sequences of 1024 to 16384 tokens, 32 heads over 8 of 128 columns, 8-bit codes: 147 us with the join's 7, 5.1 TB/s of 752 MB (a copy has 5.9); 4-bit codes 92 us.  One
// token over 1000 keys 9.5 us, 6.5 and 3.8 of them the two kernels: launches, and three rounds of memory in the first.
#include "mx_attention.h"

namespace hago {

namespace {

constexpr int kThreads = 256, kWaves = 4, kRows = 16, kKeys = 32, kBlock = kWaves * kKeys;
// Workgroups that share the keys, by blocks of a row: about three times what is resident, so that the last ones are short (the 64 sequences above with 1024, 2048 and
// 4096 of them: 167, 158 and 173 us when each began more slowly).
template <int DB>
constexpr int kRuns = DB == 8 ? 1024 : 2048;
constexpr int kMostRuns = 2048;

__device__ __forceinline__ float max_of_parts(float v) {
  v = fmaxf(v, __shfl_xor(v, 16));
  return fmaxf(v, __shfl_xor(v, 32));
}
__device__ __forceinline__ float sum_of_parts(float v) {
  v += __shfl_xor(v, 16);
  return v + __shfl_xor(v, 32);
}

template <int TYPE, int KF, int VF, int DB, bool EVEN>
__global__ __launch_bounds__(kThreads, TYPE != kMxBf16 && DB == 8 ? 1 : 2) void attention_kernel(CacheArgs c, AttentionArgs a, AttentionWork work, uint32_t group) {
  using E = typename MxElement<TYPE>::type;
  constexpr int PIECES = kAttentionPieces<TYPE>, PROBABILITIES = TYPE == kMxF32 ? 3 : 2, D = 32 * DB;
  constexpr int kRow = 2 * D + 32;                          // bytes of a row of values in LDS: 4 x 16 elements of it fall on different banks
  constexpr int kSums = D + 4;                              // floats of a row of results there
  constexpr int kRegion = kKeys * kRow;                     // of a wavefront
  static_assert(16 * kSums * 4 + 128 <= kRegion);
  __shared__ __align__(16) uint8_t lds[kWaves * kRegion];

  AttentionRun run;
  AttentionSpan span;
  if (!attention_run<kRows, kBlock, kRuns<DB>>(c, a, work, group, blockIdx.x, run, span)) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), r = lane & 15, part = lane / 16;
  // (rows of all heads: at most 2^27)
  const uint32_t all_rows = (uint32_t)span.rows * group, tiles = (all_rows + kRows - 1) / kRows;
  const uint32_t unit = (uint32_t)run.local / (uint32_t)c.kv_heads;
  const int head = run.local - (int)unit * c.kv_heads, split = (int)(unit / tiles), tile = (int)(unit - (uint32_t)split * tiles);
  const int blocks = (c.dim + 31) / 32;
  const float factor = a.scale * kAttentionLog2e;

  // this lane's query: its row of the call, and the keys it sees
  const uint32_t index = (uint32_t)tile * kRows + r;
  const bool row_there = index < all_rows;
  const int token = row_there ? (int)(index / group) : 0;
  const int64_t t = span.first + token;
  const int q_head = head * (int)group + (row_there ? (int)(index - token * group) : 0);
  const auto end_of = [&](int i) {
    const int64_t p = span.position + i + 1;
    return !a.causal || p > span.high ? span.high : p < 0 ? 0 : (int)p;
  };
  const auto low_of = [&](int i) {
    const int64_t p = a.window ? span.position + i - a.window + 1 : 0;
    return p < 0 ? 0 : p < span.high ? (int)p : span.high;
  };
  const int end = row_there ? end_of(token) : 0, low = row_there ? low_of(token) : 0;
  typedef E elements __attribute__((ext_vector_type(8)));
  typedef elements elements_any __attribute__((aligned(sizeof(E))));
  elements x_q[DB] = {};
  {
    const E* const row = static_cast<const E*>(a.q.data) + t * a.q.row + (int64_t)q_head * a.q.head;
    if (c.dim % 8 == 0) {
      // all under way before the first is waited for; columns behind the last are others of the row, and zero after that
#pragma unroll
      for (int st = 0; st < DB; ++st) {
        const int col = part * 8 * DB + 8 * st;
        x_q[st] = *reinterpret_cast<const elements_any*>(row + (col < c.dim ? col : 0));
      }
    } else {
#pragma unroll
      for (int st = 0; st < DB; ++st)
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (part * 8 * DB + 8 * st + i < c.dim) x_q[st][i] = row[part * 8 * DB + 8 * st + i];
    }
  }

  // the keys of this run that any of the tile's rows sees
  const uint32_t first_row = (uint32_t)tile * kRows, last_row = first_row + kRows < all_rows ? first_row + kRows - 1 : all_rows - 1;
  const int start = span.low & ~15, all_blocks = span.high > span.low ? (span.high - start + kBlock - 1) / kBlock : 1;
  const int each = (all_blocks + run.runs - 1) / run.runs;
  // (positions stay 2^16 below 2^31; of the runs' ends only what is below `high` counts)
  const int64_t run_first = start + (int64_t)split * each * kBlock, run_end = run_first + (int64_t)each * kBlock;
  int k0 = run_first < span.high ? (int)run_first : span.high, k1 = run_end < span.high ? (int)run_end : span.high;
  const int tile_low = low_of((int)(first_row / group)) & ~15, tile_end = end_of((int)(last_row / group));
  if (k0 < tile_low) k0 = tile_low;
  if (k1 > tile_end) k1 = tile_end;

  uint8_t* mine = lds + wave * kRegion;
  float m = -INFINITY, l = 0.0f;
  at_f4 o[2 * DB] = {};
  using KeyChunk = AttentionChunk<KF, DB>;
  using ValueChunk = AttentionChunk<VF, DB>;
  // On their way: the pages of the keys after the next ones, the next keys and values.  Where pages are whole sixteens (EVEN), all about a tile's page is the same in
  // every lane.
  uint32_t key_code[KeyChunk::kLoads], value_code[ValueChunk::kLoads], key_scale[KeyChunk::kScales], value_scale[ValueChunk::kScales];
#pragma unroll
  for (int i = 0; i < KeyChunk::kLoads; ++i) key_code[i] = KeyChunk::code_at(blocks, part, i) + (EVEN ? r * (blocks * KeyChunk::kRowWords * 4) : 0);
#pragma unroll
  for (int i = 0; i < ValueChunk::kLoads; ++i) value_code[i] = ValueChunk::code_at(blocks, part, i) + (EVEN ? r * (blocks * ValueChunk::kRowWords * 4) : 0);
  // (a tile's first place is a multiple of its keys: the scales' places in their words are a lane's own)
  uint32_t key_shift[KeyChunk::kScales], value_shift[ValueChunk::kScales];
#pragma unroll
  for (int i = 0; i < KeyChunk::kScales; ++i) {
    const uint32_t at = KeyChunk::scale_at(blocks, part, i) + (EVEN ? r * blocks : 0);
    key_scale[i] = EVEN ? at & ~3u : at;
    key_shift[i] = EVEN ? (at & 3) * 8 : 0;
  }
#pragma unroll
  for (int i = 0; i < ValueChunk::kScales; ++i) {
    const uint32_t at = ValueChunk::scale_at(blocks, part, i) + (EVEN ? r * blocks : 0);
    value_scale[i] = EVEN ? at & ~3u : at;
    value_shift[i] = EVEN ? (at & 3) * 8 : 0;
  }
  const int32_t* const table = c.table + run.seq * c.table_stride;
  int own = 0;  // (zero; vector loads come back in the order that they are asked for)
  asm volatile("" : "+v"(own));
  KeyChunk kc[2];
  ValueChunk vc[2];
  int32_t next_page[2];
  bool there[2];  // the page is there
  const auto look_up = [&](int base) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int key = base + 16 * i + (EVEN ? 0 : r);
      next_page[i] = -1;
      if (key < k1) next_page[i] = table[cache_page_of(c, (uint32_t)key) + own];
    }
  };
  const auto load = [&](int base) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint32_t key = base + 16 * i + (EVEN ? 0 : r);
      const int32_t page = EVEN ? __builtin_amdgcn_readfirstlane(next_page[i]) : next_page[i];
      there[i] = (uint32_t)page < (uint32_t)c.pages;
      // (any row, where there is none)
      const int64_t place = there[i] ? ((int64_t)page * c.kv_heads + head) * c.page + (key - cache_page_of(c, key) * (uint32_t)c.page) : 0;
      kc[i].template load<EVEN>(c.k_codes + place * (blocks * KeyChunk::kRowWords * 4), c.k_scales + place * blocks, key_code, key_scale);
      vc[i].template load<EVEN>(c.v_codes + place * (blocks * ValueChunk::kRowWords * 4), c.v_scales + place * blocks, value_code, value_scale);
    }
  };
  int base = k0 + wave * kKeys;
  look_up(base);
  if (base < k1) load(base);
  look_up(base + kBlock);
  at_b8 q[PIECES][DB];
#pragma unroll
  for (int st = 0; st < DB; ++st)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float v = row_there && part * 8 * DB + 8 * st < c.dim ? (float)x_q[st][i] : 0.0f;
      __bf16 p[PIECES];
      attention_split<PIECES>(v, p);
#pragma unroll
      for (int k = 0; k < PIECES; ++k) q[k][st][i] = p[k];
    }
  for (; base < k1; base += kBlock) {
    // S^T, values into LDS
    constexpr int kScales = ValueChunk::kScales, kEach = ValueChunk::kWords / kScales;
    at_f4 s[2] = {};
    uint64_t none[2][kScales] = {}, any = 0;  // lanes whose blocks of a value stand for NaN
    uint32_t seen = EVEN ? (there[0] ? 0xffffu : 0) | (there[1] ? 0xffff0000u : 0) : ((uint32_t)__ballot(there[0]) & 0xffff) | (uint32_t)__ballot(there[1]) << 16;
    if (k1 - base < 32) seen &= ~(~0u << (k1 - base));
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if (EVEN) kc[i].unpack(key_shift), vc[i].unpack(value_shift);
#pragma unroll
      for (int st = 0; st < DB; ++st) {
        const at_b8 k = kc[i].values(st);
#pragma unroll
        for (int p = PIECES - 1; p >= 0; --p) s[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, q[p][st], s[i], 0, 0, 0);
      }
      bool special = false;
#pragma unroll
      for (int b = 0; b < kScales; ++b) special |= vc[i].scale[b] == 255;
      if (__ballot(special) || (seen >> (16 * i) & 0xffff) != 0xffff) {
        // what has no place, and what is NaN, is zero in the products: a probability of zero does not take a NaN away
        const bool mine_there = seen >> (16 * i + r) & 1;
#pragma unroll
        for (int b = 0; b < kScales; ++b) {
          const bool nan = vc[i].scale[b] == 255, zero = nan || !mine_there;
          none[i][b] = __ballot(nan && mine_there);
          any |= none[i][b];
          if (zero) vc[i].scale[b] = 0;
#pragma unroll
          for (int w = 0; w < kEach; ++w) vc[i].w[b * kEach + w] = zero ? 0 : vc[i].w[b * kEach + w];
        }
      }
#pragma unroll
      for (int st = 0; st < DB; ++st) *reinterpret_cast<at_b8*>(mine + (16 * i + r) * kRow + part * 16 * DB + 16 * st) = vc[i].values(st);
    }
    // the next keys and values on their way
    if (base + kBlock < k1) load(base + kBlock);
    look_up(base + 2 * kBlock);
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
    at_b8 pr[PROBABILITIES];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float p = __builtin_amdgcn_exp2f(x[i][j] - zero);
        l += p;
        __bf16 piece[PROBABILITIES];
        attention_split<PROBABILITIES>(p, piece);
#pragma unroll
        for (int k = 0; k < PROBABILITIES; ++k) pr[k][4 * i + j] = piece[k];
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
      for (int p = PROBABILITIES - 1; p >= 0; --p) o[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v.whole, pr[p], o[d], 0, 0, 0);
    }
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
  const uint32_t out_index = first_row + row;
  if (out_index >= all_rows) return;
  const int64_t out_row = (int64_t)(span.first + out_index / group) * a.heads + head * group + out_index % group;
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

// Joins the runs of a row, whose partials are `apart` rows apart: by the four wavefronts of a workgroup where there are few rows (PARTS 4; a long sequence's token has up
// to a run a CU), by one where there are many.  The order of the sums is the runs' in either.  A wavefront looks at `each` rows together for those that were cut:
// none of a long prompt's, whose units are many (a workgroup for every row of 8192 x 32 took 110 us to find nothing; this takes 4.6).
template <int TYPE, int DB, int PARTS>
__global__ __launch_bounds__(kThreads) void join_kernel(CacheArgs c, AttentionArgs a, AttentionWork work, int64_t rows, int each, int apart, int slots) {
  using E = typename MxElement<TYPE>::type;
  constexpr int D = 32 * DB, kColumns = D / 64;  // a lane's
  typedef float columns __attribute__((ext_vector_type(kColumns)));
  __shared__ columns sums[PARTS - 1 ? PARTS - 1 : 1][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), part = PARTS == 1 ? 0 : wave;
  const int64_t first = (PARTS == 1 ? (int64_t)blockIdx.x * kWaves + wave : (int64_t)blockIdx.x) * each, mine = first + lane;
  bool cut = false;
  int2 whose = make_int2(0, 0);
  if (lane < each && mine < rows) {
    whose = work.joins[mine];
    const int t = (int)((uint32_t)mine / (uint32_t)a.heads);  // (rows of all heads: at most 2^27)
    // (what no sequence wrote may be anything)
    cut = t >= c.offsets[0] && t < c.offsets[c.seqs] && whose.y >= 2 && whose.y <= kMostRuns && whose.x >= 0 &&
          (int64_t)whose.x + (int64_t)apart * (whose.y - 1) < (int64_t)apart * slots;
  }
  for (uint64_t left = __ballot(cut); left; left &= left - 1) {
    const int at = __builtin_ctzll(left);
    const int64_t row = first + at;
    const int from = __builtin_amdgcn_readlane(whose.x, at), runs = __builtin_amdgcn_readlane(whose.y, at);
    const float2* stats = work.stats + from;
    const float* partial = work.partial + (int64_t)from * D + lane * kColumns;
    const auto partial_of = [&](int i) { return *reinterpret_cast<const columns*>(partial + (int64_t)apart * i * D); };
    // the first partials are under way while the weights are worked out
    constexpr int kEarly = 4;
    columns early[kEarly];
#pragma unroll
    for (int i = 0; i < kEarly; ++i) early[i] = part + i * PARTS < runs ? partial_of(part + i * PARTS) : columns{};
    float most = -INFINITY, sum = 0.0f;
    for (int i = lane; i < runs; i += 64) most = fmaxf(most, stats[(int64_t)apart * i].x);
#pragma unroll
    for (int d = 1; d < 64; d *= 2) most = fmaxf(most, __shfl_xor(most, d));
    const float zero = most == -INFINITY ? 0.0f : most;
    for (int i = lane; i < runs; i += 64) {
      const float2 s = stats[(int64_t)apart * i];
      sum = __builtin_fmaf(s.y, __builtin_amdgcn_exp2f(s.x - zero), sum);
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
    columns y = {};
    const auto add = [&](int i, const columns& p) {
      const float w = __builtin_amdgcn_exp2f(stats[(int64_t)apart * i].x - zero);
#pragma unroll
      for (int k = 0; k < kColumns; ++k) y[k] = __builtin_fmaf(p[k], w, y[k]);
    };
#pragma unroll
    for (int i = 0; i < kEarly; ++i)
      if (part + i * PARTS < runs) add(part + i * PARTS, early[i]);
#pragma unroll 4
    for (int i = part + kEarly * PARTS; i < runs; i += PARTS) add(i, partial_of(i));
    if constexpr (PARTS > 1) {
      if (part) sums[part - 1][lane] = y;
      __syncthreads();  // (all wavefronts go through the same rows)
      if (part) continue;
#pragma unroll
      for (int i = 0; i < PARTS - 1; ++i)
#pragma unroll
        for (int k = 0; k < kColumns; ++k) y[k] += sums[i][lane][k];
    }
    const float inverse = sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f;
#pragma unroll
    for (int k = 0; k < kColumns; ++k)
      if (kColumns * lane + k < c.dim) static_cast<E*>(a.out)[row * c.dim + kColumns * lane + k] = (E)(y[k] * inverse);
    if (a.lse && lane == 0) a.lse[row] = sum == 0.0f ? -INFINITY : (most + __builtin_amdgcn_logf(sum)) * kAttentionLn2;
  }
}

// Which kernel: the one for many rows where a sequence has more than two tiles of sixteen on the average, queries of all heads that share keys (the number of rows of
// each is not known here).  16 sequences of 4096, 16, 32, 48, 64 and 128 rows of 128 columns, us: bfloat16 47, 60, 78, 87, 151 here and 56, 60, 58, 60, 71 there; float16 53, 68,
// 88, 95, 160 and 71, 73, 74, 75, 92.  Short sequences gain later: 64 chunks of 64 rows with nothing before them 26 and 38, of 256 rows 75 and 46.  One chunk of 512 tokens over 32768 and
// 128 single tokens over 1024, 20 rows on the average, take 999 here (296 and 72 each by itself).
// binary32 queries take three products for one and have the kernel here alone.
constexpr int64_t kManyRowsFrom = 33;
bool many_rows(const AttentionArgs& a, const CacheArgs& c) { return (int64_t)a.T * (a.heads / c.kv_heads) >= kManyRowsFrom * c.seqs; }

// More sequences are planned by a launch in front.  With every workgroup looking at all of them, tokens over 512 sequences of 512, 2048 of 1024 and 4096 of 64 keys took 152, 1172 and
// 1973 us; so 115, 770 and 276, and the launch 5 of those.
constexpr int64_t kMostScanned = 256;

constexpr int64_t padded16(int64_t n) { return (n + 15) / 16 * 16; }

template <int TYPE, int DB>
hipError_t launch_join(const CacheArgs& c, const AttentionArgs& a, const AttentionWork& work, int apart, int slots, hipStream_t st) {
  const int64_t rows = (int64_t)a.T * a.heads;
  if (rows <= 4096)  // a row a workgroup
    return launch_kernel(join_kernel<TYPE, DB, 4>, dim3((uint32_t)rows), dim3(kThreads), 0, st, c, a, work, rows, 1, apart, slots);
  const int64_t each = rows < 64 * 8192 ? (rows + 8191) / 8192 : 64, waves = (rows + each - 1) / each;
  return launch_kernel(join_kernel<TYPE, DB, 1>, dim3((uint32_t)((waves + kWaves - 1) / kWaves)), dim3(kThreads), 0, st, c, a, work, rows, (int)each, apart, slots);
}
template <int TYPE, int KF, int VF, int DB>
hipError_t launch(const CacheArgs& c, const AttentionArgs& a, const AttentionWork& work, hipStream_t st) {
  const int group = a.heads / c.kv_heads;
  if (TYPE != kMxF32 && many_rows(a, c)) {
    const hipError_t e = TYPE == kMxBf16 ? launch_attention_many_bf16(c, a, work, st) : launch_attention_many_f16(c, a, work, st);
    return e != hipSuccess ? e : launch_join<TYPE, DB>(c, a, work, attention_many_rows(TYPE, DB), 2 * kAttentionManyRuns, st);
  }
  const int64_t units = ((int64_t)a.T * group / kRows + (c.seqs < a.T ? c.seqs : a.T)) * c.kv_heads;
  if (const hipError_t e = launch_plan<kRows, kBlock, kRuns<DB>>(c, a, work, st); e != hipSuccess) return e;
  auto* kernel = attention_even(c, 16) ? attention_kernel<TYPE, KF, VF, DB, true> : attention_kernel<TYPE, KF, VF, DB, false>;
  const hipError_t e = launch_kernel(kernel, dim3((uint32_t)(units + kRuns<DB>)), dim3(kThreads), 0, st, c, a, work, (uint32_t)group);
  return e != hipSuccess ? e : launch_join<TYPE, DB>(c, a, work, kRows, 2 * kRuns<DB>, st);
}
template <int TYPE, int KF, int VF>
hipError_t with_dim(const CacheArgs& c, const AttentionArgs& a, const AttentionWork& work, hipStream_t st) {
  switch (attention_blocks(c.dim)) {
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

// Rows of partials that a call can have.
static int64_t partial_rows(int64_t T, int64_t heads, int64_t kv_heads, int db) {
  const int64_t few = 2ll * (db == 8 ? kRuns<8> : kRuns<4>) * kRows;
  const int64_t many = 2ll * kAttentionManyRuns * attention_many_rows(kMxBf16, db);  // (the most of any type)
  return T * (heads / kv_heads) >= kManyRowsFrom && many > few ? many : few;
}

int64_t mx_attention_workspace_bytes(int64_t T, int64_t seqs, int64_t heads, int64_t kv_heads, int64_t dim) {
  const int db = attention_blocks(dim);
  return partial_rows(T, heads, kv_heads, db) * (32 * db * 4 + (int64_t)sizeof(float2)) + padded16(T * heads * (int64_t)sizeof(int2)) +
         (seqs > kMostScanned ? (seqs + 1) * 2 * (int64_t)sizeof(uint32_t) : 0);
}

hipError_t launch_mx_attention(const CacheArgs& c, const AttentionArgs& a, void* workspace, hipStream_t st) {
  const int db = attention_blocks(c.dim);
  const int64_t rows = partial_rows(a.T, a.heads, c.kv_heads, db);
  uint8_t* w = static_cast<uint8_t*>(workspace);
  AttentionWork work;
  work.partial = reinterpret_cast<float*>(w);
  work.stats = reinterpret_cast<float2*>(w + rows * 32 * db * 4);
  work.joins = reinterpret_cast<int2*>(w + rows * (32 * db * 4 + (int64_t)sizeof(float2)));
  const int64_t plan = rows * (32 * db * 4 + (int64_t)sizeof(float2)) + padded16((int64_t)a.T * a.heads * (int64_t)sizeof(int2));
  work.plan = c.seqs > kMostScanned ? reinterpret_cast<uint32_t*>(w + plan) : nullptr;
  return a.type == kMxF32 ? with_formats<kMxF32>(c, a, work, st) : a.type == kMxBf16 ? with_formats<kMxBf16>(c, a, work, st) : with_formats<kMxF16>(c, a, work, st);
}

}  // namespace hago
