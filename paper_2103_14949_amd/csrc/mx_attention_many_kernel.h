// Attention over a paged cache of microscaled keys and values, many rows a sequence: chunks and prompts.
//
// The matrix unit bounds it, and beside it the exponentials (four issue slots each on the same SIMD).  A workgroup is one (sequence, tile of rows, head of the cache) and a
// run of keys; its rows are the queries of all heads that share those keys, 32 a wavefront.  Keys and values of 64 positions at a time become
// bfloat16 (values float16, see many_halves) once for all of them, on their way from memory through registers into LDS, with one barrier a tile.  S^T = K Q^T leaves a
// query's scores in two lanes' registers, as the operand of O^T = V^T P^T, so that the softmax needs one lane exchange and nothing of it goes
// through LDS; values are read transposed from there.  The next tile's scores are worked out beside this tile's exponentials, in the order that is written.
//
// Eight wavefronts of 32 rows share a CU, two a SIMD, up to 128 columns of bfloat16; four where 256 registers do not do.  Prompt of 8192, 32 heads over 8 of 128 columns: 544 to 575 us,
// 955 to 1010 TFLOP/s (a product of 8192 x 8192 x 8192 has 1480, of 16384 1600), matrix unit 44 % of the cycles at 2 GHz, vector instructions 57 %: the two hardly overlap; a chunk of 1024 over 32768 517 to
// 550 us; 256 columns 835 to 855 us, 645 TFLOP/s, float16 queries 1020 to 1055, 530 TFLOP/s.  Tried and slower: 64 rows a wavefront, whose sums the compiler copies between register files (1020 us); three tiles in LDS and the
// first operands read in front of the barrier (registers: 595 for 555); eight operands ahead (660 for 590).  LDS is not what bounds it: half the operand reads, on the same
// data twice, 634 us for 652.
#pragma once

#include "mx_attention.h"

namespace hago {

namespace {

typedef float at_f16 __attribute__((ext_vector_type(16)));
typedef _Float16 at_h2 __attribute__((ext_vector_type(2)));
typedef _Float16 at_h8 __attribute__((ext_vector_type(8)));

constexpr int kTile = 64;  // keys

// A lane's value and its partner's (lane ^ 32), which hold the two halves of a query's keys.
__device__ __forceinline__ float2 pair_of(float v) {
  const uint32_t bits = __builtin_bit_cast(uint32_t, v);
  const auto x = __builtin_amdgcn_permlane32_swap(bits, bits, false, false);
  const uint32_t first = x[0], second = x[1];  // (a bit cast of an element of a vector takes the vector's first)
  return make_float2(__builtin_bit_cast(float, first), __builtin_bit_cast(float, second));
}
__device__ __forceinline__ float pair_max(float v) {
  const float2 p = pair_of(v);
  return fmaxf(p.x, p.y);
}
__device__ __forceinline__ float pair_sum(float v) {
  const float2 p = pair_of(v);
  return p.x + p.y;
}

// Bytes of a row in LDS: neighbours on different banks, as they are read.
constexpr int many_key_row(int db) { return 64 * db + 16; }
constexpr int many_value_row(int db) { return 64 * db + 64; }

// In the second product a probability is two bfloat16 numbers, which hold it to 2^-16.  In bfloat16 calls of up to 128 columns, whose loop the matrix unit and the vector
// instructions take turns in, the second would cost 38 % (prompt of 8192 536 -> 743 us, 64 columns 385 -> 504; of 256 columns 8 %), and one alone made the error against 64 bits 1.35 times that of
// the result's own rounding (0.00223 and 0.00166 of it).  There the product is one of float16 numbers, which hold a probability to 2^-11: 2^kHead times the probability, so
// that those down to 2^-27 of the largest have all their bits and those down to 2^-30 the eight of the result, and up to 2^kSlack times that.  Values are in it 2^kValuesUp times theirs,
// exactly, if the scale of their block, so much higher, lies between 2^narrow_low and 2^narrow_high: blocks whose largest magnitude is at least 2^-12 (8 bits; 2^-26 with 4) and below 2^11.  A
// run of keys that meets another block begins again, with two bfloat16 numbers and no tile ahead (prompt of 8192 800 to 830 us, wherever the block is).
constexpr bool many_halves(int type, int db) { return type == kMxBf16 && db != 8; }
constexpr int kValuesUp = 5;
constexpr float kHead = 13.0f;
// (E4M3: 2^-9 to 448, E2M1: 2^-1 to 6; float16: 2^-24 to 65504)
constexpr int narrow_low(int format) { return format == kMxFp4 ? -23 : -15; }
constexpr int narrow_high(int format) { return format == kMxFp4 ? 13 : 7; }

// Eight codes of a block as float16: dwords `w` (fp8: two, fp4: one), scale 2^(byte - 127).
template <int FORMAT>
__device__ __forceinline__ at_h8 attention_halves8(const uint32_t* w, float scale) {
  at_h2 d[4];
  if constexpr (FORMAT == kMxFp4) {
    d[0] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w[0], scale, 0);
    d[1] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w[0], scale, 1);
    d[2] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w[0], scale, 2);
    d[3] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w[0], scale, 3);
  } else {
    d[0] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[0], scale, false);
    d[1] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[0], scale, true);
    d[2] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[1], scale, false);
    d[3] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[1], scale, true);
  }
  at_h8 v;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = d[i / 2][i % 2];
  return v;
}

// A workgroup's LDS; rows are written sixteen bytes at a time.  WAVES threads load a value, each one or two blocks of it.
template <int DB, int WAVES>
struct ManyShared {
  static constexpr int kScales = AttentionChunk<kMxFp8, 4 * DB / WAVES>::kScales;
  struct Values {
    alignas(16) uint8_t rows[kTile * many_value_row(DB)];
    uint64_t none[kScales][WAVES];  // bit WAVES * (key % kKeysAWave) + part: the part's block of a value stands for NaN
    uint64_t gone[WAVES];           // the key has no place
    uint8_t flags[8];               // of the wavefronts that loaded it: 1: some key is gone, 2: some block is NaN, 4: float16 does not hold some block
  };
  alignas(16) uint8_t keys[2][kTile * many_key_row(DB)];
  Values values[2];
};

template <int TYPE, int KF, int VF, int DB, int WAVES, bool EVEN>
__global__ __launch_bounds__(64 * WAVES, WAVES / 4) void many_kernel(CacheArgs c, AttentionArgs a, AttentionWork work, uint32_t group) {
  constexpr int slots = 2 * kAttentionManyRuns;
  using E = typename MxElement<TYPE>::type;
  constexpr int PIECES = kAttentionPieces<TYPE>, D = 32 * DB, THREADS = 64 * WAVES, ROWS = 32 * WAVES, STEPS = 2 * DB, kProducts = 2 * STEPS, kAhead = 4, kLead = kProducts / 4;
  constexpr int kKeyRow = many_key_row(DB), kValueRow = many_value_row(DB);
  constexpr int PARTS = THREADS / kTile, kChunk = 4 * DB / PARTS;   // threads that load a key, and a value
  constexpr int kKeysAWave = 64 / PARTS;
  using KeyChunk = AttentionChunk<KF, kChunk>;
  using ValueChunk = AttentionChunk<VF, kChunk>;
  using Shared = ManyShared<DB, WAVES>;
  using Values = typename Shared::Values;
  extern __shared__ __align__(16) uint8_t lds[];
  Shared& shared = *reinterpret_cast<Shared*>(lds);

  AttentionRun run;
  AttentionSpan span;
  if (!attention_run<ROWS, kTile, kAttentionManyRuns>(c, a, work, group, blockIdx.x, run, span)) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), half = lane / 32;
  // (rows of all heads: at most 2^27)
  const uint32_t all_rows = (uint32_t)span.rows * group, tiles = (all_rows + ROWS - 1) / ROWS;
  // (the last rows see the most keys: they come first)
  const uint32_t unit = (uint32_t)run.local / (uint32_t)c.kv_heads;
  const int head = run.local - (int)unit * c.kv_heads, split = (int)(unit / tiles), tile = (int)(tiles - 1 - (unit - (uint32_t)split * tiles));
  const int blocks = (c.dim + 31) / 32;
  // scores times a factor above zero (what a query does not see is minus infinity before it): the queries take its sign, and are zero where it is
  const float factor = a.scale == 0.0f ? 1.0f : fabsf(a.scale) * kAttentionLog2e;
  const auto end_of = [&](int i) {
    const int64_t p = span.position + i + 1;
    return !a.causal || p > span.high ? span.high : p < 0 ? 0 : (int)p;
  };
  const auto low_of = [&](int i) {
    const int64_t p = a.window ? span.position + i - a.window + 1 : 0;
    return p < 0 ? 0 : p < span.high ? (int)p : span.high;
  };

  // this lane's query
  at_b8 q[PIECES][STEPS];
  const uint32_t index = (uint32_t)tile * ROWS + wave * 32 + (lane & 31);
  const bool row_there = index < all_rows;
  const int token = row_there ? (int)(index / group) : 0;  // (the first row where there is none)
  const int q_head = head * (int)group + (row_there ? (int)(index - token * group) : 0);
  const int low = row_there ? low_of(token) : 0, end = row_there ? end_of(token) : 0;
  {
    typedef E elements __attribute__((ext_vector_type(8)));
    typedef elements elements_any __attribute__((aligned(sizeof(E))));
    const E* const row = static_cast<const E*>(a.q.data) + (int64_t)(span.first + token) * a.q.row + (int64_t)q_head * a.q.head;
    elements x[STEPS] = {};
    if (c.dim % 8 == 0) {
      // all under way before the first is waited for; columns behind the last are others of the row, and zero after that
#pragma unroll
      for (int st = 0; st < STEPS; ++st) {
        const int col = 16 * st + 8 * half;
        x[st] = *reinterpret_cast<const elements_any*>(row + (col < c.dim ? col : 0));
      }
    } else {
#pragma unroll
      for (int st = 0; st < STEPS; ++st)
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (16 * st + 8 * half + i < c.dim) x[st][i] = row[16 * st + 8 * half + i];
    }
#pragma unroll
    for (int st = 0; st < STEPS; ++st)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float v = row_there && 16 * st + 8 * half < c.dim ? (float)x[st][i] : 0.0f;
        __bf16 p[PIECES];
        attention_split<PIECES>(a.scale == 0.0f ? 0.0f : a.scale < 0 ? -v : v, p);
#pragma unroll
        for (int k = 0; k < PIECES; ++k) q[k][st][i] = p[k];
      }
  }

  // the keys of this run that any row of the workgroup sees, of a wavefront, and that all of its rows see
  const uint32_t first_row = (uint32_t)tile * ROWS, last_row = first_row + ROWS < all_rows ? first_row + ROWS - 1 : all_rows - 1;
  const int start = span.low & ~15, all_blocks = span.high > span.low ? (span.high - start + kTile - 1) / kTile : 1;
  const int each = (all_blocks + run.runs - 1) / run.runs;
  const int64_t run_first = start + (int64_t)split * each * kTile, run_end = run_first + (int64_t)each * kTile;
  int k0 = run_first < span.high ? (int)run_first : span.high, k1 = run_end < span.high ? (int)run_end : span.high;
  const int tile_low = low_of((int)(first_row / group)) & ~15, tile_end = end_of((int)(last_row / group));
  if (k0 < tile_low) k0 = tile_low;
  if (k1 > tile_end) k1 = tile_end;
  const uint32_t wave_first = first_row + wave * 32, wave_last = wave_first + 31 < last_row ? wave_first + 31 : last_row;
  const bool wave_there = wave_first <= last_row;
  const int wave_low = wave_there ? low_of((int)(wave_first / group)) : 0, wave_end = wave_there ? end_of((int)(wave_last / group)) : 0;
  // (rows behind the last one see nothing, but nothing of theirs is kept: they may as well see all)
  const int wave_all_low = wave_there ? low_of((int)(wave_last / group)) : 0, wave_all_end = wave_there ? end_of((int)(wave_first / group)) : 0;

  // On their way: the pages of a tile's keys, then its codes, one tile of values and two of keys ahead of the products.  A wavefront loads kKeysAWave
  // neighbours, PARTS lanes each; where pages are whole numbers of those (EVEN), they lie in one page, and all about it is the same in every lane.
  const int loader_key = threadIdx.x / PARTS, part = threadIdx.x % PARTS;
  uint32_t key_code[KeyChunk::kLoads], key_scale[KeyChunk::kScales], value_code[ValueChunk::kLoads], value_scale[ValueChunk::kScales];
#pragma unroll
  for (int i = 0; i < KeyChunk::kLoads; ++i) key_code[i] = KeyChunk::code_at(blocks, part, i) + (EVEN ? lane / PARTS * (blocks * KeyChunk::kRowWords * 4) : 0);
#pragma unroll
  for (int i = 0; i < ValueChunk::kLoads; ++i) value_code[i] = ValueChunk::code_at(blocks, part, i) + (EVEN ? lane / PARTS * (blocks * ValueChunk::kRowWords * 4) : 0);
  // (a tile's first place is a multiple of its keys: the scales' places in their words are a lane's own)
  uint32_t key_shift[KeyChunk::kScales], value_shift[ValueChunk::kScales];
#pragma unroll
  for (int i = 0; i < KeyChunk::kScales; ++i) {
    const uint32_t at = KeyChunk::scale_at(blocks, part, i) + (EVEN ? lane / PARTS * blocks : 0);
    key_scale[i] = EVEN ? at & ~3u : at;
    key_shift[i] = EVEN ? (at & 3) * 8 : 0;
  }
#pragma unroll
  for (int i = 0; i < ValueChunk::kScales; ++i) {
    const uint32_t at = ValueChunk::scale_at(blocks, part, i) + (EVEN ? lane / PARTS * blocks : 0);
    value_scale[i] = EVEN ? at & ~3u : at;
    value_shift[i] = EVEN ? (at & 3) * 8 : 0;
  }
  const int first_key = EVEN ? wave * kKeysAWave : loader_key;
  const int32_t* const table = c.table + run.seq * c.table_stride;
  int own = 0;  // (zero; a vector load waits for no LDS)
  asm volatile("" : "+v"(own));
  int32_t next_page;
  KeyChunk kc;
  ValueChunk vc;
  const auto look_up = [&](int base) {
    const int key = base + first_key;
    next_page = -1;
    if (key < k1) next_page = table[cache_page_of(c, (uint32_t)key) + own];
  };
  // the row of [pages, kv_heads, page] (some row where the key has no place), and whether it is there
  const auto place_of = [&](int base, bool& there) -> int64_t {
    const uint32_t key = base + first_key;
    const int32_t page = EVEN ? __builtin_amdgcn_readfirstlane(next_page) : next_page;
    there = (uint32_t)page < (uint32_t)c.pages;
    return there ? ((int64_t)page * c.kv_heads + head) * c.page + (key - cache_page_of(c, key) * (uint32_t)c.page) : 0;
  };
  const auto load_keys = [&](int64_t place) {
    kc.template load<EVEN>(c.k_codes + place * (blocks * KeyChunk::kRowWords * 4), c.k_scales + place * blocks, key_code, key_scale);
  };
  const auto load_values = [&](int64_t place) {
    vc.template load<EVEN>(c.v_codes + place * (blocks * ValueChunk::kRowWords * 4), c.v_scales + place * blocks, value_code, value_scale);
  };
  const auto store_keys = [&](int turn, int st) {
    if (EVEN && st == 0) kc.unpack(key_shift);
    *reinterpret_cast<at_b8*>(shared.keys[turn] + loader_key * kKeyRow + part * 16 * kChunk + 16 * st) = kc.values(st);
  };
  float m, l;
  at_f16 o[DB];
  // Goes through the keys of the run, HALF: with float16 values; false: float16 does not hold some of them
  const auto go_through = [&]<bool HALF>() -> bool {
    // Values of a tile before they go to LDS.  What has no place, and what is NaN, is zero there: a probability of zero does not take a NaN away
    const auto prepare_values = [&](int turn, int base, bool page_there) {
      Values& v = shared.values[turn];
      constexpr int kScales = ValueChunk::kScales;
      // scales between which nothing has to be looked at: float16 holds their blocks, or they are no NaN
      constexpr uint32_t kLow = HALF ? 127 + narrow_low(VF) - kValuesUp : 0, kHigh = HALF ? 127 + narrow_high(VF) - kValuesUp : 254;
      if (EVEN) vc.unpack(value_shift);
      bool look = false;
#pragma unroll
      for (int s = 0; s < kScales; ++s) look |= vc.scale[s] - kLow > kHigh - kLow;
      const bool there = page_there && base + loader_key < k1;
      const uint64_t gone = __ballot(!there), any_look = __ballot(look && there);
      if (lane == 0) v.flags[wave] = gone != 0;
      if (!(gone | any_look)) return;
      if (lane == 0) v.gone[wave] = gone;
      constexpr int kEach = ValueChunk::kWords / kScales;
      bool any_none = false, any_wide = false;
#pragma unroll
      for (int s = 0; s < kScales; ++s) {
        const bool nan = vc.scale[s] == 255;
        bool zero = nan || !there;
        const uint64_t none_here = __ballot(nan && there);
        any_none |= none_here != 0;
        if (lane == 0) v.none[s][wave] = none_here;
        if (HALF) {
          // (zeros are zeros whatever their scale, which 2^kValuesUp times may be none)
          uint32_t bits = 0;
#pragma unroll
          for (int w = 0; w < kEach; ++w) bits |= vc.w[s * kEach + w];
          zero |= !(bits & (VF == kMxFp4 ? 0x77777777u : 0x7f7f7f7fu));
          any_wide |= __ballot(!zero && vc.scale[s] - kLow > kHigh - kLow) != 0;
        }
        if (zero) vc.scale[s] = 0;
#pragma unroll
        for (int w = 0; w < kEach; ++w) vc.w[s * kEach + w] = zero ? 0 : vc.w[s * kEach + w];
      }
      if (lane == 0) v.flags[wave] = (gone != 0) | any_none << 1 | any_wide << 2;
    };
    const auto store_values = [&](int turn, int st) {
      uint8_t* const to = shared.values[turn].rows + loader_key * kValueRow + part * 16 * kChunk + 16 * st;
      if constexpr (HALF) *reinterpret_cast<at_h8*>(to) = attention_halves8<VF>(vc.words(st), vc.scale_of(st, kValuesUp));
      else *reinterpret_cast<at_b8*>(to) = vc.values(st);
    };

    m = -INFINITY, l = 0.0f;
    float most = -INFINITY;
#pragma unroll
    for (int d = 0; d < DB; ++d) o[d] = at_f16{};
    // S^T: keys 32 i + 8 (e / 4) + 4 half + e % 4 of query lane % 32, element 16 i + e of a lane's 32.
    struct Scores {
      at_f16 s[2];
    };
    const auto key_of = [&](int turn, int k) {  // operand k of the scores' products: keys 32 (k % 2) on, columns 16 (k / 2) on
      return *reinterpret_cast<const at_b8*>(shared.keys[turn] + (32 * (k % 2) + (lane & 31)) * kKeyRow + 32 * (k / 2) + 16 * half);
    };
    const auto score = [&](Scores& s, int k, const at_b8& key) {
      if (k < 2) s.s[k] = at_f16{};
#pragma unroll
      for (int p = PIECES - 1; p >= 0; --p) s.s[k % 2] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(key, q[p][k / 2], s.s[k % 2], 0, 0, 0);
    };
    const auto value_of = [&](int turn, int k) {  // operand k of the results' products: keys 16 (k / DB) on, columns 32 (k % DB) on
      union {
        at_s4 half[2];
        at_b8 whole;
      } v;
      const uint8_t* from = shared.values[turn].rows + (4 * half + (lane & 15) / 4) * kValueRow + 2 * ((lane & 16) + 4 * (lane & 3)) + 16 * (k / DB) * kValueRow + 64 * (k % DB);
      v.half[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((at_lds_s4*)from);
      v.half[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((at_lds_s4*)(from + 8 * kValueRow));
      return v.whole;
    };
    const auto result = [&](at_f16& sum, const at_b8& value, const mx_u4& p) {
      if constexpr (HALF) sum = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(at_h8, value), __builtin_bit_cast(at_h8, p), sum, 0, 0, 0);
      else sum = __builtin_amdgcn_mfma_f32_32x32x16_bf16(value, __builtin_bit_cast(at_b8, p), sum, 0, 0, 0);
    };
    const auto most_of = [&](const Scores& s) {
      float most = s.s[0][0];
#pragma unroll
      for (int e = 1; e < 32; ++e) most = fmaxf(most, s.s[e / 16][e % 16]);
      return most;
    };
    const auto seen_by_wave = [&](int base) { return base < wave_end && base + kTile > wave_low; };
    const auto all_scores = [&](int turn, Scores& s) {
#pragma unroll
      for (int k = 0; k < kProducts; ++k) score(s, k, key_of(turn, k));
    };
    bool values_there = false, keys_there = false;
    int64_t next_place = 0;
    // values of the next tile and keys of the one after it into LDS, those behind them under way; in kForward parts
    constexpr int kForward = 2 * kChunk + 1;
    const auto forward = [&](int turn, int base, int k) {
      if (k == 0) prepare_values(turn ^ 1, base + kTile, values_there);
      if (k >= 1 && k <= kChunk) store_values(turn ^ 1, k - 1);
      if (k > kChunk && k <= 2 * kChunk) store_keys(turn, k - 1 - kChunk);
    };
    const auto load_next = [&](int base) {
      values_there = keys_there;
      load_values(next_place);
      next_place = place_of(base + 3 * kTile, keys_there);
      load_keys(next_place);
      look_up(base + 4 * kTile);
    };
    // what a tile's rows do not see is minus infinity; the largest of the rest
    const auto hide = [&](int base, const Values& b, Scores& s, bool any_gone) {
      if (base < wave_all_low || base + kTile > wave_all_end || any_gone) {
        const int from = low - base, to = end - base;
        uint64_t seen = from >= kTile || to <= 0 || from >= to ? 0 : (from <= 0 ? ~0ull : ~0ull << from) & (to >= kTile ? ~0ull : ~(~0ull << to));
        if (any_gone) {
#pragma unroll 1
          for (int at = 0; at < kTile; ++at)
            if ((b.flags[at / kKeysAWave] & 1) && (b.gone[at / kKeysAWave] >> (PARTS * (at % kKeysAWave)) & 1)) seen &= ~(1ull << at);
        }
        seen >>= 4 * half;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (!((uint32_t)(seen >> (32 * i)) >> (8 * (e / 4) + e % 4) & 1)) s.s[i][e] = -INFINITY;
        most = pair_max(most_of(s));
      }
    };
    const auto raise = [&] {
      // m, 2^kDown below the maximum, is raised only where scores are 2^kSlack times beyond that: the sums hold it
      constexpr float kDown = HALF ? kHead : 0.0f, kSlack = HALF ? 2.0f : 6.0f;
      most *= factor;
      if (__ballot(most - m > kDown + kSlack)) {
        // (from larger maxima the difference may be rounded to 2^16 and more)
        const float raised = fmaxf(m, fabsf(most) < 0x1p22f ? most - kDown : most), fade = raised == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - raised);
        m = raised;
        l *= fade;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
          for (int e = 0; e < 16; ++e) o[d][e] *= fade;
      }
    };
    // The product in the exponent is not rounded, the maximum's was: half a step of m apart, which 2^16 keeps at 2^-8.  Larger scores are rounded like the maximum.  What they are to
    // be multiplied by, and what is added
    const auto exponent = [&](Scores& s) -> float2 {
      const float zero = m == -INFINITY ? 0.0f : -m;
      const bool far = __ballot(fabsf(zero) >= 0x1p16f);
      if (far) [[unlikely]] {
#pragma unroll
        for (int e = 0; e < 32; ++e) s.s[e / 16][e % 16] *= factor;
      }
      const float times = far ? 1.0f : factor;
      return make_float2(times, zero);
    };
    // NaN for the queries that see such a value, and for no other: block d lies in part d PARTS / DB
    const auto set_none = [&](int base, const Values& b) {
      constexpr int kScales = ValueChunk::kScales;
      for (int at = 0; at < kTile; ++at) {
        if (!(b.flags[at / kKeysAWave] & 2)) continue;
        uint32_t bits[kScales], any = 0;
#pragma unroll
        for (int x = 0; x < kScales; ++x) {
          bits[x] = (uint32_t)(b.none[x][at / kKeysAWave] >> (PARTS * (at % kKeysAWave))) & ((1 << PARTS) - 1);
          any |= bits[x];
        }
        if (!any) continue;
        const bool seen = base + at >= low && base + at < end;
#pragma unroll
        for (int d = 0; d < DB; ++d) {
          const bool nan = bits[d % kScales] >> (d * PARTS / DB) & 1;
#pragma unroll
          for (int e = 0; e < 16; ++e) o[d][e] = nan && seen ? NAN : o[d][e];
        }
      }
    };
    // Tile `base`, whose scores and their largest are there: its share of the results; and the scores of the next one.  In the order that it is written in
    // (the fences hold the compiler to it): operands are read kAhead products ahead, the next tile's scores alternate with this one's
    // exponentials, this one's results with what is under way and the next one's maximum.
    const auto step = [&](int base, int turn, Scores& s, Scores& next) {
      const Values& b = shared.values[turn];
      const uint64_t flags64 = *reinterpret_cast<const uint64_t*>(b.flags);
      const auto any_flag = [&] { return __builtin_amdgcn_readfirstlane((uint32_t)flags64 | (uint32_t)(flags64 >> 32)); };
      uint32_t flags;
      if (seen_by_wave(base)) {
        at_b8 keys[kAhead], values[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) keys[k] = key_of(turn ^ 1, k);
        const auto next_score = [&](int k) {
          score(next, k, keys[k % kAhead]);
          if (k + kAhead < kProducts) keys[k % kAhead] = key_of(turn ^ 1, k + kAhead);
          else values[k % kAhead] = value_of(turn, k + kAhead - kProducts);
        };
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int k = 0; k < kLead; ++k) {
          next_score(k);
          __builtin_amdgcn_sched_barrier(0);
        }
        flags = any_flag();
        const bool any_gone = flags & 0x01010101, any_none = flags & 0x02020202;
        hide(base, b, s, any_gone);
        raise();
        const auto [times, zero] = exponent(s);
        constexpr int kPieces = HALF ? 1 : 2;
        mx_u4 pr[kPieces][4];
        float x[2];
        const auto exponentials = [&](int e) {  // elements e and e + 1
#pragma unroll
          for (int j = 0; j < 2; ++j) x[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(s.s[(e + j) / 16][(e + j) % 16], times, zero));
          asm volatile("" : "+v"(x[0]), "+v"(x[1]));  // (here, not where they are used)
        };
        const auto probabilities = [&](int e) {
          l += x[0] + x[1];
          __bf16 piece[2][kPieces];
          if constexpr (!HALF) {
#pragma unroll
            for (int j = 0; j < 2; ++j) attention_split<kPieces>(x[j], piece[j]);
          }
#pragma unroll
          for (int k = 0; k < kPieces; ++k) {
            uint32_t pair = HALF ? __builtin_bit_cast(uint32_t, at_h2{(_Float16)x[0], (_Float16)x[1]}) : __builtin_bit_cast(uint32_t, at_b2{piece[0][k], piece[1][k]});
            asm volatile("" : "+v"(pair), "+v"(l));
            pr[k][e / 8][e % 8 / 2] = pair;
          }
        };
        // share k of kProducts of the 32 elements: the last pair's probabilities, the next pair's exponentials
        const auto some = [&](int k) {
#pragma unroll
          for (int e = 32 * k / kProducts; e < 32 * (k + 1) / kProducts; ++e)
            if (e % 2) {
              if (e > 1) probabilities(e - 3);
              exponentials(e - 1);
            }
        };
        // a wavefront that has its exponentials under way goes first on its SIMD: the two are not at the same place then (prompt of 8192 579 -> 566 us)
        __builtin_amdgcn_s_setprio(1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int k = kLead; k < kProducts; ++k) {
          next_score(k);
          some(k - kLead);
          __builtin_amdgcn_sched_barrier(0);
        }
        most = -INFINITY;
#pragma unroll
        for (int k = 0; k < kProducts; ++k) {
          const int u = k / DB, d = k % DB;
#pragma unroll
          for (int p = kPieces - 1; p >= 0; --p) result(o[d], values[k % kAhead], pr[p][u]);
          if (k + kAhead < kProducts) values[k % kAhead] = value_of(turn, k + kAhead);
          if (k < kLead) some(k + kProducts - kLead);
          if (k == kLead) probabilities(30);
          if (k >= kLead) {
            constexpr int kRest = kProducts - kLead;
            const int at = k - kLead;
#pragma unroll
            for (int f = kForward * at / kRest; f < kForward * (at + 1) / kRest; ++f) forward(turn, base, f);
#pragma unroll
            for (int e = 32 * at / kRest; e < 32 * (at + 1) / kRest; ++e) most = fmaxf(most, next.s[e / 16][e % 16]);
            asm volatile("" : "+v"(most));
          }
          __builtin_amdgcn_sched_barrier(0);
        }
        __builtin_amdgcn_s_setprio(0);
        most = pair_max(most);
        if (any_none) set_none(base, b);
      } else {
        flags = any_flag();
        if (seen_by_wave(base + kTile)) {
          all_scores(turn ^ 1, next);
          most = pair_max(most_of(next));
        }
#pragma unroll
        for (int k = 0; k < kForward; ++k) forward(turn, base, k);
      }
      load_next(base);
      __syncthreads();
      return !HALF || !(flags & 0x04040404);  // (the same in all wavefronts)
    };
    // The same for values that float16 does not hold.
    const auto plain_step = [&](int base, int turn) {
      const Values& b = shared.values[turn];
      const bool seen = seen_by_wave(base);
      Scores s;
      if (seen) {
        all_scores(turn, s);
        most = pair_max(most_of(s));
      }
      __syncthreads();  // (what follows writes over these keys)
#pragma unroll
      for (int k = 0; k < kForward; ++k) forward(turn, base, k);
      if (seen) {
        const uint64_t flags64 = *reinterpret_cast<const uint64_t*>(b.flags);
        const uint32_t flags = __builtin_amdgcn_readfirstlane((uint32_t)flags64 | (uint32_t)(flags64 >> 32));
        hide(base, b, s, flags & 0x01010101);
        raise();
        const auto [times, zero] = exponent(s);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          at_b8 p[2];
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s.s[u / 2][8 * (u % 2) + j], times, zero));
            l += x;
            __bf16 piece[2];
            attention_split<2>(x, piece);
            p[0][j] = piece[0], p[1][j] = piece[1];
          }
#pragma unroll
          for (int d = 0; d < DB; ++d) {
            const at_b8 v = value_of(turn, u * DB + d);
#pragma unroll
            for (int k = 1; k >= 0; --k) o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, p[k], o[d], 0, 0, 0);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
        if (flags & 0x02020202) set_none(base, b);
      }
      load_next(base);
      __syncthreads();
    };

    if (k0 < k1) {
      if (threadIdx.x < 16) shared.values[threadIdx.x / 8].flags[threadIdx.x % 8] = 0;  // (of wavefronts that there are not, too)
      __syncthreads();
      // what does not wait for one another, together
      int32_t pages[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        look_up(k0 + j * kTile);
        pages[j] = next_page;
      }
      KeyChunk early[2];
      ValueChunk first;
      bool early_there = false;
#pragma unroll
      for (int j = 0; j < 3; ++j) {
        next_page = pages[j];
        next_place = place_of(k0 + j * kTile, j == 0 ? early_there : j == 1 ? values_there : keys_there);
        load_keys(next_place);
        if (j < 2) load_values(next_place);
        if (j < 2) early[j] = kc;
        if (j == 0) first = vc;
      }
      next_page = pages[3];
      const KeyChunk last = kc;
      const ValueChunk second = vc;
      vc = first;
      prepare_values(0, k0, early_there);
#pragma unroll
      for (int st = 0; st < kChunk; ++st) store_values(0, st);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        kc = early[j];
#pragma unroll
        for (int st = 0; st < kChunk; ++st) store_keys(j, st);
      }
      kc = last;
      vc = second;
      __syncthreads();
      if constexpr (!HALF && many_halves(TYPE, DB)) {
        for (int base = k0; base < k1; base += 2 * kTile) {
          plain_step(base, 0);
          if (base + kTile < k1) plain_step(base + kTile, 1);
        }
      } else {
        Scores even, odd;
        if (seen_by_wave(k0)) {
          all_scores(0, even);
          most = pair_max(most_of(even));
        }
        __syncthreads();  // (the first step writes over these keys)
        for (int base = k0; base < k1; base += 2 * kTile) {
          if (!step(base, 0, even, odd)) return false;
          if (base + kTile < k1 && !step(base + kTile, 1, odd, even)) return false;
        }
      }
    }
    return true;
  };
  const bool half_values = many_halves(TYPE, DB) && go_through.template operator()<many_halves(TYPE, DB)>();
  if (!half_values) (void)go_through.template operator()<false>();

  // a lane has columns 32 d + 8 i + 4 half .. + 3 of its query
  const float sum = pair_sum(l), back = half_values ? 1.0f / (1 << kValuesUp) : 1.0f;
  if (!row_there) return;
  const int64_t out_row = (int64_t)(span.first + token) * a.heads + q_head;
  if (run.runs == 1) {
    const float inverse = sum > 0.0f || sum != sum ? back / sum : 0.0f;
    E* out = static_cast<E*>(a.out) + out_row * c.dim;
    typedef E elements __attribute__((ext_vector_type(4)));
    typedef elements elements_any __attribute__((aligned(sizeof(E))));
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int col = 32 * d + 8 * i + 4 * half;
        elements y;
#pragma unroll
        for (int j = 0; j < 4; ++j) y[j] = (E)(o[d][4 * i + j] * inverse);
        if (col + 4 <= c.dim) {
          *reinterpret_cast<elements_any*>(out + col) = y;
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (col + j < c.dim) out[col + j] = y[j];
        }
      }
    if (half == 0) {
      if (a.lse) a.lse[out_row] = sum == 0.0f ? -INFINITY : (m + __builtin_amdgcn_logf(sum)) * kAttentionLn2;
      work.joins[out_row] = make_int2(0, 1);
    }
    return;
  }
  const int64_t first = run.slot + ((int64_t)tile * c.kv_heads + head) * run.runs, slot = first + split;
  if (slot < 0 || slot >= slots) return;  // (only offsets that break the contract)
  const int row = wave * 32 + (lane & 31);
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *reinterpret_cast<at_f4*>(work.partial + (slot * ROWS + row) * D + 32 * d + 8 * i + 4 * half) = at_f4{o[d][4 * i], o[d][4 * i + 1], o[d][4 * i + 2], o[d][4 * i + 3]} * back;
  if (half == 0) {
    work.stats[slot * ROWS + row] = make_float2(m, sum);
    if (split == 0) work.joins[out_row] = make_int2((int)(first * ROWS + row), run.runs);
  }
}

template <int TYPE, int KF, int VF, int DB, int WAVES, bool EVEN>
hipError_t launch_even(const CacheArgs& c, const AttentionArgs& a, const AttentionWork& work, hipStream_t st) {
  constexpr int ROWS = 32 * WAVES;
  using Shared = ManyShared<DB, WAVES>;
  constexpr size_t bytes = sizeof(Shared);
  static_assert(many_key_row(DB) % 16 == 0 && many_value_row(DB) % 16 == 0 && sizeof(typename Shared::Values) % 16 == 0, "whole vectors");
  static_assert(bytes <= 160 * 1024);
  static_assert(ROWS == attention_many_rows(TYPE, DB), "partials are laid out by it");
  auto* kernel = many_kernel<TYPE, KF, VF, DB, WAVES, EVEN>;
  static std::atomic<uint64_t> raised{0};
  if (const hipError_t e = raise_lds_limit(reinterpret_cast<const void*>(kernel), (int)bytes, raised); e != hipSuccess) return e;
  const int group = a.heads / c.kv_heads;
  const int64_t units = ((int64_t)a.T * group / ROWS + (c.seqs < a.T ? c.seqs : a.T)) * c.kv_heads;
  if (const hipError_t e = launch_plan<ROWS, kTile, kAttentionManyRuns>(c, a, work, st); e != hipSuccess) return e;
  return launch_kernel(kernel, dim3((uint32_t)(units + kAttentionManyRuns)), dim3(64 * WAVES), bytes, st, c, a, work, (uint32_t)group);
}
template <int TYPE, int KF, int VF, int DB, int WAVES>
hipError_t launch(const CacheArgs& c, const AttentionArgs& a, const AttentionWork& work, hipStream_t st) {
  constexpr int keys_a_wave = kTile / WAVES;
  return attention_even(c, keys_a_wave) ? launch_even<TYPE, KF, VF, DB, WAVES, true>(c, a, work, st) : launch_even<TYPE, KF, VF, DB, WAVES, false>(c, a, work, st);
}
template <int TYPE, int KF, int VF>
hipError_t with_dim(const CacheArgs& c, const AttentionArgs& a, const AttentionWork& work, hipStream_t st) {
  switch (attention_blocks(c.dim)) {
    case 2: return launch<TYPE, KF, VF, 2, attention_many_waves(TYPE, 2)>(c, a, work, st);
    case 4: return launch<TYPE, KF, VF, 4, attention_many_waves(TYPE, 4)>(c, a, work, st);
  }
  return launch<TYPE, KF, VF, 8, attention_many_waves(TYPE, 8)>(c, a, work, st);
}
template <int TYPE>
hipError_t with_formats(const CacheArgs& c, const AttentionArgs& a, const AttentionWork& work, hipStream_t st) {
  if (c.k_format == kMxFp4) return c.v_format == kMxFp4 ? with_dim<TYPE, kMxFp4, kMxFp4>(c, a, work, st) : with_dim<TYPE, kMxFp4, kMxFp8>(c, a, work, st);
  return c.v_format == kMxFp4 ? with_dim<TYPE, kMxFp8, kMxFp4>(c, a, work, st) : with_dim<TYPE, kMxFp8, kMxFp8>(c, a, work, st);
}

}  // namespace

}  // namespace hago
