// Attention over a paged cache of microscaled keys and values, many rows a sequence: chunks and prompts.
//
// The matrix unit bounds it.  A workgroup is one (sequence, tile of rows, head of the cache) and a run of keys; its rows are the queries of all heads
// that share those keys, 32 or 64 a wavefront.  Keys and values of 64 positions at a time become bfloat16 once for all of them, on their way from
// memory through registers into LDS, two tiles deep with one barrier a tile; the conversions are hidden behind the products.  S^T = K Q^T leaves a
// query's scores in two lanes' registers, as the operand of O^T = V^T P^T, so that the softmax needs one lane exchange and nothing of it goes
// through LDS; values are read transposed from there.
#include "mx_attention.h"

namespace hago {

namespace {

typedef float at_f16 __attribute__((ext_vector_type(16)));

constexpr int kTile = 64;  // keys

// Of a lane and its partner (lane ^ 32), which hold the two halves of a query's keys.
__device__ __forceinline__ float pair_max(float v) { return fmaxf(v, __shfl_xor(v, 32)); }
__device__ __forceinline__ float pair_sum(float v) { return v + __shfl_xor(v, 32); }

template <int TYPE, int KF, int VF, int DB, int RG, int WAVES>
__global__ __launch_bounds__(64 * WAVES, WAVES / 4) void many_kernel(CacheArgs c, AttentionArgs a, AttentionWork work, int group, int share_of, int slots) {
  using E = typename MxElement<TYPE>::type;
  constexpr int PIECES = kAttentionPieces<TYPE>, D = 32 * DB, THREADS = 64 * WAVES, ROWS = 32 * RG * WAVES, STEPS = 2 * DB;
  constexpr int kKeyRow = 2 * D + 16, kValueRow = 2 * D + 64;  // bytes in LDS: neighbours on different banks, as they are read
  constexpr int kLoaders = 256;                                // threads that load a tile's keys, and its values
  using KeyChunk = AttentionChunk<KF, DB>;
  using ValueChunk = AttentionChunk<VF, DB>;
  struct Buffer {
    uint8_t keys[kTile * kKeyRow];
    uint8_t values[kTile * kValueRow];
    uint64_t none[2][4];  // bit 4 (key % 16) + part of [block of the part][key / 16]: a value's block that stands for NaN
    uint64_t gone[4];     // the key has no place
  };
  extern __shared__ __align__(16) uint8_t lds[];
  Buffer* const buffers = reinterpret_cast<Buffer*>(lds);

  AttentionRun run;
  if (!attention_run<THREADS, ROWS, kTile>(c, a, group, share_of, blockIdx.x, run)) return;
  const AttentionSpan span = attention_span(c, a, run.seq);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), half = lane / 32;
  const int tiles = (int)(((int64_t)span.rows * group + ROWS - 1) / ROWS);
  // (the last rows see the most keys: they come first)
  const int head = run.local % c.kv_heads, tile = tiles - 1 - run.local / c.kv_heads % tiles, split = run.local / c.kv_heads / tiles;
  const int blocks = (c.dim + 31) / 32;
  // scores times a factor that is not negative: the queries take its sign
  const float factor = fabsf(a.scale) * kAttentionLog2e;
  const int64_t all_rows = (int64_t)span.rows * group;
  const auto end_of = [&](int i) {
    const int64_t p = span.position + i + 1;
    return !a.causal || p > span.high ? span.high : p < 0 ? 0 : (int)p;
  };
  const auto low_of = [&](int i) {
    const int64_t p = a.window ? span.position + i - a.window + 1 : 0;
    return p < 0 ? 0 : p < span.high ? (int)p : span.high;
  };

  // this lane's queries
  at_b8 q[RG][PIECES][STEPS];
  int low[RG], end[RG];
#pragma unroll
  for (int g = 0; g < RG; ++g) {
    const int64_t index = (int64_t)tile * ROWS + (wave * RG + g) * 32 + (lane & 31);
    const bool row_there = index < all_rows;
    const int token = row_there ? (int)(index / group) : 0;
    const int64_t t = span.first + token;
    const int q_head = head * group + (int)(index - (int64_t)token * group);
    low[g] = row_there ? low_of(token) : 0;
    end[g] = row_there ? end_of(token) : 0;
#pragma unroll
    for (int st = 0; st < STEPS; ++st) {
      const int col = 16 * st + 8 * half;
      float x[8];
      if (row_there && col < c.dim)
        mx_load8<TYPE>(static_cast<const E*>(a.q.data) + t * a.q.row + (int64_t)q_head * a.q.head + col, c.dim - col, x);
      else
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = 0.0f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        __bf16 p[PIECES];
        attention_split<PIECES>(a.scale < 0 ? -x[i] : x[i], p);
#pragma unroll
        for (int k = 0; k < PIECES; ++k) q[g][k][st][i] = p[k];
      }
    }
  }

  // the keys of this run that any row of the workgroup sees, of a wavefront, and that all of its rows see
  const int64_t last_row = ((int64_t)tile + 1) * ROWS < all_rows ? ((int64_t)tile + 1) * ROWS - 1 : all_rows - 1;
  const int start = span.low & ~15, all_blocks = span.high > span.low ? (span.high - start + kTile - 1) / kTile : 1;
  const int each = (all_blocks + run.runs - 1) / run.runs;
  const int64_t run_first = start + (int64_t)split * each * kTile, run_end = run_first + (int64_t)each * kTile;
  int k0 = run_first < span.high ? (int)run_first : span.high, k1 = run_end < span.high ? (int)run_end : span.high;
  const int tile_low = low_of((int)((int64_t)tile * ROWS / group)) & ~15, tile_end = end_of((int)(last_row / group));
  if (k0 < tile_low) k0 = tile_low;
  if (k1 > tile_end) k1 = tile_end;
  const int64_t wave_first = (int64_t)tile * ROWS + wave * RG * 32;
  const int64_t wave_last = wave_first + RG * 32 - 1 < last_row ? wave_first + RG * 32 - 1 : last_row;
  const bool wave_there = wave_first <= last_row;
  const int wave_low = wave_there ? low_of((int)(wave_first / group)) : 0, wave_end = wave_there ? end_of((int)(wave_last / group)) : 0;
  // (rows behind the last one see nothing, but nothing of theirs is kept: they may as well see all)
  const int wave_all_low = wave_there ? low_of((int)(wave_last / group)) : 0, wave_all_end = wave_there ? end_of((int)(wave_first / group)) : 0;

  // loaders: four threads a key
  const int loader = threadIdx.x & (kLoaders - 1), loader_key = loader / 4, part = loader & 3;
  const bool loads_keys = threadIdx.x < kLoaders, loads_values = WAVES == 4 || !loads_keys;
  int32_t next_page;
  KeyChunk kc;
  ValueChunk vc;
  bool there;
  const auto look_up = [&](int base) {  // the page of this thread's key of a tile
    const int key = base + loader_key;
    next_page = key < k1 ? c.table[run.seq * c.table_stride + cache_page_of(c, (uint32_t)key)] : -1;
  };
  const auto load = [&](int base) {
    const uint32_t key = base + loader_key;
    there = (uint32_t)next_page < (uint32_t)c.pages;
    const int64_t place = there ? ((int64_t)next_page * c.kv_heads + head) * c.page + (key - cache_page_of(c, key) * (uint32_t)c.page) : 0;
    if (loads_keys) kc.load(c.k_codes, c.k_scales, place, blocks, part);
    if (loads_values) vc.load(c.v_codes, c.v_scales, place, blocks, part);
  };
  const auto store = [&](Buffer& b) {
    if (loads_keys) {
#pragma unroll
      for (int st = 0; st < DB; ++st) *reinterpret_cast<at_b8*>(b.keys + loader_key * kKeyRow + part * 16 * DB + 16 * st) = kc.values(st);
    }
    if (loads_values) {
      constexpr int kScales = ValueChunk::kScales, kEach = ValueChunk::kWords / kScales;
#pragma unroll
      for (int s = 0; s < kScales; ++s) {
        const bool nan = vc.scale[s] == 255, zero = nan || !there;
        const uint64_t none = __ballot(nan && there);
        if (lane == 0) b.none[s][wave & 3] = none;
        if (zero) vc.scale[s] = 0;
#pragma unroll
        for (int w = 0; w < kEach; ++w) vc.w[s * kEach + w] = zero ? 0 : vc.w[s * kEach + w];
      }
      const uint64_t gone = __ballot(!there);
      if (lane == 0) b.gone[wave & 3] = gone;
#pragma unroll
      for (int st = 0; st < DB; ++st) *reinterpret_cast<at_b8*>(b.values + loader_key * kValueRow + part * 16 * DB + 16 * st) = vc.values(st);
    }
  };

  float m[RG], l[RG];
  at_f16 o[RG][DB];
#pragma unroll
  for (int g = 0; g < RG; ++g) {
    m[g] = -INFINITY, l[g] = 0.0f;
#pragma unroll
    for (int d = 0; d < DB; ++d) o[g][d] = at_f16{};
  }

  if (k0 < k1) {
    look_up(k0);
    load(k0);
    look_up(k0 + kTile);
    store(buffers[0]);
    load(k0 + kTile);
    look_up(k0 + 2 * kTile);
  }
  __syncthreads();
  for (int base = k0, turn = 0; base < k1; base += kTile, turn ^= 1) {
    const Buffer& b = buffers[turn];
    if (base < wave_end && base + kTile > wave_low) {
      // S^T: keys 32 i + 8 (e / 4) + 4 half + e % 4 of query lane % 32
      at_f16 s[RG][2];
#pragma unroll
      for (int g = 0; g < RG; ++g) s[g][0] = s[g][1] = at_f16{};
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int st = 0; st < STEPS; ++st) {
          const at_b8 k = *reinterpret_cast<const at_b8*>(b.keys + (32 * i + (lane & 31)) * kKeyRow + 32 * st + 16 * half);
#pragma unroll
          for (int g = 0; g < RG; ++g)
#pragma unroll
            for (int p = PIECES - 1; p >= 0; --p) s[g][i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, q[g][p][st], s[g][i], 0, 0, 0);
        }
      const uint64_t any_gone = b.gone[0] | b.gone[1] | b.gone[2] | b.gone[3];
      const uint32_t gone32 = __builtin_amdgcn_readfirstlane((uint32_t)any_gone | (uint32_t)(any_gone >> 32));
      if (base < wave_all_low || base + kTile > wave_all_end || gone32) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const int at = 32 * i + 8 * (e / 4) + 4 * half + e % 4, key = base + at;
            const bool gone = b.gone[at / 16] >> (4 * (at % 16)) & 1;
#pragma unroll
            for (int g = 0; g < RG; ++g)
              if (key < low[g] || key >= end[g] || gone) s[g][i][e] = -INFINITY;
          }
      }
      // softmax: the maximum is raised only where scores are 2^kSlack times beyond it, the sums hold that
      constexpr float kSlack = 6.0f;
      at_b8 pr[RG][PIECES][4];
#pragma unroll
      for (int g = 0; g < RG; ++g) {
        float most = s[g][0][0];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int e = 0; e < 16; ++e) most = fmaxf(most, s[g][i][e]);
        most = pair_max(most) * factor;
        if (__ballot(most > m[g] + kSlack)) {
          const float raised = fmaxf(m[g], most), fade = raised == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m[g] - raised);
          m[g] = raised;
          l[g] *= fade;
#pragma unroll
          for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int e = 0; e < 16; ++e) o[g][d][e] *= fade;
        }
        const float zero = m[g] == -INFINITY ? 0.0f : -m[g];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[g][i][e], factor, zero));
            l[g] += p;
            __bf16 piece[PIECES];
            attention_split<PIECES>(p, piece);
#pragma unroll
            for (int k = 0; k < PIECES; ++k) pr[g][k][2 * i + e / 8][e % 8] = piece[k];
          }
      }
      // O^T
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int d = 0; d < DB; ++d) {
          union {
            at_s4 half[2];
            at_b8 whole;
          } v;
          const int row = 16 * u + 4 * half + (lane & 15) / 4, col = 32 * d + (lane & 16) + 4 * (lane & 3);
          v.half[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((at_lds_s4*)(b.values + row * kValueRow + 2 * col));
          v.half[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((at_lds_s4*)(b.values + (row + 8) * kValueRow + 2 * col));
#pragma unroll
          for (int g = 0; g < RG; ++g)
#pragma unroll
            for (int p = PIECES - 1; p >= 0; --p) o[g][d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v.whole, pr[g][p][u], o[g][d], 0, 0, 0);
        }
      constexpr int kScales = ValueChunk::kScales;
      uint64_t any_none = 0;
#pragma unroll
      for (int x = 0; x < kScales; ++x) any_none |= b.none[x][0] | b.none[x][1] | b.none[x][2] | b.none[x][3];
      if (__builtin_amdgcn_readfirstlane((uint32_t)any_none | (uint32_t)(any_none >> 32))) {
        // NaN for the queries that see such a value, and for no other: block d is part 4 d / DB, or half of it
        for (int at = 0; at < kTile; ++at) {
          const uint32_t bits0 = (uint32_t)(b.none[0][at / 16] >> (4 * (at % 16))) & 15, bits1 = kScales > 1 ? (uint32_t)(b.none[kScales - 1][at / 16] >> (4 * (at % 16))) & 15 : 0;
          if (!(bits0 | bits1)) continue;
#pragma unroll
          for (int g = 0; g < RG; ++g) {
            const bool seen = base + at >= low[g] && base + at < end[g];
#pragma unroll
            for (int d = 0; d < DB; ++d) {
              const bool nan = (DB == 8 && d % 2 ? bits1 : bits0) >> (DB == 2 ? 2 * d : DB == 4 ? d : d / 2) & 1;
#pragma unroll
              for (int e = 0; e < 16; ++e) o[g][d][e] = nan && seen ? NAN : o[g][d][e];
            }
          }
        }
      }
    }
    if (base + kTile < k1) {
      store(buffers[turn ^ 1]);
      load(base + 2 * kTile);
      look_up(base + 3 * kTile);
    }
    __syncthreads();
  }

  // a lane has columns 32 d + 8 i + 4 half .. + 3 of its queries
#pragma unroll
  for (int g = 0; g < RG; ++g) {
    const float sum = pair_sum(l[g]);
    const int64_t index = (int64_t)tile * ROWS + (wave * RG + g) * 32 + (lane & 31);
    if (index >= all_rows) continue;
    const int64_t out_row = (span.first + index / group) * a.heads + head * group + index % group;
    if (run.runs == 1) {
      const float inverse = sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f;
      E* out = static_cast<E*>(a.out) + out_row * c.dim;
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (32 * d + 8 * i + 4 * half + j < c.dim) out[32 * d + 8 * i + 4 * half + j] = (E)(o[g][d][4 * i + j] * inverse);
      if (half == 0) {
        if (a.lse) a.lse[out_row] = sum == 0.0f ? -INFINITY : (m[g] + __builtin_amdgcn_logf(sum)) * kAttentionLn2;
        work.joins[out_row] = make_int2(0, 1);
      }
      continue;
    }
    const int64_t first = run.slot + ((int64_t)tile * c.kv_heads + head) * run.runs, slot = first + split;
    if (slot < 0 || slot >= slots) continue;  // (only offsets that break the contract)
    const int row = (wave * RG + g) * 32 + (lane & 31);
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<at_f4*>(work.partial + (slot * ROWS + row) * D + 32 * d + 8 * i + 4 * half) =
            at_f4{o[g][d][4 * i], o[g][d][4 * i + 1], o[g][d][4 * i + 2], o[g][d][4 * i + 3]};
    if (half == 0) {
      work.stats[slot * ROWS + row] = make_float2(m[g], sum);
      if (split == 0) work.joins[out_row] = make_int2((int)(first * ROWS + row), run.runs);
    }
  }
}

template <int TYPE, int KF, int VF, int DB, int RG, int WAVES>
hipError_t launch(const CacheArgs& c, const AttentionArgs& a, const AttentionWork& work, hipStream_t st) {
  constexpr int D = 32 * DB, ROWS = 32 * RG * WAVES;
  constexpr size_t bytes = 2 * (kTile * (4 * D + 80) + 96);
  static_assert(ROWS == attention_many_rows(DB), "partials are laid out by it");
  auto* kernel = many_kernel<TYPE, KF, VF, DB, RG, WAVES>;
  static std::atomic<uint64_t> raised{0};
  if (const hipError_t e = raise_lds_limit(reinterpret_cast<const void*>(kernel), (int)bytes, raised); e != hipSuccess) return e;
  const int group = a.heads / c.kv_heads, share_of = kAttentionManyRuns;
  const int64_t units = ((int64_t)a.T * group / ROWS + (c.seqs < a.T ? c.seqs : a.T)) * c.kv_heads;
  return launch_kernel(kernel, dim3((uint32_t)(units + share_of)), dim3(64 * WAVES), bytes, st, c, a, work, group, share_of, 2 * share_of);
}
template <int TYPE, int KF, int VF>
hipError_t with_dim(const CacheArgs& c, const AttentionArgs& a, const AttentionWork& work, hipStream_t st) {
  switch (attention_blocks(c.dim)) {
    case 2: return launch<TYPE, KF, VF, 2, kManyGroups<2>, kManyWaves<2>>(c, a, work, st);
    case 4: return launch<TYPE, KF, VF, 4, kManyGroups<4>, kManyWaves<4>>(c, a, work, st);
  }
  return launch<TYPE, KF, VF, 8, kManyGroups<8>, kManyWaves<8>>(c, a, work, st);
}
template <int TYPE>
hipError_t with_formats(const CacheArgs& c, const AttentionArgs& a, const AttentionWork& work, hipStream_t st) {
  if (c.k_format == kMxFp4) return c.v_format == kMxFp4 ? with_dim<TYPE, kMxFp4, kMxFp4>(c, a, work, st) : with_dim<TYPE, kMxFp4, kMxFp8>(c, a, work, st);
  return c.v_format == kMxFp4 ? with_dim<TYPE, kMxFp8, kMxFp4>(c, a, work, st) : with_dim<TYPE, kMxFp8, kMxFp8>(c, a, work, st);
}

}  // namespace

hipError_t launch_attention_many(const CacheArgs& c, const AttentionArgs& a, const AttentionWork& work, hipStream_t st) { return with_formats<kMxBf16>(c, a, work, st); }

}  // namespace hago
