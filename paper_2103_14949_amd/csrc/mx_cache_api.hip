// C ABI of the rotary positions and of the operators around a paged microscaled cache: argument validation (host only, before any
// launch) and dispatch.  See include/hago.h for the contract.
#include "../../include/hago.h"

#include <cmath>

#include "mx_cache.h"

namespace {

constexpr int64_t kI32Max = 2147483647ll, kMostHeads = 65536, kMostPositions = (1ll << 31) - (1 << 16), kMostElements = 1ll << 62;

int real_type(hago_dtype t) { return t == HAGO_F32 ? hago::kMxF32 : t == HAGO_BF16 ? hago::kMxBf16 : t == HAGO_F16 ? hago::kMxF16 : -1; }
size_t real_size(hago_dtype t) { return t == HAGO_F32 ? 4 : 2; }
bool is_format(hago_mx_format f) { return f == HAGO_MX_FP4 || f == HAGO_MX_FP8; }
hago_status from_hip(hipError_t e) { return e == hipSuccess ? HAGO_OK : HAGO_ERR_DEVICE; }

// a * b <= most, for a, b >= 0
bool product_fits(int64_t a, int64_t b, int64_t most) { return !a || b <= most / a; }
// rows [T, heads, dim] at these distances lie within 2^62 elements
bool strides_fit(int64_t T, int64_t heads, int64_t row, int64_t head) {
  return row >= 0 && head >= 0 && product_fits(T, row, kMostElements) && product_fits(heads, head, kMostElements);
}

// What is wrong with a cache and sequences; OK, and whether there is anything to do.
hago_status check_cache(const hago_mx_cache* m, const hago_mx_sequences* s, int64_t T, hago_dtype t, bool& empty, hago::CacheArgs& c) {
  if (!m || !s) return HAGO_ERR_NULL;
  if (m->pages < 0 || m->pages > kI32Max || m->kv_heads < 0 || m->kv_heads > kMostHeads || m->page_size < 1 || m->dim < 0 || m->dim > hago::kCacheMostDim ||
      T < 0 || T > kI32Max || s->seqs < 0 || s->seqs > kI32Max - 1 || s->table_cols < 0 || s->table_stride < s->table_cols)
    return HAGO_ERR_SHAPE;
  if (m->page_size > kMostPositions || !product_fits(s->table_cols, m->page_size, kMostPositions) || !product_fits(s->seqs, s->table_stride, kMostElements) ||
      !product_fits(m->pages, m->kv_heads * m->page_size * (m->dim + 32), kMostElements))
    return HAGO_ERR_SHAPE;
  if (real_type(t) < 0) return HAGO_ERR_DTYPE;
  if (!is_format(m->k_format) || !is_format(m->v_format)) return HAGO_ERR_PARAM;
  empty = T == 0 || s->seqs == 0 || m->kv_heads == 0 || m->dim == 0;
  if (empty) return HAGO_OK;
  if (!s->lengths || !s->offsets || (s->table_cols && !s->table) || (m->pages && (!m->k_codes || !m->k_scales || !m->v_codes || !m->v_scales))) return HAGO_ERR_NULL;
  if (!hago::ptr_aligned(m->k_codes, 16) || !hago::ptr_aligned(m->v_codes, 16) || !hago::ptr_aligned(s->table, 4) || !hago::ptr_aligned(s->lengths, 4) ||
      !hago::ptr_aligned(s->offsets, 4))
    return HAGO_ERR_PARAM;
  c.k_codes = static_cast<uint8_t*>(m->k_codes);
  c.k_scales = static_cast<uint8_t*>(m->k_scales);
  c.v_codes = static_cast<uint8_t*>(m->v_codes);
  c.v_scales = static_cast<uint8_t*>(m->v_scales);
  c.table = s->table;
  c.lengths = s->lengths;
  c.offsets = s->offsets;
  c.table_stride = s->table_stride;
  c.pages = (int32_t)m->pages;
  c.page = (int32_t)m->page_size;
  c.kv_heads = (int32_t)m->kv_heads;
  c.dim = (int32_t)m->dim;
  c.seqs = (int32_t)s->seqs;
  c.places = m->pages ? (int32_t)(s->table_cols * m->page_size) : 0;
  // With 2^(l - 1) < page <= 2^l and f = floor(2^(31 + l) / page) + 1, position * f / 2^(31 + l) lies less than position / 2^(31 + l) < 1 / page
  // above position / page: it has the same whole part.
  int l = 0;
  while ((1ll << l) < m->page_size) ++l;
  c.page_shift = l;
  c.page_factor = (uint32_t)(((uint64_t)1 << (31 + l)) / (uint64_t)m->page_size + 1);
  c.k_format = m->k_format;
  c.v_format = m->v_format;
  return HAGO_OK;
}

}  // namespace

extern "C" {

hago_status hago_rope(const void* x, hago_dtype x_t, int64_t T, int64_t heads, int64_t dim, int64_t row_stride, int64_t head_stride, const int32_t* positions,
                      int64_t axes, const float* frequencies, const int32_t* axis, int64_t pairs, hago_rope_order order, void* out, int64_t out_row_stride,
                      int64_t out_head_stride, void* stream) {
  if (T < 0 || T > kI32Max || heads < 0 || heads > kMostHeads || dim < 0 || dim > hago::kRopeMostDim || pairs < 0 || 2 * pairs > dim || axes < 1 || axes > kI32Max)
    return HAGO_ERR_SHAPE;
  if (!strides_fit(T, heads, row_stride, head_stride) || !strides_fit(T, heads, out_row_stride, out_head_stride)) return HAGO_ERR_SHAPE;
  if (real_type(x_t) < 0) return HAGO_ERR_DTYPE;
  if (order != HAGO_ROPE_HALVES && order != HAGO_ROPE_NEIGHBOURS) return HAGO_ERR_PARAM;
  if (T == 0 || heads == 0 || dim == 0) return HAGO_OK;
  // rows of heads side by side, or heads of rows
  const bool rows_apart = T == 1 || out_row_stride >= (heads - 1) * out_head_stride + dim, heads_apart = heads == 1 || out_head_stride >= (T - 1) * out_row_stride + dim;
  if (!((rows_apart && (heads == 1 || out_head_stride >= dim)) || (heads_apart && (T == 1 || out_row_stride >= dim)))) return HAGO_ERR_SHAPE;
  if (!x || !out || (pairs && (!positions || !frequencies))) return HAGO_ERR_NULL;
  const size_t size = real_size(x_t);
  if (!hago::ptr_aligned(x, size) || !hago::ptr_aligned(out, size) || !hago::ptr_aligned(positions, 4) || !hago::ptr_aligned(frequencies, 4) || !hago::ptr_aligned(axis, 4))
    return HAGO_ERR_PARAM;
  if (out == x && ((T > 1 && out_row_stride != row_stride) || (heads > 1 && out_head_stride != head_stride))) return HAGO_ERR_PARAM;
  hago::RopeArgs r{};
  r.x = {x, row_stride, head_stride};
  r.out = out;
  r.out_row = out_row_stride;
  r.out_head = out_head_stride;
  r.positions = positions;
  r.frequencies = frequencies;
  r.axis = axis;
  r.T = (int32_t)T;
  r.heads = (int32_t)heads;
  r.dim = (int32_t)dim;
  r.pairs = (int32_t)pairs;
  r.axes = (int32_t)axes;
  r.interleaved = order == HAGO_ROPE_NEIGHBOURS;
  return from_hip(hago::launch_rope(r, real_type(x_t), static_cast<hipStream_t>(stream)));
}

hago_status hago_mx_cache_write(const hago_mx_cache* cache, const hago_mx_sequences* sequences, const void* k, int64_t k_row_stride, int64_t k_head_stride,
                                const void* v, int64_t v_row_stride, int64_t v_head_stride, hago_dtype x_t, int64_t T, void* k_values, void* v_values, void* stream) {
  hago::CacheArgs c{};
  bool empty = true;
  const hago_status s = check_cache(cache, sequences, T, x_t, empty, c);
  if (s != HAGO_OK) return s;
  if (!strides_fit(T, cache->kv_heads, k_row_stride, k_head_stride) || !strides_fit(T, cache->kv_heads, v_row_stride, v_head_stride)) return HAGO_ERR_SHAPE;
  if (empty) return HAGO_OK;
  if (!k || !v) return HAGO_ERR_NULL;
  const size_t size = real_size(x_t);
  if (!hago::ptr_aligned(k, size) || !hago::ptr_aligned(v, size) || !hago::ptr_aligned(k_values, size) || !hago::ptr_aligned(v_values, size)) return HAGO_ERR_PARAM;
  return from_hip(hago::launch_mx_cache_write(c, {k, k_row_stride, k_head_stride}, {v, v_row_stride, v_head_stride}, real_type(x_t), T, k_values, v_values,
                                              static_cast<hipStream_t>(stream)));
}

hago_status hago_mx_cache_read(const hago_mx_cache* cache, const hago_mx_sequences* sequences, hago_dtype out_t, int64_t T, void* k, void* v, void* stream) {
  hago::CacheArgs c{};
  bool empty = true;
  const hago_status s = check_cache(cache, sequences, T, out_t, empty, c);
  if (s != HAGO_OK || empty) return s;
  if (!k || !v) return HAGO_ERR_NULL;
  if (!hago::ptr_aligned(k, real_size(out_t)) || !hago::ptr_aligned(v, real_size(out_t))) return HAGO_ERR_PARAM;
  return from_hip(hago::launch_mx_cache_read(c, real_type(out_t), T, k, v, static_cast<hipStream_t>(stream)));
}

int64_t hago_mx_attention_workspace_bytes(int64_t T, int64_t seqs, int64_t heads, int64_t kv_heads, int64_t dim) {
  if (T < 0 || seqs < 0 || heads < 0 || kv_heads < 0 || kv_heads > kMostHeads || dim < 0 || dim > hago::kCacheMostDim || !product_fits(T, heads, hago::kMostRows) || !product_fits(seqs, kv_heads, hago::kMostUnits) ||
      seqs > kI32Max - 1 ||
      (kv_heads ? heads % kv_heads : heads) != 0)
    return -1;
  return T && heads && dim ? hago::mx_attention_workspace_bytes(T, seqs, heads, kv_heads, dim) : 0;
}

hago_status hago_mx_attention(const hago_mx_cache* cache, const hago_mx_sequences* sequences, const void* q, hago_dtype q_t, int64_t T, int64_t heads,
                              int64_t q_row_stride, int64_t q_head_stride, float scale, int32_t causal, int64_t window, void* out, float* lse, void* workspace,
                              int64_t workspace_bytes, void* stream) {
  hago::CacheArgs c{};
  bool empty = true;
  const hago_status s = check_cache(cache, sequences, T, q_t, empty, c);
  if (s != HAGO_OK) return s;
  const int64_t need = hago_mx_attention_workspace_bytes(T, sequences->seqs, heads, cache->kv_heads, cache->dim);
  if (need < 0 || window < 0 || !strides_fit(T, heads, q_row_stride, q_head_stride))
    return HAGO_ERR_SHAPE;
  if (!(std::fabs(scale) <= 0x1p100f)) return HAGO_ERR_PARAM;  // (NaN too)
  if (empty || heads == 0) return HAGO_OK;
  if (!q || !out || !workspace) return HAGO_ERR_NULL;
  const size_t size = real_size(q_t);
  if (!hago::ptr_aligned(q, size) || !hago::ptr_aligned(out, size) || !hago::ptr_aligned(lse, 4) || !hago::ptr_aligned(workspace, 256) || workspace_bytes < need)
    return HAGO_ERR_PARAM;
  hago::AttentionArgs a{};
  a.q = {q, q_row_stride, q_head_stride};
  a.out = out;
  a.lse = lse;
  a.scale = scale;
  a.T = (int32_t)T;
  a.heads = (int32_t)heads;
  a.causal = causal != 0;
  a.window = window > kI32Max ? 0 : (int32_t)window;  // (as far back as positions go)
  a.type = real_type(q_t);
  return from_hip(hago::launch_mx_attention(c, a, workspace, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
