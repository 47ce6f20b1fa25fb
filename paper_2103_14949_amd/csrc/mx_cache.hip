// Keys and values of new tokens into a paged cache as microscaled codes, and back.
//
// Both move bytes.  A lane takes eight consecutive columns of a row's keys and of its values, a quad of lanes a block of 32 (as in the
// other operators by rows).  A workgroup takes consecutive tokens of one head: they are neighbours in a page, so that its codes and
// its scales, four bytes a row at 128 columns, leave as whole lines, and a row of the tensors is 256 bytes together anyway.  Where a row lies (its
// sequence, page, place) is found by one thread for all lanes of it, while the tensors' loads are under way.
//
// Four prompts of 8954 tokens in all, 8 heads of 128 columns, with values: 16.8 us, 5.2 TB/s; 131072 tokens read back: 145 us, 5.6 TB/s (a copy has 5.9).  One, two and four
// rows a thread: 17.9, 16.8 and 19.3 us, and 158 (191 with every lane looking for itself), 146 and 156.
#include "mx_cache_device.h"

namespace hago {

namespace {

constexpr int kThreads = 256;

template <int TYPE, int FORMAT>
__device__ __forceinline__ void put8(uint8_t* codes, uint8_t* scales, void* values, int64_t place, int64_t row, int blocks, int dim, int col, float (&v)[8]) {
  uint32_t code[2];
  const uint32_t byte = mx_encode8<FORMAT>(v, code);
  if (place >= 0) {
    if constexpr (FORMAT == kMxFp4)
      *reinterpret_cast<uint32_t*>(codes + (place * blocks * 32 + col) / 2) = code[0];
    else
      *reinterpret_cast<uint2*>(codes + place * blocks * 32 + col) = make_uint2(code[0], code[1]);
    if ((col & 31) == 0) scales[place * blocks + col / 32] = (uint8_t)byte;
  }
  if (values && col < dim) mx_store8<TYPE>(static_cast<typename MxElement<TYPE>::type*>(values) + row * dim + col, dim - col, v);
}

// Where a workgroup's rows lie, each found by a thread: places of the tokens first .. first + count - 1 for a head, -1: none, -2: the row is in no sequence.
__device__ __forceinline__ void find_places(const CacheArgs& c, int64_t first, int count, int64_t T, int head, int64_t (&places)[kThreads]) {
  if ((int)threadIdx.x < count) {
    int seq;
    int64_t position, place = -2;
    if (first + threadIdx.x < T && cache_row(c, first + threadIdx.x, seq, position)) place = cache_place(c, seq, position, head);
    places[threadIdx.x] = place;
  }
}

// EACH rows a thread: their loads are under way while the rows are found, and together.
template <int TYPE, int KF, int VF, int EACH>
__global__ __launch_bounds__(kThreads) void write_kernel(CacheArgs c, HeadsTensor k, HeadsTensor v, void* k_values, void* v_values, int64_t T, int64_t first_tile) {
  using E = typename MxElement<TYPE>::type;
  __shared__ int64_t places[kThreads];
  const int blocks = (c.dim + 31) / 32, lanes = blocks * 4, rows = kThreads / lanes;
  const int64_t tile = first_tile + blockIdx.x, unit = tile / c.kv_heads, first = unit * (rows * EACH);
  const int head = (int)(tile - unit * c.kv_heads), slot = threadIdx.x / lanes, col = (threadIdx.x - slot * lanes) * 8;
  float a[EACH][8], b[EACH][8];
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    const int64_t t = first + i * rows + slot;
    if (slot < rows && t < T) {
      mx_load8<TYPE>(static_cast<const E*>(k.data) + t * k.row + head * k.head + (col < c.dim ? col : 0), c.dim - col, a[i]);
      mx_load8<TYPE>(static_cast<const E*>(v.data) + t * v.row + head * v.head + (col < c.dim ? col : 0), c.dim - col, b[i]);
    }
  }
  find_places(c, first, rows * EACH, T, head, places);
  __syncthreads();
  if (slot >= rows) return;
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    // (all lanes of a quad are of one row, and take part in its exchange or not)
    const int64_t t = first + i * rows + slot, place = places[i * rows + slot], row = t * c.kv_heads + head;
    if (place == -2 || (place < 0 && !k_values && !v_values)) continue;
    put8<TYPE, KF>(c.k_codes, c.k_scales, k_values, place, row, blocks, c.dim, col, a[i]);
    put8<TYPE, VF>(c.v_codes, c.v_scales, v_values, place, row, blocks, c.dim, col, b[i]);
  }
}

// Eight codes of a row: the words they lie in, and their scale.
template <int FORMAT>
struct Eight {
  uint32_t w[2];
  uint32_t byte;
  __device__ __forceinline__ void load(const uint8_t* codes, const uint8_t* scales, int64_t place, int blocks, int col) {
    byte = scales[place * blocks + col / 32];
    if constexpr (FORMAT == kMxFp4) {
      w[0] = *reinterpret_cast<const uint32_t*>(codes + (place * blocks * 32 + col) / 2);
    } else {
      const uint2 u = *reinterpret_cast<const uint2*>(codes + place * blocks * 32 + col);
      w[0] = u.x, w[1] = u.y;
    }
  }
  template <int TYPE>
  __device__ __forceinline__ void put(void* out, int64_t row, int dim, int col) const {
    const float scale = __builtin_bit_cast(float, byte == 255 ? 0x7fc00000u : byte ? byte << 23 : 0x00400000u);
    mx_f2 d[4];
    if constexpr (FORMAT == kMxFp4) {
      d[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[0], 1.0f, 0);
      d[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[0], 1.0f, 1);
      d[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[0], 1.0f, 2);
      d[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[0], 1.0f, 3);
    } else {
      d[0] = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[0], false);
      d[1] = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[0], true);
      d[2] = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[1], false);
      d[3] = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[1], true);
    }
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = d[i / 2][i % 2] * scale;
    mx_store8<TYPE>(static_cast<typename MxElement<TYPE>::type*>(out) + row * dim + col, dim - col, v);
  }
};

template <int TYPE, int KF, int VF, int EACH>
__global__ __launch_bounds__(kThreads) void read_kernel(CacheArgs c, void* k, void* v, int64_t T, int64_t first_tile) {
  __shared__ int64_t places[kThreads];
  const int blocks = (c.dim + 31) / 32, lanes = (c.dim + 7) / 8, rows = kThreads / lanes;
  const int64_t tile = first_tile + blockIdx.x, unit = tile / c.kv_heads, first = unit * (rows * EACH);
  const int head = (int)(tile - unit * c.kv_heads), slot = threadIdx.x / lanes, col = (threadIdx.x - slot * lanes) * 8;
  find_places(c, first, rows * EACH, T, head, places);
  __syncthreads();
  if (slot >= rows) return;
  Eight<KF> a[EACH];
  Eight<VF> b[EACH];
  int64_t place[EACH];
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    place[i] = places[i * rows + slot];
    if (place[i] < 0) continue;
    a[i].load(c.k_codes, c.k_scales, place[i], blocks, col);
    b[i].load(c.v_codes, c.v_scales, place[i], blocks, col);
  }
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    if (place[i] < 0) continue;
    const int64_t row = (first + i * rows + slot) * c.kv_heads + head;
    a[i].template put<TYPE>(k, row, c.dim, col);
    b[i].template put<TYPE>(v, row, c.dim, col);
  }
}

// Several launches where one would hold too many threads.
template <class Each>
hipError_t by_tiles(const CacheArgs& c, int64_t T, int rows, Each&& each) {
  const int64_t tiles = (T + rows - 1) / rows * c.kv_heads, most = max_blocks(kThreads);
  hipError_t e = hipSuccess;
  for (int64_t first = 0; first < tiles && e == hipSuccess; first += most) e = each(dim3((uint32_t)(tiles - first < most ? tiles - first : most)), first);
  return e;
}
// Two rows a thread where that leaves eight workgroups a CU.
constexpr int kRowsAThread = 2, kManyTiles = 2048;
bool many_rows(const CacheArgs& c, int64_t T, int rows) { return (T + rows * kRowsAThread - 1) / (rows * kRowsAThread) * c.kv_heads >= kManyTiles; }

template <int TYPE, class Pick>
hipError_t with_formats(const CacheArgs& c, Pick&& pick) {
  if (c.k_format == kMxFp4) return c.v_format == kMxFp4 ? pick.template operator()<TYPE, kMxFp4, kMxFp4>() : pick.template operator()<TYPE, kMxFp4, kMxFp8>();
  return c.v_format == kMxFp4 ? pick.template operator()<TYPE, kMxFp8, kMxFp4>() : pick.template operator()<TYPE, kMxFp8, kMxFp8>();
}
template <class Pick>
hipError_t with_types(const CacheArgs& c, int type, Pick&& pick) {
  return type == kMxF32 ? with_formats<kMxF32>(c, pick) : type == kMxBf16 ? with_formats<kMxBf16>(c, pick) : with_formats<kMxF16>(c, pick);
}

}  // namespace

hipError_t launch_mx_cache_write(const CacheArgs& c, const HeadsTensor& k, const HeadsTensor& v, int type, int64_t T, void* k_values, void* v_values, hipStream_t st) {
  const int rows = kThreads / ((int)cache_blocks(c.dim) * 4);
  const bool many = many_rows(c, T, rows);
  return with_types(c, type, [&]<int TYPE, int KF, int VF>() {
    return by_tiles(c, T, many ? rows * kRowsAThread : rows, [&](dim3 grid, int64_t first) {
      return launch_kernel(many ? write_kernel<TYPE, KF, VF, kRowsAThread> : write_kernel<TYPE, KF, VF, 1>, grid, dim3(kThreads), 0, st, c, k, v, k_values, v_values, T, first);
    });
  });
}

hipError_t launch_mx_cache_read(const CacheArgs& c, int type, int64_t T, void* k, void* v, hipStream_t st) {
  // (of a row a thread, rows behind the first 256 would have no thread to find them)
  const int rows = kThreads / ((c.dim + 7) / 8);
  const bool many = rows * kRowsAThread <= kThreads && many_rows(c, T, rows);
  return with_types(c, type, [&]<int TYPE, int KF, int VF>() {
    return by_tiles(c, T, many ? rows * kRowsAThread : rows, [&](dim3 grid, int64_t first) {
      return launch_kernel(many ? read_kernel<TYPE, KF, VF, kRowsAThread> : read_kernel<TYPE, KF, VF, 1>, grid, dim3(kThreads), 0, st, c, k, v, T, first);
    });
  });
}

}  // namespace hago
