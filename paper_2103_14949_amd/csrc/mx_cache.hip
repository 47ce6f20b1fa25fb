// Keys and values of new tokens into a paged cache as microscaled codes, and back.
//
// Both move bytes.  A lane takes eight consecutive columns of a row's keys and of its values, a quad of lanes a block of 32 (as in the
// other operators by rows).  A workgroup takes consecutive tokens of one head: they are neighbours in a page, so that its codes and
// its scales, four bytes a row at 128 columns, leave as whole lines, and a row of the tensors is 256 bytes together anyway.
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

template <int TYPE, int KF, int VF>
__global__ __launch_bounds__(kThreads) void write_kernel(CacheArgs c, HeadsTensor k, HeadsTensor v, void* k_values, void* v_values, int64_t T, int64_t first_tile) {
  using E = typename MxElement<TYPE>::type;
  const int blocks = (c.dim + 31) / 32, lanes = blocks * 4, rows = kThreads / lanes;
  const int64_t tile = first_tile + blockIdx.x;
  const int head = (int)(tile % c.kv_heads), slot = threadIdx.x / lanes, col = (threadIdx.x - slot * lanes) * 8;
  const int64_t t = tile / c.kv_heads * rows + slot;
  int seq;
  int64_t position;
  const bool ours = slot < rows && t < T;
  // (all lanes of a quad are of one row, and take part in its exchange or not)
  if (!ours || !cache_row(c, t, seq, position)) return;
  float a[8], b[8];
  mx_load8<TYPE>(static_cast<const E*>(k.data) + t * k.row + head * k.head + (col < c.dim ? col : 0), c.dim - col, a);
  mx_load8<TYPE>(static_cast<const E*>(v.data) + t * v.row + head * v.head + (col < c.dim ? col : 0), c.dim - col, b);
  const int64_t place = cache_place(c, seq, position, head), row = t * c.kv_heads + head;
  if (place < 0 && !k_values && !v_values) return;
  put8<TYPE, KF>(c.k_codes, c.k_scales, k_values, place, row, blocks, c.dim, col, a);
  put8<TYPE, VF>(c.v_codes, c.v_scales, v_values, place, row, blocks, c.dim, col, b);
}

template <int TYPE, int FORMAT>
__device__ __forceinline__ void get8(const uint8_t* codes, const uint8_t* scales, void* out, int64_t place, int64_t row, int blocks, int dim, int col) {
  const uint32_t byte = scales[place * blocks + col / 32];
  const float scale = __builtin_bit_cast(float, byte == 255 ? 0x7fc00000u : byte ? byte << 23 : 0x00400000u);
  mx_f2 d[4];
  if constexpr (FORMAT == kMxFp4) {
    const uint32_t u = *reinterpret_cast<const uint32_t*>(codes + (place * blocks * 32 + col) / 2);
    d[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(u, 1.0f, 0);
    d[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(u, 1.0f, 1);
    d[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(u, 1.0f, 2);
    d[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(u, 1.0f, 3);
  } else {
    const uint2 u = *reinterpret_cast<const uint2*>(codes + place * blocks * 32 + col);
    d[0] = __builtin_amdgcn_cvt_pk_f32_fp8((int)u.x, false);
    d[1] = __builtin_amdgcn_cvt_pk_f32_fp8((int)u.x, true);
    d[2] = __builtin_amdgcn_cvt_pk_f32_fp8((int)u.y, false);
    d[3] = __builtin_amdgcn_cvt_pk_f32_fp8((int)u.y, true);
  }
  float v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = d[i / 2][i % 2] * scale;
  mx_store8<TYPE>(static_cast<typename MxElement<TYPE>::type*>(out) + row * dim + col, dim - col, v);
}

template <int TYPE, int KF, int VF>
__global__ __launch_bounds__(kThreads) void read_kernel(CacheArgs c, void* k, void* v, int64_t T, int64_t first_tile) {
  const int blocks = (c.dim + 31) / 32, lanes = (c.dim + 7) / 8, rows = kThreads / lanes;
  const int64_t tile = first_tile + blockIdx.x;
  const int head = (int)(tile % c.kv_heads), slot = threadIdx.x / lanes, col = (threadIdx.x - slot * lanes) * 8;
  const int64_t t = tile / c.kv_heads * rows + slot;
  int seq;
  int64_t position;
  if (slot >= rows || t >= T || !cache_row(c, t, seq, position)) return;
  const int64_t place = cache_place(c, seq, position, head), row = t * c.kv_heads + head;
  if (place < 0) return;
  get8<TYPE, KF>(c.k_codes, c.k_scales, k, place, row, blocks, c.dim, col);
  get8<TYPE, VF>(c.v_codes, c.v_scales, v, place, row, blocks, c.dim, col);
}

// Several launches where one would hold too many threads.
template <class Each>
hipError_t by_tiles(const CacheArgs& c, int64_t T, int lanes, Each&& each) {
  const int rows = kThreads / lanes;
  const int64_t tiles = (T + rows - 1) / rows * c.kv_heads, most = max_blocks(kThreads);
  hipError_t e = hipSuccess;
  for (int64_t first = 0; first < tiles && e == hipSuccess; first += most) e = each(dim3((uint32_t)(tiles - first < most ? tiles - first : most)), first);
  return e;
}

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
  return with_types(c, type, [&]<int TYPE, int KF, int VF>() {
    return by_tiles(c, T, (int)cache_blocks(c.dim) * 4, [&](dim3 grid, int64_t first) {
      return launch_kernel(write_kernel<TYPE, KF, VF>, grid, dim3(kThreads), 0, st, c, k, v, k_values, v_values, T, first);
    });
  });
}

hipError_t launch_mx_cache_read(const CacheArgs& c, int type, int64_t T, void* k, void* v, hipStream_t st) {
  return with_types(c, type, [&]<int TYPE, int KF, int VF>() {
    return by_tiles(c, T, (c.dim + 7) / 8, [&](dim3 grid, int64_t first) {
      return launch_kernel(read_kernel<TYPE, KF, VF>, grid, dim3(kThreads), 0, st, c, k, v, T, first);
    });
  });
}

}  // namespace hago
