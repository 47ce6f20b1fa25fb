// The rotary positions and the operators around a paged cache against a runtime that stands in for HIP: which kernels serve a call, with how many threads, and
// that a refused launch is reported by the call that made it, once, and by no later one.
#include "fake_runtime.h"

#include <cstdio>
#include <cstring>
#include <functional>
#include <string>
#include <vector>

#include "hago.h"

static std::string launches;

int main() {
  void *kc = fake::at(0), *ks = fake::at(1), *vc = fake::at(2), *vs = fake::at(3), *x = fake::at(4), *out = fake::at(5), *ws = fake::at(6);
  auto* ints = fake::at<int32_t>(7);
  auto* floats = fake::at<float>(8);
  const auto cache = [&](int64_t pages, int64_t heads, int64_t page, int64_t dim) {
    return hago_mx_cache{kc, ks, vc, vs, HAGO_MX_FP8, HAGO_MX_FP4, pages, heads, page, dim};
  };
  const auto sequences = [&](int64_t n, int64_t cols) { return hago_mx_sequences{ints, ints, ints, n, cols, cols}; };
  const auto attend = [&](hago_dtype t, int64_t T, int64_t heads, int64_t kv_heads, int64_t dim, int64_t seqs, int64_t page) {
    const hago_mx_cache c = cache(1000, kv_heads, page, dim);
    const hago_mx_sequences s = sequences(seqs, 10);
    return hago_mx_attention(&c, &s, x, t, T, heads, heads * dim, dim, 0.1f, 1, 0, out, nullptr, ws, 1ll << 40, nullptr);
  };
  const auto write = [&](int64_t T, int64_t heads, int64_t dim) {
    const hago_mx_cache c = cache(1000, heads, 16, dim);
    const hago_mx_sequences s = sequences(4, 10);
    return hago_mx_cache_write(&c, &s, x, heads * dim, dim, x, heads * dim, dim, HAGO_BF16, T, nullptr, nullptr, nullptr);
  };
  const auto read = [&](int64_t T, int64_t heads, int64_t dim) {
    const hago_mx_cache c = cache(1000, heads, 16, dim);
    const hago_mx_sequences s = sequences(4, 10);
    return hago_mx_cache_read(&c, &s, HAGO_F16, T, x, out, nullptr);
  };
  const auto rope = [&](int64_t T, int64_t heads, int64_t dim, int64_t pairs) {
    return hago_rope(x, HAGO_BF16, T, heads, dim, heads * dim, dim, ints, 1, floats, nullptr, pairs, HAGO_ROPE_HALVES, out, heads * dim, dim, nullptr);
  };
  struct Call {
    const char* name;
    std::function<hago_status()> run;
  };
  const std::vector<Call> calls = {
      {"rope", [&] { return rope(100, 4, 128, 64); }},
      {"rope most", [&] { return rope(2147483647, 65536, 4096, 2048); }},
      {"write", [&] { return write(5, 8, 128); }},
      {"write many", [&] { return write(100000, 8, 128); }},
      {"write most", [&] { return write(2147483647, 65536, 256); }},
      {"read", [&] { return read(5, 8, 128); }},
      {"read many", [&] { return read(100000, 8, 128); }},
      {"read one column", [&] { return read(100000000, 8, 1); }},
      {"read most", [&] { return read(2147483647, 1024, 256); }},
      {"token", [&] { return attend(HAGO_BF16, 1, 32, 8, 128, 1, 64); }},
      {"token odd pages", [&] { return attend(HAGO_F16, 1, 32, 8, 64, 1, 50); }},
      {"prompt", [&] { return attend(HAGO_BF16, 8192, 32, 8, 128, 1, 64); }},
      {"prompt odd pages", [&] { return attend(HAGO_BF16, 8192, 32, 8, 64, 1, 50); }},
      {"prompt wide", [&] { return attend(HAGO_F16, 512, 32, 8, 256, 1, 64); }},
      {"prompt f32", [&] { return attend(HAGO_F32, 8192, 32, 8, 128, 1, 64); }},
      {"chunks of sixteen rows", [&] { return attend(HAGO_BF16, 64, 32, 8, 128, 16, 64); }},
      {"many chunks", [&] { return attend(HAGO_BF16, 257 * 20, 32, 8, 128, 257, 64); }},
      {"most rows", [&] { return attend(HAGO_BF16, 1 << 27, 1, 1, 128, 1 << 22, 64); }},
      {"most tokens", [&] { return attend(HAGO_F32, 1 << 27, 1, 1, 128, 1 << 22, 64); }},
  };
  fake::seen = [](dim3 grid, dim3 block, void**) { launches += std::to_string(grid.x) + "|" + std::to_string(block.x) + ";"; };
  int bad = 0;
  auto expect = [&](bool ok, const char* name, const char* what) {
    if (!ok) std::printf("%s: %s\n", name, what), ++bad;
  };
  for (const Call& c : calls) {
    fake::launched.clear(), launches.clear();
    fake::calls = 0, fake::refused = -1;
    expect(c.run() == HAGO_OK, c.name, "refused");
    expect(!fake::launched.empty(), c.name, "nothing launched");
    std::string kernels = fake::launched;
    for (char& ch : kernels) ch = ch == '\n' ? ';' : ch;
    std::printf("%s\t%s\t%s\n", c.name, launches.c_str(), kernels.c_str());
    fake::calls = 0;
    (void)c.run();  // (a kernel's LDS limit is raised by its first call only)
    const int again = fake::calls < 6 ? fake::calls : 6;
    for (int i = 0; i < again; ++i) {
      fake::calls = 0, fake::refused = i, fake::launches_after = 0;
      expect(c.run() == HAGO_ERR_DEVICE, c.name, "a refused call of the runtime is not reported");
      expect(fake::launches_after == 0, c.name, "launches behind the refused one");
      expect(fake::pending == hipSuccess, c.name, "the error stays behind");
      fake::refused = -1;
      expect(c.run() == HAGO_OK, c.name, "reported again");
    }
  }
  if (!bad) std::printf("cache statuses: ok\n");
  return bad != 0;
}
