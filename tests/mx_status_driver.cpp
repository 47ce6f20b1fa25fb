// The microscaled entry points against a runtime that stands in for HIP: which kernels serve a call, and that a refused launch is reported by
// the call that made it, once, and by no later one.
#include "fake_runtime.h"

#include <cstdio>
#include <functional>
#include <string>
#include <vector>

#include "hago.h"

int main() {
  void *a = fake::at(0), *s = fake::at(1), *w = fake::at(2), *ws = fake::at(3), *out = fake::at(4), *x = fake::at(5);
  auto* off = fake::at<int32_t>(6);
  auto* bias = fake::at<float>(7);
  struct Call {
    const char* name;
    std::function<hago_status()> run;
  };
  const std::vector<Call> calls = {
      {"quantize", [&] { return hago_mx_quantize(x, HAGO_BF16, 100, 300, 300, HAGO_MX_FP4, a, s, out, nullptr); }},
      {"rmsnorm", [&] { return hago_mx_rmsnorm(x, out, w, HAGO_F16, 100, 5000, 5000, 1e-5f, HAGO_MX_FP8, out, a, s, nullptr, nullptr); }},
      {"rmsnorm short", [&] { return hago_mx_rmsnorm(x, nullptr, nullptr, HAGO_F32, 100, 50, 60, 0.0f, HAGO_MX_FP8, nullptr, a, s, nullptr, nullptr); }},
      {"silu_mul", [&] { return hago_mx_silu_mul(x, HAGO_F32, 7, 64, 128, HAGO_MX_FP8, a, s, nullptr, nullptr); }},
      {"dense few", [&] { return hago_mx_dense(a, s, HAGO_MX_FP8, w, ws, bias, 1, 4096, 4096, HAGO_BF16, out, nullptr); }},
      {"dense large", [&] { return hago_mx_dense(a, s, HAGO_MX_FP4, w, ws, nullptr, 8192, 8192, 8192, HAGO_F32, out, nullptr); }},
      {"grouped", [&] { return hago_mx_dense_grouped(a, s, HAGO_MX_FP8, 4096, off, w, ws, nullptr, off, 16384, 32, 4096, 2048, HAGO_F16, out, nullptr); }},
  };
  int bad = 0;
  auto expect = [&](bool ok, const char* name, const char* what) {
    if (!ok) std::printf("%s: %s\n", name, what), ++bad;
  };
  for (const Call& c : calls) {
    fake::launched.clear();
    fake::calls = 0, fake::refused = -1;
    expect(c.run() == HAGO_OK, c.name, "refused");
    expect(!fake::launched.empty(), c.name, "nothing launched");
    std::printf("%s\t%s", c.name, fake::launched.c_str());
    const int made = fake::calls;   // (a kernel's LDS limit is raised by its first call only)
    fake::calls = 0, fake::refused = -1;
    (void)c.run();
    const int again = fake::calls;
    for (int i = 0; i < again; ++i) {
      fake::calls = 0, fake::refused = i, fake::launches_after = 0;
      expect(c.run() == HAGO_ERR_DEVICE, c.name, "a refused call of the runtime is not reported");
      expect(fake::launches_after == 0, c.name, "launches behind the refused one");
      expect(fake::pending == hipSuccess, c.name, "the error stays behind");
      fake::refused = -1;
      expect(c.run() == HAGO_OK, c.name, "reported again");
    }
    expect(made >= again && again >= 1, c.name, "calls");
  }
  if (!bad) std::printf("microscaled statuses: ok\n");
  return bad != 0;
}
