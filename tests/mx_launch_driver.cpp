// Launches of the microscaled products against a runtime that stands in for HIP.  Calls come as lines "dense KERNEL FORMAT M N K" or
// "grouped KERNEL FORMAT T EXPERTS N K" (KERNEL -1: the library's choice); each is answered by a line of "name|workgroups|threads|argument" per
// launch, the argument being the one that tells a launch where it is among others.
#include "fake_runtime.h"

#include <cstdio>
#include <cstring>

#include "hago.h"

static std::string launches;

int main() {
  void *a = fake::at(0), *s = fake::at(1), *w = fake::at(2), *ws = fake::at(3), *out = fake::at(4);
  auto* off = fake::at<int32_t>(5);
  fake::seen = [](dim3 grid, dim3 block, void** args) {
    char text[96];
    uint32_t from;
    std::memcpy(&from, args[7], sizeof(from));   // (pointers to a, w and their scales, then T, N, K)
    std::snprintf(text, sizeof text, "%u|%u|%u\t", grid.x, block.x, from);
    launches += text;
  };
  char kind[16];
  int kernel, format;
  while (std::scanf("%15s %d %d", kind, &kernel, &format) == 3) {
    long long n[4];
    const bool grouped = !std::strcmp(kind, "grouped");
    for (int i = 0; i < (grouped ? 4 : 3); ++i)
      if (std::scanf("%lld", &n[i]) != 1) return 1;
    fake::launched.clear(), launches.clear();
    hago_set_test_hook(HAGO_HOOK_MX_KERNEL, kernel);
    const hago_status st = grouped ? hago_mx_dense_grouped(a, s, (hago_mx_format)format, n[0], nullptr, w, ws, nullptr, off, n[0], n[1], n[2], n[3], HAGO_BF16, out, nullptr)
                                   : hago_mx_dense(a, s, (hago_mx_format)format, w, ws, nullptr, n[0], n[1], n[2], HAGO_BF16, out, nullptr);
    std::printf("%d\t%s%s\n", (int)st, launches.c_str(), fake::launched.substr(0, fake::launched.find('\n')).c_str());
  }
  return 0;
}
