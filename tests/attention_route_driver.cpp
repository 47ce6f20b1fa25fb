// Which kernels serve a call of the attention, against a runtime that stands in for HIP: a call a line of standard input, as
// "type T heads kv_heads dim seqs page" with type 0 binary32, 1 bfloat16, 2 float16; its kernels and the bytes of its workspace a line of standard output.
#include "fake_runtime.h"

#include <cstdio>
#include <string>

#include "hago.h"

int main() {
  void *kc = fake::at(0), *ks = fake::at(1), *vc = fake::at(2), *vs = fake::at(3), *x = fake::at(4), *out = fake::at(5), *ws = fake::at(6);
  auto* ints = fake::at<int32_t>(7);
  long long type, T, heads, kv_heads, dim, seqs, page;
  while (std::scanf("%lld %lld %lld %lld %lld %lld %lld", &type, &T, &heads, &kv_heads, &dim, &seqs, &page) == 7) {
    const hago_mx_cache c{kc, ks, vc, vs, HAGO_MX_FP8, HAGO_MX_FP4, 1000, kv_heads, page, dim};
    const hago_mx_sequences s{ints, ints, ints, seqs, 10, 10};
    const hago_dtype t = type == 0 ? HAGO_F32 : type == 1 ? HAGO_BF16 : HAGO_F16;
    const long long bytes = hago_mx_attention_workspace_bytes(T, seqs, heads, kv_heads, dim);
    fake::launched.clear(), fake::calls = 0, fake::refused = -1;
    if (hago_mx_attention(&c, &s, x, t, T, heads, heads * dim, dim, 0.1f, 1, 0, out, nullptr, ws, bytes, nullptr) != HAGO_OK) return 1;
    std::string kernels = fake::launched;
    for (char& ch : kernels) ch = ch == '\n' ? ';' : ch;
    std::printf("%s\t%lld\n", kernels.c_str(), bytes);
  }
  return 0;
}
