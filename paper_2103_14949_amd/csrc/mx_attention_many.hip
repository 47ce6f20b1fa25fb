// The attention's kernels for many rows a sequence, bfloat16 queries.
#include "mx_attention_many_kernel.h"

namespace hago {

hipError_t launch_attention_many_bf16(const CacheArgs& c, const AttentionArgs& a, const AttentionWork& work, hipStream_t st) {
  return with_formats<kMxBf16>(c, a, work, st);
}

}  // namespace hago
