// The attention's kernels for many rows a sequence, float16 queries: two bfloat16 numbers each, and two for a probability.
#include "mx_attention_many_kernel.h"

namespace hago {

hipError_t launch_attention_many_f16(const CacheArgs& c, const AttentionArgs& a, const AttentionWork& work, hipStream_t st) {
  return with_formats<kMxF16>(c, a, work, st);
}

}  // namespace hago
