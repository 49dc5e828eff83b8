// The dense layer's kernels: bfloat16 rows, fp32 weights.
#include "dl_calls.h"

namespace dl {
Entries entries_bf16() {
  typedef EntryOf<__bf16, float> E;
  return {E::forward, E::backward, E::double_backward, E::zero};
}
}  // namespace dl
