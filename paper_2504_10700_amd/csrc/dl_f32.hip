// The dense layer's kernels: fp32 rows.
#include "dl_calls.h"

namespace dl {
Entries entries_f32() {
  typedef EntryOf<float, float> E;
  return {E::forward, E::backward, E::double_backward, E::zero};
}
}  // namespace dl
