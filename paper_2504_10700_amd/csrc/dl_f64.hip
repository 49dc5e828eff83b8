// The dense layer's kernels: fp64.
#include "dl_calls.h"

namespace dl {
Entries entries_f64() {
  typedef EntryOf<double, double> E;
  return {E::forward, E::backward, E::double_backward, E::zero};
}
}  // namespace dl
