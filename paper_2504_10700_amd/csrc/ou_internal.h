// What the kernels of the orthogonalised update (include/ou.h) share: the list of tensors as the device has it.
#pragma once
#include <hip/hip_runtime.h>

#include "sc_internal.h"
#include "../../include/ou.h"

namespace ou {

using sc::align_up;
using sc::kLanes;

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kLanes;

// A tensor of the list.  Work is dealt out in units (chunks of elements, tiles of a product); `unit[k]` is the number of units of kind k in the tensors
// before this one.
enum Kind { kChunks, kGram, kProduct, kKinds };

struct Item {
  const void* grad;
  void* momentum;
  void* weight;
  void* update;
  double scale;
  int64_t count;
  int64_t x, s;            // where X and S begin in their buffers, in elements
  int64_t unit[kKinds];
  int32_t rows, cols, dtype, pad;
};
constexpr int kSent = 36;  // items of one launch's kernel arguments
struct Sent {
  int32_t first, count;
  Item item[kSent];
};
static_assert(sizeof(Sent) <= 4000, "the kernel arguments hold 4 KB");

// The last of items[0..n) whose first unit of that kind is not beyond `unit` (tensors without units share it with the next one).
__device__ __forceinline__ int item_of(const Item* __restrict__ items, int n, int kind, int64_t unit) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (items[mid].unit[kind] <= unit) lo = mid; else hi = mid - 1;
  }
  return lo;
}

}  // namespace ou
