// What the kernels of the products by element (include/gp.h) share: the grouping and how work is found in it.
//
// A grouping is int32 data: offsets[Z + 2] (bucket Z: the atoms outside 0..Z-1), order[n] (atoms by bucket, in the order of the batch within each)
// and the counts of the sort.  The rows of a bucket are those of its atoms one after the other: row r is component r % components of
// atom r / components.  Work is dealt out in units of rows of one bucket; how many units each has is known on the device alone, so
// launches have room for the most there can be and every workgroup finds its own.
#pragma once
#include <hip/hip_runtime.h>

#include "sc_internal.h"
#include "../../include/gp.h"

namespace gp {

using sc::align_up;
using sc::kLanes;

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kLanes;
constexpr int kSortThreads = 1024;
constexpr int kSortWaves = kSortThreads / kLanes;
constexpr int kSortGroups = 128;   // workgroups of the sort of a large batch
constexpr int kSortAtoms = 2048;   // atoms that one workgroup sorts alone

struct Grouping {
  const int32_t* offsets;
  const int32_t* order;
};

inline size_t offsets_bytes(int elements) { return align_up((static_cast<size_t>(elements) + 2) * 4, 256); }
inline size_t order_bytes(int64_t n) { return align_up(static_cast<size_t>(n) * 4, 256); }
inline size_t grouping_bytes(int elements, int64_t n) {
  return n <= GP_UNGROUPED ? 0 : offsets_bytes(elements) + order_bytes(n) + align_up(static_cast<size_t>(kSortGroups) * (elements + 1) * 4, 256);
}
inline Grouping grouping_of(const void* base, int elements) {
  const char* p = static_cast<const char*>(base);
  return {reinterpret_cast<const int32_t*>(p), reinterpret_cast<const int32_t*>(p + offsets_bytes(elements))};
}

hipError_t launch_group(const gp_config* cfg, int64_t n, const int32_t* z, void* grouping, hipStream_t stream);

// A unit's bucket, the unit's number among the bucket's units, and the slots of the buckets before it.
struct Place {
  int bucket;   // -1: beyond the last unit
  int local, units, slots;
  int begin, atoms;   // positions of the bucket in the order
};

// units(atoms): of a bucket.  A bucket of several units has a slot for each of them, one of a single unit none.  The whole wave calls it; every lane sums
// the buckets of its stretch.
template <typename U>
__device__ __forceinline__ Place place_of(const int32_t* __restrict__ offsets, int buckets, int64_t n, int unit, U&& units) {
  const int lane = threadIdx.x & (kLanes - 1);
  const int per = (buckets + kLanes - 1) / kLanes, first = lane * per;
  const int most = static_cast<int>(n);
  auto at = [&](int b) { return min(max(offsets[min(b, buckets)], 0), most); };   // (whatever stands there: inside the order)
  int u = 0, s = 0;
  int from = at(first);
  for (int i = 0; i < per; ++i) {
    const int to = at(first + i + 1);
    if (first + i < buckets) {
      const int k = units(max(to - from, 0));
      u += k;
      s += k > 1 ? k : 0;
    }
    from = to;
  }
  int u_end = u, s_end = s;
#pragma unroll
  for (int d = 1; d < kLanes; d *= 2) {
    const int a = __shfl_up(u_end, d), b = __shfl_up(s_end, d);
    if (lane >= d) {
      u_end += a;
      s_end += b;
    }
  }
  const unsigned long long mine = __builtin_amdgcn_ballot_w64(unit < u_end);
  if (mine == 0) return {-1, 0, 0, 0, 0, 0};
  const int owner = __builtin_ctzll(mine);
  int local = unit - __builtin_amdgcn_readlane(u_end - u, owner);
  int slot = __builtin_amdgcn_readlane(s_end - s, owner);
  int bucket = owner * per;
  from = at(bucket);
  int atoms = 0, k = 0;
  for (; bucket < buckets; ++bucket) {
    const int to = at(bucket + 1);
    atoms = max(to - from, 0);
    k = units(atoms);
    if (local < k) break;
    local -= k;
    slot += k > 1 ? k : 0;
    from = to;
  }
  return {__builtin_amdgcn_readfirstlane(bucket), __builtin_amdgcn_readfirstlane(local), __builtin_amdgcn_readfirstlane(k),
          __builtin_amdgcn_readfirstlane(slot), __builtin_amdgcn_readfirstlane(from), __builtin_amdgcn_readfirstlane(atoms)};
}

}  // namespace gp
