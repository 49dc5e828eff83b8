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
constexpr int64_t kMaxGrid = int64_t(1) << 23;   // workgroups of a launch; they go on to the units beyond

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

// Which unit a workgroup takes: consecutive ones go to the same XCD (workgroups are dealt out to the XCDs in turn), whose L2 then holds the weights that they share.
constexpr int kXcds = 8;
__device__ __forceinline__ int64_t unit_of(int64_t block, int64_t total) {
  const int64_t per = (total + kXcds - 1) / kXcds, u = block % kXcds * per + block / kXcds;
  return block / kXcds < per ? u : total;
}

// units(atoms): of a bucket.  A bucket of several units has a slot for each of them, one of a single unit none.  `each`: workgroups of a unit; `block` is the
// workgroup, *which its number among the unit's.  The whole wave calls it; every lane sums the buckets of its stretch.
template <typename U>
__device__ __forceinline__ Place place_of(const int32_t* __restrict__ offsets, int buckets, int64_t n, int64_t block, int each, U&& units, int* which) {
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
  const int total = __builtin_amdgcn_readlane(u_end, kLanes - 1);
  const int64_t mine = unit_of(block, static_cast<int64_t>(total) * each);
  const int unit = static_cast<int>(mine / each);
  *which = static_cast<int>(mine - static_cast<int64_t>(unit) * each);
  const unsigned long long beyond = __builtin_amdgcn_ballot_w64(unit < u_end);
  if (beyond == 0) return {-1, 0, 0, 0, 0, 0};
  const int owner = __builtin_ctzll(beyond);
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

// ---- the products' arguments

struct Rows {
  int64_t n;            // atoms
  int64_t ld_src, ld_dst;
  const int32_t* z;
  Grouping group;       // offsets NULL: none
  int elements, components;
  int reduced, columns;
  const void* src;
  const void* W;        // [elements][k_in][k_out]
  const void* residual;
  void* dst;
};

struct Outer {
  int64_t n;
  int64_t ld_in, ld_out;
  const int32_t* z;
  Grouping group;
  int elements, components;
  int k_in, k_out;
  int per;              // rows of a chunk
  int slots;            // partial matrices that the workspace holds
  const void* X;
  const void* dY;
  void* dW;
  void* partial;        // [slots][k_in][k_out]
};

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Where row r of a bucket begins: component r % components of atom r / components.
__device__ __forceinline__ int64_t row_offset(const int32_t* order, int64_t n, int begin, int r, int components, int64_t ld, int width) {
  const int a = components == 1 ? r : static_cast<int>(static_cast<unsigned>(r) / static_cast<unsigned>(components));
  const int64_t atom = min(static_cast<unsigned>(order[begin + a]), static_cast<unsigned>(n - 1));
  return atom * ld + static_cast<int64_t>(r - a * components) * width;
}
template <typename T>
__device__ __forceinline__ T* row_at(T* p, const int32_t* order, int64_t n, int begin, int r, int components, int64_t ld, int width) {
  return p + row_offset(order, n, begin, r, components, ld, width);
}

// An element without rows has a chunk too, which zeroes its matrix.
__device__ __forceinline__ int chunks_of(int rows, int per) { return max(1, static_cast<int>((static_cast<unsigned>(rows) + per - 1) / static_cast<unsigned>(per))); }

// Rows of fp32 and bfloat16, widths from 2 on, on bfloat16 parts (gp_parts.hip).
bool parts_serve(const gp_config* c);
hipError_t launch_rows_parts(const gp_config* c, const Rows& a, bool back, hipStream_t stream);
hipError_t launch_outer_parts(const gp_config* c, const Outer& a, hipStream_t stream);
// Batches without a grouping: rows (gp_few.hip).
hipError_t launch_rows_few(const gp_config* c, const Rows& a, bool back, hipStream_t stream);

}  // namespace gp
