// What the kernels of the orthogonalised update (include/ou.h) share: the list of tensors as the device has it, the operations on elements.
#pragma once
#include <hip/hip_runtime.h>

#include <vector>

#include "sc_internal.h"
#include "../../include/ou.h"

namespace ou {

using sc::align_up;
using sc::kLanes;

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kLanes;
constexpr int kChunk = 4096;   // elements of a chunk of the first pass

// A matrix as the iteration sees it is m x l, m <= l: the tensor's matrix, or its transpose where rows > cols.  Work is dealt out in units; `unit[k]` is
// the number of units of kind k in the tensors before this one.
enum Kind { kChunks, kBlocks, kGram, kProduct, kGramSmall, kProductSmall, kKinds };   // (products: in tiles of 128, in tiles of 64)

struct Item {
  const void* grad;
  void* momentum;
  void* weight;
  void* update;
  double scale;
  int64_t unit[kKinds];
  int64_t x, s;            // where the tensor's X and (fp64) S begin in their buffers, in elements
  int64_t px, pt, ps;      // and the parts of X, of X transposed, of S and P
  int32_t rows, cols, dtype;
  int32_t width;           // of a slice (ou_small.hip)
};
constexpr int kSent = 27;  // items of one launch's kernel arguments
struct Sent {
  int32_t first, count;
  Item item[kSent];
};
static_assert(sizeof(Sent) <= 4000, "the kernel arguments hold 4 KB");

struct Step {
  double a, b, c, mu, rate, keep, eps;   // keep: 1 - rate * decay
  int nesterov;
};

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Tensors of one way through the kernels.
struct Part {
  std::vector<Item> items;
  int64_t units[kKinds] = {};
  int64_t x = 0, s = 0, px = 0, pt = 0, ps = 0;
  size_t at_items = 0, at_partial = 0, at_x = 0;
  size_t at[5] = {};   // the way's other buffers
};

// What workspace there is: room(bytes) is the offset of the next piece.
struct Room {
  size_t bytes = 0;
  size_t operator()(size_t n) {
    const size_t from = bytes;
    bytes += align_up(n, 256);
    return from;
  }
};

// The last of items[0..n) whose first unit of that kind is not beyond `unit` (tensors without units share it with the next one).
__device__ __forceinline__ int item_of(const Item* __restrict__ items, int n, int kind, int64_t unit) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (items[mid].unit[kind] <= unit) lo = mid; else hi = mid - 1;
  }
  return lo;
}

__device__ __forceinline__ int64_t chunks_of(int64_t elements) { return (elements + kChunk - 1) / kChunk; }

// Two fp32 values as two fp16 parts each, v = h + l, a 16-bit half each.
typedef _Float16 H2 __attribute__((ext_vector_type(2)));
typedef float F2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ void split2(float v, float w, unsigned& h, unsigned& l) {
  const F2 x{v, w};
  const H2 y = __builtin_convertvector(x, H2);
  h = __builtin_bit_cast(unsigned, y);
  l = __builtin_bit_cast(unsigned, __builtin_convertvector(x - __builtin_convertvector(y, F2), H2));
}

// U of an element from its gradient and the momentum that the step leaves.
template <typename TA>
__device__ __forceinline__ TA direction(TA g, TA m, TA mu, bool nesterov) { return nesterov ? g + mu * m : m; }

// G of an element in the arithmetic type.
template <typename TA>
__device__ __forceinline__ TA gradient(const Item& it, int64_t at) {
  if constexpr (sizeof(TA) == 8) return static_cast<const double*>(it.grad)[at];
  else return it.dtype == SC_BF16 ? static_cast<float>(static_cast<const __bf16*>(it.grad)[at]) : static_cast<const float*>(it.grad)[at];
}

// A finished element of X: into the update and the weight.
template <typename TA>
__device__ __forceinline__ void put_update(const Item& it, int64_t at, TA x) {
  if (sizeof(TA) == 4 && it.dtype == SC_BF16) static_cast<__bf16*>(it.update)[at] = static_cast<__bf16>(static_cast<float>(x));
  else static_cast<TA*>(it.update)[at] = x;
}
template <typename TA>
__device__ __forceinline__ TA new_weight(const Item& it, const Step& st, TA w, TA x) { return static_cast<TA>(st.keep) * w - static_cast<TA>(st.rate * it.scale) * x; }
template <typename TA>
__device__ __forceinline__ void finish(const Item& it, const Step& st, int64_t at, TA x) {
  if (it.update) put_update(it, at, x);
  if (it.weight) {
    TA* const w = static_cast<TA*>(it.weight) + at;
    *w = new_weight(it, st, *w, x);
  }
}

__device__ __forceinline__ double workgroup_sum(double v, double* slots) {
#pragma unroll
  for (int d = 32; d > 0; d /= 2) v += __shfl_xor(v, d);
  if ((threadIdx.x & 63) == 0) slots[threadIdx.x / 64] = v;
  __syncthreads();
  double s = slots[0];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) s += slots[w];
  __syncthreads();
  return s;
}

// 1 / (|U| + eps) of a matrix with that sum of squares.  A matrix of zeros stays zero for every eps (below 2^-1024 the quotient is beyond the largest number).
__device__ __forceinline__ double down_from(double sum, double eps) { return sum == 0 ? 0 : 1.0 / (sqrt(sum) + eps); }

// The same of a matrix whose chunks left their sums of squares in partial[0..n).
__device__ __forceinline__ double down_of(const double* __restrict__ partial, int64_t n, double eps, double* slots) {
  double sum = 0;
  for (int64_t i = threadIdx.x; i < n; i += kThreads) sum += partial[i];
  return down_from(workgroup_sum(sum, slots), eps);
}

// fp64: squares of elements beyond 2^480 or below 2^-480 can leave the range of the numbers (or add up to more), so these have sums of their own, of the elements times 2^-600
// and 2^600.
struct Squares {
  double small, middle, large;
};
__device__ __forceinline__ void add_square(Squares& s, double u) {
  const double v = fabs(u);
  if (v >= 0x1p480) s.large = fma(u * 0x1p-600, u * 0x1p-600, s.large);
  else if (v < 0x1p-480) s.small = fma(u * 0x1p600, u * 0x1p600, s.small);
  else s.middle = fma(u, u, s.middle);   // (NaN too)
}
// What an element is multiplied with, one factor after the other: together 1 / (|U| + eps).
struct Down {
  double first, second;
};
__device__ __forceinline__ Down down_of(const Squares* __restrict__ partial, int64_t n, double eps, double* slots) {
  Squares s{0, 0, 0};
  for (int64_t i = threadIdx.x; i < n; i += kThreads) {
    s.small += partial[i].small;
    s.middle += partial[i].middle;
    s.large += partial[i].large;
  }
  s.small = workgroup_sum(s.small, slots);
  s.middle = workgroup_sum(s.middle, slots);
  s.large = workgroup_sum(s.large, slots);
  if (s.large != 0) return {down_from(s.large + s.middle * 0x1p-600 * 0x1p-600, eps * 0x1p-600), 0x1p-600};
  if (s.middle != 0) return {down_from(s.middle + s.small * 0x1p-600 * 0x1p-600, eps), 1.0};
  return {0x1p600, down_from(s.small, eps * 0x1p600)};
}

// The largest |a x + b x^3 + c x^5| of 0 <= x <= top: what the largest singular value can be after a step that began with top.
double growth(const ou_config* c, double top);

// fp32 matrices of any size, on parts (ou_parts.hip).  place: the units and places of a tensor's matrices; layout: the buffers; run: from the sums of squares on.
void parts_place(Part& p, Item& it, int64_t count);
void parts_layout(Part& p, Room& room, int steps);
hipError_t parts_run(const Part& p, const ou_config* cfg, const Step& st, char* base, hipStream_t stream);

// fp32 matrices whose shorter side is at most 64 (large: 128): those whose longer side is too, from the gradient to the weight; and wider ones, from the sums of squares
// on (ou_small.hip).
hipError_t whole_run(const Part& p64, const Part& p128, const ou_config* cfg, const Step& st, char* base, hipStream_t stream);
void slice_place(Part& p, Item& it, int64_t count, int64_t matrices, bool large);   // (matrices: of this way in the list)
void slice_layout(Part& p, Room& room, int steps, bool large);
hipError_t slice_run(const Part& p, const ou_config* cfg, const Step& st, bool large, char* base, hipStream_t stream);

// The power of two that brings `top` to at most 2^14 (fp16 parts); a bound below kLeastBound counts as that.
constexpr double kLeastBound = 1e-3;
int exponent_of(double top);

}  // namespace ou
