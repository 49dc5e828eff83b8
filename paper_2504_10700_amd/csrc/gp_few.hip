// The rows of the products by element for batches without a grouping (GP_UNGROUPED atoms at most) whose weights are read once or a few times; with more rows or wider ones
// the call takes the tiles (gp_products.hip has the rule).  64 atoms, 89 elements, 128 x 128: 4.7 us forward, 5.3 dX, all launch and latency, where the tiles with their grouping take 14; 64 atoms,
// one element, 512 x 512: 18 and 12 us, in tiles 25 and 23; 16 atoms, 1024 x 1024: 17 and 12 of bfloat16, in tiles 40 and 33.
//
// The rows of one element are taken four at a time: a workgroup's row finds, from the indices of the whole batch (a lane an atom), its rank among the rows of
// its element; those whose rank is a multiple of four compute it and the three after it.  Forward: 32 columns a workgroup, 64 groups of eight threads along the
// reduced index, each four rows of W at a time; their sums meet in the lanes and in LDS.  dX: a row of W a wave at a time, four for each wave.
#include <algorithm>

#include "gp_internal.h"

namespace gp {
namespace {

constexpr int kFewThreads = 512, kFewWaves = kFewThreads / kLanes;
constexpr int kRows = 4;          // rows of an element at a time
constexpr int kColumns = 32;      // of a workgroup

template <typename T>
struct Vec4 {
  typedef T type __attribute__((ext_vector_type(4), aligned(sizeof(T))));   // element alignment is enough for wide accesses
};

// Four elements from p on, those from `inside` on zero.
template <typename T, typename TA>
__device__ __forceinline__ void load4(const T* p, int inside, TA (&v)[4]) {
  if (inside >= 4) {
    const typename Vec4<T>::type x = *reinterpret_cast<const typename Vec4<T>::type*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = static_cast<TA>(x[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = i < inside ? static_cast<TA>(p[i]) : TA(0);
  }
}

// The rows of a workgroup: where they begin in src and dst.
struct Group {
  int element;                    // a.elements: no product
  int count;                      // 0: another workgroup has this row
  int64_t src[kRows], dst[kRows];
};
__device__ __forceinline__ Group group_of(const Rows& a, int row) {
  const int lane = threadIdx.x & (kLanes - 1);
  const int atom = row / a.components, c = row - atom * a.components;
  const int n = static_cast<int>(a.n);
  const int z = a.z[min(lane, n - 1)];
  const int bucket = static_cast<unsigned>(z) < static_cast<unsigned>(a.elements) ? z : a.elements;
  Group g;
  g.element = __builtin_amdgcn_readlane(bucket, atom);
  unsigned long long same = __builtin_amdgcn_ballot_w64(lane < n && bucket == g.element);
  const int rank = __popcll(same & ((1ull << atom) - 1)) * a.components + c;
  const int all = __popcll(same) * a.components;
  g.count = rank % kRows == 0 ? min(kRows, all - rank) : 0;
  same &= ~((1ull << atom) - 1);
  int at = atom, component = c;
#pragma unroll
  for (int r = 0; r < kRows; ++r) {
    g.src[r] = at * a.ld_src + static_cast<int64_t>(component) * a.reduced;
    g.dst[r] = at * a.ld_dst + static_cast<int64_t>(component) * a.columns;
    if (r + 1 < g.count && ++component == a.components) {   // (beyond the last: the last one again)
      component = 0;
      same &= same - 1;
      at = __builtin_ctzll(same);
    }
  }
  return g;
}

template <typename T, typename TA>
__device__ __forceinline__ void store_row(const Rows& a, int64_t row, int column, TA v) {
  const int64_t at = row + column;
  static_cast<T*>(a.dst)[at] = static_cast<T>(a.residual ? v + static_cast<TA>(static_cast<const T*>(a.residual)[at]) : v);
}

template <typename T, typename TA>
__global__ __launch_bounds__(kFewThreads) void few_forward_kernel(const Rows a) {
  __shared__ TA shared[kFewWaves][kRows][kColumns];
  const Group g = group_of(a, blockIdx.x);
  if (g.count == 0) return;
  const int lane = threadIdx.x & (kLanes - 1), wave = threadIdx.x / kLanes;
  const int c0 = blockIdx.y * kColumns, c = c0 + lane % 8 * 4, inside = max(0, min(4, a.columns - c));
  TA acc[kRows][4] = {};
  if (g.element < a.elements) {
    const TA* const W = static_cast<const TA*>(a.W) + static_cast<int64_t>(g.element) * a.reduced * a.columns + min(c, a.columns - 1);
    const T* const x = static_cast<const T*>(a.src);
    constexpr int kUnroll = sizeof(TA) == 8 ? 1 : 4;   // (requests under way)
#pragma unroll kUnroll
    for (int k = 4 * (threadIdx.x / 8); k < a.reduced; k += 4 * (kFewThreads / 8)) {
      const int depth = min(4, a.reduced - k);
      TA w[4][4], v[kRows][4];
#pragma unroll
      for (int i = 0; i < 4; ++i) load4(W + static_cast<int64_t>(min(k + i, a.reduced - 1)) * a.columns, inside, w[i]);
#pragma unroll
      for (int r = 0; r < kRows; ++r) load4(x + g.src[r] + k, depth, v[r]);
#pragma unroll
      for (int r = 0; r < kRows; ++r)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (i < depth) acc[r][j] = fma(v[r][i], w[i][j], acc[r][j]);
    }
  }
#pragma unroll
  for (int r = 0; r < kRows; ++r)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
#pragma unroll
      for (int d = 8; d < kLanes; d *= 2) acc[r][j] += __shfl_xor(acc[r][j], d);
      if (lane < 8) shared[wave][r][lane * 4 + j] = acc[r][j];
    }
  __syncthreads();
  const int r = threadIdx.x / kColumns, column = threadIdx.x % kColumns;
  if (r >= g.count || c0 + column >= a.columns) return;
  TA sum = shared[0][r][column];
#pragma unroll
  for (int w = 1; w < kFewWaves; ++w) sum += shared[w][r][column];
  const int64_t to = r == 0 ? g.dst[0] : r == 1 ? g.dst[1] : r == 2 ? g.dst[2] : g.dst[3];
  store_row<T, TA>(a, to, c0 + column, sum);
}

template <typename T, typename TA>
__global__ __launch_bounds__(kFewThreads) void few_back_kernel(const Rows a) {
  const Group g = group_of(a, blockIdx.x);
  if (g.count == 0) return;
  const int lane = threadIdx.x & (kLanes - 1), wave = threadIdx.x / kLanes;
  const int c0 = blockIdx.y * kColumns + wave * 4;   // four rows of W, which are columns of dX
  if (c0 >= a.columns) return;
  TA acc[kRows][4] = {};
  if (g.element < a.elements) {
    const TA* const W = static_cast<const TA*>(a.W) + static_cast<int64_t>(g.element) * a.reduced * a.columns;
    const T* const x = static_cast<const T*>(a.src);
#pragma unroll 2
    for (int k = 4 * lane; k < a.reduced; k += 4 * kLanes) {
      const int depth = min(4, a.reduced - k);
      TA w[4][4], v[kRows][4];
#pragma unroll
      for (int j = 0; j < 4; ++j) load4(W + static_cast<int64_t>(min(c0 + j, a.columns - 1)) * a.reduced + k, depth, w[j]);
#pragma unroll
      for (int r = 0; r < kRows; ++r) load4(x + g.src[r] + k, depth, v[r]);
#pragma unroll
      for (int r = 0; r < kRows; ++r)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[r][j] = fma(v[r][i], w[j][i], acc[r][j]);   // (beyond the end both are zero)
    }
  }
  TA mine = 0;   // lane 4 r + j keeps the sum (r, j)
#pragma unroll
  for (int r = 0; r < kRows; ++r)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      TA v = acc[r][j];
#pragma unroll
      for (int d = 1; d < kLanes; d *= 2) v += __shfl_xor(v, d);
      if (lane == 4 * r + j) mine = v;
    }
  const int r = lane / 4, column = c0 + lane % 4;
  if (r >= g.count || column >= a.columns) return;
  const int64_t to = r == 0 ? g.dst[0] : r == 1 ? g.dst[1] : r == 2 ? g.dst[2] : g.dst[3];
  store_row<T, TA>(a, to, column, mine);
}

}  // namespace

hipError_t launch_rows_few(const gp_config* c, const Rows& a, bool back, hipStream_t stream) {
  const dim3 grid(static_cast<unsigned>(a.n * c->components), static_cast<unsigned>(ceil_div(a.columns, kColumns)));
  auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(kFewThreads), 0, stream, a);
    return hipGetLastError();
  };
  if (c->dtype == SC_F64) return back ? launch(&few_back_kernel<double, double>) : launch(&few_forward_kernel<double, double>);
  if (c->dtype == SC_F32) return back ? launch(&few_back_kernel<float, float>) : launch(&few_forward_kernel<float, float>);
  return back ? launch(&few_back_kernel<__bf16, float>) : launch(&few_forward_kernel<__bf16, float>);
}

}  // namespace gp
