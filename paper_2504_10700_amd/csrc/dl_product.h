// Products of the dense layer that go from memory through registers into the matrix instruction.
//
// The 16x16x4 instruction takes from lane l one value of each operand, non-reduced index j = l % 16, reduced index q = l / 16, and leaves in the
// lane four results: rows row(r), r = 0..3, of column j.  Which column of a tensor stands behind an index is free, so a lane reads four
// consecutive elements with one 16-byte access and uses them for four instructions:
//   - elements along the non-reduced index (W in the forward, both operands of dW) belong to four tiles u, tile u holding column 4 j + u; the 16
//     lanes of a q read 256 contiguous bytes, and the four results of a row are neighbours again where they are stored;
//   - elements along the reduced index k (the rows X, G) belong to four steps s, k = 4 q + s.  Read in that place, neighbouring lanes would
//     touch different rows, and the cache serves 64 bytes of neighbouring lanes at a time (measured: 53 accesses per instruction instead of 16,
//     62% of what the L1 cache can do, the matrix cores waiting half of the time).  So four neighbouring lanes read the 64 bytes of a row, and
//     the wave turns the 16 x 16 elements in its own corner of LDS.
// An fp32 instruction of this shape occupies the matrix core for 32 cycles and an fp64 one for 64, so a wave that holds 64 x 32 or more results
// needs less than 32 bytes a cycle and CU from the L1 cache: sharing the operands of several waves through LDS would save nothing.
#pragma once
#include <type_traits>

#include "dl_gate.h"
#include "el_tile.h"

namespace dl {

using el::Mma;
using sc::kLanes;

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kLanes;
constexpr int kCols = 64;      // columns of a wave's results: four tiles
constexpr int kDepth = 16;     // reduced index per round: four instructions deep

template <typename T>
struct Vec4 {
  typedef T type __attribute__((ext_vector_type(4), aligned(sizeof(T))));   // wide accesses need element alignment only
};

// One row-major tensor: element (r, c) at p[r * ld + c].
template <typename T>
struct Matrix {
  const T* p;
  int64_t ld;
};

// Where a lane's elements lie: `base` elements from the start, the same for the whole wave, and `lane` further on.  Kept apart, the first is scalar
// arithmetic and the second one register that does not change (the strides are limited so that it fits: DL_MAX_STRIDE).
struct Spot {
  int64_t base;
  unsigned lane;
};
template <typename T>
__device__ __forceinline__ T* at(T* p, const Spot& s) {
  typedef std::conditional_t<std::is_const<T>::value, const char, char> Byte;
  return reinterpret_cast<T*>(reinterpret_cast<Byte*>(p + s.base) + static_cast<size_t>(s.lane * static_cast<unsigned>(sizeof(T))));
}

// Four elements of a row from column c on.  kFours: the row's length is a multiple of four, so four elements are all inside or all
// beyond the end; then the address is clamped and zeros are put in when the values are used, without a branch (requests behind branches
// wait for each other).  Otherwise every element is tested.
template <bool kFours, typename T, typename TA>
__device__ __forceinline__ void load4(const T* __restrict__ p, int c, int cols, TA (&v)[4]) {
  if (kFours || c + 4 <= cols) {
    const typename Vec4<T>::type x = *reinterpret_cast<const typename Vec4<T>::type*>(p + (kFours ? min(c, cols - 4) : c));
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = static_cast<TA>(x[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = c + i < cols ? static_cast<TA>(p[c + i]) : TA(0);
  }
}

template <typename TA>
__device__ __forceinline__ void zero_unless(bool inside, TA (&v)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = inside ? v[i] : TA(0);
}

// p: where the first of them goes, column c of a row of `cols`.
template <bool kFours, typename T, typename TA>
__device__ __forceinline__ void store4(T* __restrict__ p, int c, int cols, const TA (&v)[4]) {
  if (kFours || c + 4 <= cols) {
    typename Vec4<T>::type x;
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = static_cast<T>(v[i]);
    *reinterpret_cast<typename Vec4<T>::type*>(p) = x;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (c + i < cols) p[i] = static_cast<T>(v[i]);
  }
}

// Rows as an operand.  kPlain: a tensor of the caller (X, HX, dY).  kMade: G or S as a tensor of its own.  kGated: dY act'(Z), z beside x.
enum Source { kPlain, kMade, kGated };

template <typename TA, typename T, Source kSource>
struct Operand {
  static constexpr Source source = kSource;
  Matrix<T> x, z;
  Gate<TA> gate;   // kGated
  // raw elements first (so that many requests can be under way), arithmetic later
  struct Raw {
    TA v[4], z[kSource == kGated ? 4 : 1];
  };
  template <bool kFours>
  __device__ __forceinline__ void request(int64_t row, int c, int cols, Raw& raw) const {
    load4<kFours>(x.p + row * x.ld, c, cols, raw.v);
    if constexpr (kSource == kGated) load4<kFours>(z.p + row * z.ld, c, cols, raw.z);
  }
  template <bool kFours>
  __device__ __forceinline__ void finish(const Raw& raw, int c, int cols, TA (&v)[4]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[i] = raw.v[i];
      if constexpr (kSource == kGated) v[i] *= gate.first(raw.z[i]);
    }
    if constexpr (kFours) zero_unless(c < cols, v);
  }
};

// A matrix [k_end][n_end] as the operand of a product over its first index (W in the forward, W transposed in dX): tile u holds columns n0 + 4 j + u.
template <typename TA>
struct AlongRows {
  const TA* W;
  int k_end, n_end;
  template <bool kFours>
  __device__ __forceinline__ void request(int n0, int k0, TA (&w)[4][4]) const {   // [s][u]
    const int lane = threadIdx.x & (kLanes - 1);
#pragma unroll
    for (int s = 0; s < 4; ++s)
      load4<kFours>(W + static_cast<int64_t>(min(k0 + 4 * (lane / 16) + s, k_end - 1)) * n_end, n0 + 4 * (lane & 15), n_end, w[s]);
  }
  // the operand of step s and tile u; indices beyond k_end give zero (columns beyond n_end are computed and not stored)
  static __device__ __forceinline__ void operands(const TA (&w)[4][4], int k0, int k_end, TA (&c)[4][4]) {
    const int k = k0 + 4 * ((threadIdx.x & (kLanes - 1)) / 16);
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
      for (int u = 0; u < 4; ++u) c[s][u] = k + s < k_end ? w[s][u] : TA(0);
  }
};

// A matrix [n_end][k_end] as the operand of a product over its second index (W as it is in dX): the same tiles, from accesses that are not
// contiguous between lanes.
template <typename TA>
struct AlongColumns {
  const TA* W;
  int k_end, n_end;
  template <bool kFours>
  __device__ __forceinline__ void request(int n0, int k0, TA (&w)[4][4]) const {   // [u][s]
    const int lane = threadIdx.x & (kLanes - 1);
#pragma unroll
    for (int u = 0; u < 4; ++u)
      load4<kFours>(W + static_cast<int64_t>(min(n0 + 4 * (lane & 15) + u, n_end - 1)) * k_end, k0 + 4 * (lane / 16), k_end, w[u]);
  }
  static __device__ __forceinline__ void operands(const TA (&w)[4][4], int k0, int k_end, TA (&c)[4][4]) {
    const int k = k0 + 4 * ((threadIdx.x & (kLanes - 1)) / 16);
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
      for (int u = 0; u < 4; ++u) c[s][u] = k + s < k_end ? w[u][s] : TA(0);
  }
};

// The wave's corner of LDS: kRT blocks of 16 rows x 16 elements, the four pieces of row j at places that the 16 rows of a piece find in different
// banks.
template <typename TA>
struct Corner {
  typedef TA Piece __attribute__((ext_vector_type(4)));
  static constexpr int kBlock = 256;   // elements of a block
  static __device__ __forceinline__ int at(int row, int piece) { return 16 * row + 4 * (piece ^ (row / 4)); }
  // LDS serves a wave's requests in their order: between put and get the compiler alone has to keep it
  static __device__ __forceinline__ void sync() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
  static __device__ __forceinline__ void put(TA* block, const TA (&v)[4]) {   // lane 4 row + piece
    const int lane = threadIdx.x & (kLanes - 1);
    *reinterpret_cast<Piece*>(block + at(lane / 4, lane % 4)) = Piece{v[0], v[1], v[2], v[3]};
  }
  static __device__ __forceinline__ void get(const TA* block, TA (&v)[4]) {   // lane 16 q + j: row j, piece q
    const int lane = threadIdx.x & (kLanes - 1);
    const Piece p = *reinterpret_cast<const Piece*>(block + at(lane & 15, lane / 16));
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = p[i];
  }
};

// Results of 16 kRT rows from row0 and 64 columns from n0: acc[rt][u], over the reduced indices [k_from, k_to), not empty.  Rows beyond the
// last are computed from the last one and not stored.  corner: kRT blocks of this wave.
template <typename TA, int kRT, bool kFours, typename Rows, typename Weights>
__device__ __forceinline__ void rows_product(const Rows& a, const Weights& w, int64_t row0, int64_t rows, int n0, int k_from, int k_to,
                                             TA* corner, typename Mma<TA>::acc_t (&acc)[kRT][4]) {
  typedef Corner<TA> C;
  const int lane = threadIdx.x & (kLanes - 1), kp = 4 * (lane % 4);
  int64_t at[kRT];
#pragma unroll
  for (int i = 0; i < kRT; ++i) at[i] = min(row0 + 16 * i + lane / 4, rows - 1);
#pragma unroll
  for (int i = 0; i < kRT; ++i)
#pragma unroll
    for (int t = 0; t < 4; ++t) acc[i][t] = typename Mma<TA>::acc_t{0, 0, 0, 0};
  typename Rows::Raw raw[kRT];
  TA next[4][4];
  auto request = [&](int k) {
#pragma unroll
    for (int i = 0; i < kRT; ++i) a.template request<kFours>(at[i], k + kp, w.k_end, raw[i]);
    w.template request<kFours>(n0, k, next);
  };
  request(k_from);
  for (int k = k_from; k < k_to; k += kDepth) {
    TA x[kRT][4], c[4][4];
#pragma unroll
    for (int i = 0; i < kRT; ++i) {
      TA v[4];
      a.template finish<kFours>(raw[i], k + kp, w.k_end, v);
      C::put(corner + i * C::kBlock, v);
    }
    Weights::operands(next, k, w.k_end, c);
    if (k + kDepth < k_to) request(k + kDepth);
    C::sync();
#pragma unroll
    for (int i = 0; i < kRT; ++i) C::get(corner + i * C::kBlock, x[i]);
    C::sync();
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = 0; i < kRT; ++i) acc[i][t] = Mma<TA>::mma(x[i][s], c[s][t], acc[i][t]);
  }
}

// Tensors with a row per result row that the epilogue reads (residual; Z and dY): requested a row tile ahead.
template <typename T, int N>
struct Beside {
  Matrix<T> m[N > 0 ? N : 1];
};

// Rows row0 + base + lane of a tile's results r: fp32 lane 4 q, base r; fp64 lane q, base 4 r.
template <typename TA>
__device__ __forceinline__ int lane_row() {
  const int q = (threadIdx.x & (kLanes - 1)) / 16;
  return sizeof(TA) == 8 ? q : 4 * q;
}
template <typename TA>
__device__ __forceinline__ constexpr int base_row(int r) { return sizeof(TA) == 8 ? 4 * r : r; }

// f(base row, lane row, column, values of four neighbouring columns plus their bias, the same elements of the tensors beside) for a wave's
// results.
template <typename TA, int kRT, bool kFours, typename T, int N, typename F>
__device__ __forceinline__ void each_four(int64_t row0, int64_t rows, int n0, int n_end, const typename Mma<TA>::acc_t (&acc)[kRT][4],
                                          const TA* __restrict__ bias, const Beside<T, N>& beside, F&& f) {
  const int lane = threadIdx.x & (kLanes - 1), c = n0 + 4 * (lane & 15), lr = lane_row<TA>();
  constexpr int M = N > 0 ? N : 1;
  TA next[4][M][4];
  auto request = [&](int i) {
#pragma unroll
    for (int e = 0; e < N; ++e)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        load4<kFours>(beside.m[e].p + min(row0 + 16 * i + base_row<TA>(r) + lr, rows - 1) * beside.m[e].ld, c, n_end, next[r][e]);
  };
  request(0);
  TA b[4] = {0, 0, 0, 0};
  if (bias) load4<kFours>(bias, c, n_end, b);
#pragma unroll
  for (int i = 0; i < kRT; ++i) {
    TA x[4][M][4];
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int e = 0; e < N; ++e)
#pragma unroll
        for (int k = 0; k < 4; ++k) x[r][e][k] = next[r][e][k];
    if (i + 1 < kRT) request(i + 1);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int64_t row = row0 + 16 * i + base_row<TA>(r);
      TA v[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) v[u] = acc[i][u][r] + b[u];
      if (row + lr < rows && c < n_end) f(row, lr, c, v, x[r]);
    }
  }
}

// dW of 64 x 64 (k_in from m0, k_out from n0) over the rows [from, to): acc[t][u], the lane's result r of tile (t, u) is row m0 + 4 row(r) + t,
// column n0 + 4 j + u.  sum[u]: the lane's share of the column sums of B.  Rounds of 16 rows, four at a time (one per q).
template <typename TA, bool kFours, typename A, typename B>
__device__ __forceinline__ void outer_product(const A& a, const B& b, int m0, int m_end, int n0, int n_end, int64_t from, int64_t to,
                                              typename Mma<TA>::acc_t (&acc)[4][4], TA (&sum)[4]) {
  const int lane = threadIdx.x & (kLanes - 1), q = lane / 16, j = lane & 15;
  typename A::Raw ra[4];
  typename B::Raw rb[4];
  auto request = [&](int64_t row) {
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const int64_t r = min(row + 4 * s + q, to - 1);
      a.template request<kFours>(r, m0 + 4 * j, m_end, ra[s]);
      b.template request<kFours>(r, n0 + 4 * j, n_end, rb[s]);
    }
  };
  if (from < to) request(from);
  for (int64_t row = from; row < to; row += 16) {
    TA x[4][4], g[4][4];
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      a.template finish<kFours>(ra[s], m0 + 4 * j, m_end, x[s]);
      b.template finish<kFours>(rb[s], n0 + 4 * j, n_end, g[s]);
    }
    if (row + 16 > to) {   // rows beyond the range have no part
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        zero_unless(row + 4 * s + q < to, x[s]);
        zero_unless(row + 4 * s + q < to, g[s]);
      }
    }
    if (row + 16 < to) request(row + 16);
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
      for (int i = 0; i < 4; ++i) sum[i] += g[s][i];
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int u = 0; u < 4; ++u) acc[t][u] = Mma<TA>::mma(x[s][t], g[s][u], acc[t][u]);
  }
}

}  // namespace dl
