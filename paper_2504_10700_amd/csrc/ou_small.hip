// The orthogonalised update of matrices whose shorter side one workgroup can hold (m <= 64 or 128).
//
// S = X X^T, P = b S + c S S and P X are products of rows with rows on fp16 parts (ou_parts.hip has the arithmetic).  A workgroup keeps the parts of a square
// matrix (X, S or P) in one half of its LDS and those of X transposed in the other; X and S in fp32 stay in registers, where the matrix instruction leaves its
// results: four waves, each with every second 32 x 32 block of every second row of blocks, so that a matrix of half the size keeps all of them busy.
//
// Up to 64 or 128 columns (whole_kernel) everything from the gradient to the weight is one launch: 89 x 64 x 64 with five steps take 21 us, 89 x 128 x 128 64 (47 and 134
// in slices, 91 and 140 in tiles); 19 of the 64 are matrix instructions, the rest is splitting into parts, LDS and memory.  Wider matrices are cut along their columns into at most
// kSlices slices (slice_kernel): a launch a step, in which each workgroup adds up the slices' S in order, makes P for itself, its slice of the
// next X, and that slice's share of the next S.
#include <algorithm>
#include <cmath>

#include "ou_internal.h"

namespace ou {
namespace {

typedef _Float16 H8 __attribute__((ext_vector_type(8)));
typedef _Float16 H4 __attribute__((ext_vector_type(4)));
typedef float F16 __attribute__((ext_vector_type(16)));
typedef float F4 __attribute__((ext_vector_type(4)));
typedef unsigned U2 __attribute__((ext_vector_type(2)));
typedef unsigned U4 __attribute__((ext_vector_type(4)));

constexpr int kSlices = 64;
constexpr int kUnits = 256;   // compute units

// Powers of two of a step: values to parts, and sums of parts to values.  Each step has its own, from the bound before it: P's goes with the fourth power of the bound, so one
// set for all steps, from the largest bound, loses P where the coefficients make it grow ((8.28, -23.6, 17.3), two steps, 64 x 64: X off by 150%, with these by 5e-7).
struct Scales {
  float x_up, s_up, p_up;
  float xx_down, ss_down, px_down;
};
struct AllScales {
  Scales step[OU_MAX_STEPS];
};

template <int N>
struct Shape {
  static constexpr int kSide = N / 64;           // blocks of a wave along a side: rows wave / 2 + 2 e, columns wave % 2 + 2 f
  static constexpr int kPitch = N + 8;           // halfs of a row: 16-byte accesses of neighbouring rows meet different banks
  static constexpr int kPart = N * kPitch;
  static constexpr int kBytes = 4 * kPart * 2;
  static constexpr int kResults = N * N;         // floats of a workgroup's square of results, in the order of the registers
  typedef F16 Blocks[kSide][kSide];
};

__device__ __forceinline__ int wave_of() { return __builtin_amdgcn_readfirstlane(threadIdx.x / kLanes); }

// f(e, f, q, i, j) for the lane's results: element (i, j).
template <int N, typename F>
__device__ __forceinline__ void each_result(F&& body) {
  const int lane = threadIdx.x & (kLanes - 1), wave = wave_of();
#pragma unroll
  for (int e = 0; e < Shape<N>::kSide; ++e)
#pragma unroll
    for (int f = 0; f < Shape<N>::kSide; ++f)
#pragma unroll
      for (int q = 0; q < 16; ++q)
        body(e, f, q, 32 * (wave / 2 + 2 * e) + 8 * (q / 4) + 4 * (lane / 32) + q % 4, 32 * (wave % 2 + 2 * f) + (lane & 31));
}

// sum over k of A[i][k] B[j][k] for the wave's blocks that begin inside rows x cols; the parts of A and B at a and b, `depth` a multiple of 32.  The
// products of the first parts have one sum, the smaller ones another.
template <int N>
__device__ __forceinline__ void multiply(const _Float16* a, const _Float16* b, int rows, int cols, int depth, typename Shape<N>::Blocks& sum) {
  using S = Shape<N>;
  constexpr int kSide = S::kSide;
  const int lane = threadIdx.x & (kLanes - 1), wave = wave_of();
  typename S::Blocks small, other;
  const _Float16* const pa = a + (wave / 2 * 32 + (lane & 31)) * S::kPitch + lane / 32 * 8;
  const _Float16* const pb = b + (wave % 2 * 32 + (lane & 31)) * S::kPitch + lane / 32 * 8;
  bool in_row[kSide], in_col[kSide];
#pragma unroll
  for (int e = 0; e < kSide; ++e) {
    in_row[e] = 32 * (wave / 2 + 2 * e) < rows;
    in_col[e] = 32 * (wave % 2 + 2 * e) < cols;
  }
  H8 x[2][kSide][2], y[2][kSide][2];
  auto load = [&](int to, int k) {
#pragma unroll
    for (int e = 0; e < kSide; ++e)
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        x[to][e][q] = *reinterpret_cast<const H8*>(pa + q * S::kPart + e * 64 * S::kPitch + k);
        y[to][e][q] = *reinterpret_cast<const H8*>(pb + q * S::kPart + e * 64 * S::kPitch + k);
      }
  };
  auto mma = [&](auto first, int at, int p, int q, typename S::Blocks& to) {
#pragma unroll
    for (int e = 0; e < kSide; ++e)
#pragma unroll
      for (int f = 0; f < kSide; ++f) {
        if constexpr (decltype(first)::value) {
          F16 zero;
#pragma unroll
          for (int r = 0; r < 16; ++r) zero[r] = 0;
          to[e][f] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x[at][e][p], y[at][f][q], zero, 0, 0, 0);
        } else {
          to[e][f] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x[at][e][p], y[at][f][q], to[e][f], 0, 0, 0);
        }
      }
  };
  // (a block outside rows x cols is computed from whatever stands there and never used; a wave without any block inside has nothing to do)
  if (!in_row[0] || !in_col[0]) {
#pragma unroll
    for (int e = 0; e < kSide; ++e)
#pragma unroll
      for (int f = 0; f < kSide; ++f)
#pragma unroll
        for (int r = 0; r < 16; ++r) sum[e][f][r] = 0;
    return;
  }
  auto products = [&](auto first, int at) {
    mma(first, at, 1, 0, small);
    mma(first, at, 0, 0, sum);
    if constexpr (kSide == 1) mma(first, at, 0, 1, other);   // (one block: a sum of its own, so that no instruction waits for the one before it)
    else mma(std::false_type{}, at, 0, 1, small);
  };
  load(0, 0);
  load(1, 16);
  products(std::true_type{}, 0);
  for (int k = 32; k < depth; k += 32) {
    load(0, k);
    products(std::false_type{}, 1);
    load(1, k + 16);
    products(std::false_type{}, 0);
  }
  products(std::false_type{}, 1);
#pragma unroll
  for (int e = 0; e < kSide; ++e)
#pragma unroll
    for (int f = 0; f < kSide; ++f) {
      if constexpr (kSide == 1) small[e][f] += other[e][f];
      sum[e][f] += small[e][f];
    }
}

// Parts of the wave's blocks that begin inside rows x cols, times `up`: transposed (a lane's four consecutive rows are neighbours there), and as they are
// (neighbouring lanes, which are columns, exchange halves, so that each writes two columns of one of two rows).
template <int N, bool kTurned, bool kStraight>
__device__ __forceinline__ void put(const typename Shape<N>::Blocks& v, float up, int rows, int cols, _Float16* turned, _Float16* straight) {
  using S = Shape<N>;
  const int lane = threadIdx.x & (kLanes - 1), wave = wave_of();
  const unsigned select = lane & 1 ? 0x03020706u : 0x05040100u;   // odd: the neighbour's upper half, its own; even: its own lower half, the neighbour's
#pragma unroll
  for (int e = 0; e < S::kSide; ++e)
#pragma unroll
    for (int f = 0; f < S::kSide; ++f) {
      const int i = 32 * (wave / 2 + 2 * e), j = 32 * (wave % 2 + 2 * f);
      if (i >= rows || j >= cols) continue;
      unsigned h[8], l[8];
#pragma unroll
      for (int r = 0; r < 8; ++r) split2(v[e][f][2 * r] * up, v[e][f][2 * r + 1] * up, h[r], l[r]);
      if constexpr (kTurned) {
        _Float16* const at = turned + (j + (lane & 31)) * S::kPitch + i + lane / 32 * 4;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          *reinterpret_cast<U2*>(at + 8 * g) = U2{h[2 * g], h[2 * g + 1]};
          *reinterpret_cast<U2*>(at + S::kPart + 8 * g) = U2{l[2 * g], l[2 * g + 1]};
        }
      }
      if constexpr (kStraight) {
        _Float16* const at = straight + (i + lane / 32 * 4 + (lane & 1)) * S::kPitch + j + (lane & 30);
#pragma unroll
        for (int r = 0; r < 8; ++r) {
          const unsigned hn = __builtin_amdgcn_update_dpp(0u, h[r], 0xB1, 0xf, 0xf, true), ln = __builtin_amdgcn_update_dpp(0u, l[r], 0xB1, 0xf, 0xf, true);
          _Float16* const row = at + (8 * (r / 2) + 2 * (r % 2)) * S::kPitch;
          *reinterpret_cast<unsigned*>(row) = __builtin_amdgcn_perm(hn, h[r], select);
          *reinterpret_cast<unsigned*>(row + S::kPart) = __builtin_amdgcn_perm(ln, l[r], select);
        }
      }
    }
}

// A matrix m x l of a tensor; `first` is its first element.
struct Matrix {
  int m, l;
  bool turned;
  int64_t first;
};
__device__ __forceinline__ Matrix matrix_of(const Item& it, int64_t index) {
  const bool turned = it.rows > it.cols;
  return {turned ? it.cols : it.rows, turned ? it.rows : it.cols, turned, index * it.rows * it.cols};
}

// Accesses to a matrix of a tensor go through a descriptor of it: those of elements outside read zero and write nothing, without a branch for each.  (At most
// 128 x 65536 elements: 32-bit offsets.)
template <int N>
struct Places {
  unsigned at[Shape<N>::kSide][Shape<N>::kSide][16];   // elements from the first, or far beyond the last
};
template <int N>
__device__ __forceinline__ void places_of(const Matrix& mat, bool turned, int j0, Places<N>& places) {
  each_result<N>([&](int e, int f, int q, int i, int j) {
    const unsigned at = turned ? (j0 + j) * mat.m + i : i * mat.l + j0 + j;
    places.at[e][f][q] = i < mat.m && j0 + j < mat.l ? at : 0x20000000u;
  });
}
template <typename T>
__device__ __forceinline__ __amdgpu_buffer_rsrc_t descriptor(const T* p, const Matrix& mat) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<T*>(p), 0, static_cast<int>(sizeof(T)) * mat.m * mat.l, 0x00020000);
}
// A tensor's matrix that is taller than wide is read across its rows: neighbouring lanes have elements of different rows.  kWide: four consecutive values of a lane are neighbours
// in memory, all inside or none, aligned to 16 bytes, and one request (500 x 512 x 64, five steps: 246 us instead of 313; 500 x 64 x 512 take 235).
__device__ __forceinline__ bool wide_of(const Item& it, const Matrix& mat) {
  const uintptr_t all = reinterpret_cast<uintptr_t>(it.grad) | reinterpret_cast<uintptr_t>(it.momentum) | reinterpret_cast<uintptr_t>(it.weight) |
                        reinterpret_cast<uintptr_t>(it.update);
  return mat.turned && mat.m % 4 == 0 && all % 16 == 0;
}
// f(e, f, q, element) for q = 0, 4, 8, 12 of the lane's results.
template <int N, typename F>
__device__ __forceinline__ void each_four(const Places<N>& places, F&& body) {
#pragma unroll
  for (int e = 0; e < Shape<N>::kSide; ++e)
#pragma unroll
    for (int f = 0; f < Shape<N>::kSide; ++f)
#pragma unroll
      for (int q = 0; q < 16; q += 4) body(e, f, q, places.at[e][f][q]);
}
template <int N, bool kWide>
__device__ __forceinline__ void load_f32(const float* p, const Matrix& mat, const Places<N>& places, typename Shape<N>::Blocks& v) {
  const __amdgpu_buffer_rsrc_t d = descriptor(p, mat);
  if constexpr (kWide)
    each_four<N>(places, [&](int e, int f, int q, unsigned at) {
      const F4 x = __builtin_bit_cast(F4, __builtin_amdgcn_raw_buffer_load_b128(d, static_cast<int>(at * 4u), 0, 0));
#pragma unroll
      for (int k = 0; k < 4; ++k) v[e][f][q + k] = x[k];
    });
  else each_result<N>([&](int e, int f, int q, int, int) {
    v[e][f][q] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(d, static_cast<int>(places.at[e][f][q] * 4u), 0, 0));
  });
}
template <int N, bool kWide>
__device__ __forceinline__ void store_f32(float* p, const Matrix& mat, const Places<N>& places, const typename Shape<N>::Blocks& v) {
  const __amdgpu_buffer_rsrc_t d = descriptor(p, mat);
  if constexpr (kWide)
    each_four<N>(places, [&](int e, int f, int q, unsigned at) {
      const F4 x{v[e][f][q], v[e][f][q + 1], v[e][f][q + 2], v[e][f][q + 3]};
      __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(U4, x), d, static_cast<int>(at * 4u), 0, 0);
    });
  else each_result<N>([&](int e, int f, int q, int, int) {
    __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(unsigned, static_cast<float>(v[e][f][q])), d, static_cast<int>(places.at[e][f][q] * 4u), 0, 0);
  });
}

// A square of values in the workspace stands in the order of the registers: four values of a lane in a row.
template <int N, typename F>
__device__ __forceinline__ void load_square(const float* p, F&& put) {
  constexpr int kSide = Shape<N>::kSide;
  const F4* const from = reinterpret_cast<const F4*>(p) + threadIdx.x;
#pragma unroll
  for (int e = 0; e < kSide; ++e)
#pragma unroll
    for (int f = 0; f < kSide; ++f)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const F4 v = from[((e * kSide + f) * 4 + q) * kThreads];
#pragma unroll
        for (int i = 0; i < 4; ++i) put(e, f, 4 * q + i, static_cast<float>(v[i]));
      }
}
template <int N>
__device__ __forceinline__ void store_square(float* p, const typename Shape<N>::Blocks& v) {
  constexpr int kSide = Shape<N>::kSide;
  F4* const to = reinterpret_cast<F4*>(p) + threadIdx.x;
#pragma unroll
  for (int e = 0; e < kSide; ++e)
#pragma unroll
    for (int f = 0; f < kSide; ++f)
#pragma unroll
      for (int q = 0; q < 4; ++q) to[((e * kSide + f) * 4 + q) * kThreads] = F4{v[e][f][4 * q], v[e][f][4 * q + 1], v[e][f][4 * q + 2], v[e][f][4 * q + 3]};
}

// U of the lane's elements, zero outside.  kMomentum: the momentum takes its step too.
template <int N, bool kMomentum, bool kWide>
__device__ __forceinline__ void load_direction(const Item& it, const Step& st, const Matrix& mat, const Places<N>& places, typename Shape<N>::Blocks& u) {
  if (it.dtype == SC_BF16) {
    const __amdgpu_buffer_rsrc_t d = descriptor(static_cast<const __bf16*>(it.grad) + mat.first, mat);
    if constexpr (kWide)
      each_four<N>(places, [&](int e, int f, int q, unsigned at) {
        const U2 x = __builtin_bit_cast(U2, __builtin_amdgcn_raw_buffer_load_b64(d, static_cast<int>(at * 2u), 0, 0));
#pragma unroll
        for (int k = 0; k < 4; ++k) u[e][f][q + k] = __builtin_bit_cast(float, k % 2 ? x[k / 2] & 0xffff0000u : x[k / 2] << 16);
      });
    else each_result<N>([&](int e, int f, int q, int, int) {
      const unsigned short bits = __builtin_amdgcn_raw_buffer_load_b16(d, static_cast<int>(places.at[e][f][q] * 2u), 0, 0);
      u[e][f][q] = __builtin_bit_cast(float, static_cast<unsigned>(bits) << 16);
    });
  } else {
    load_f32<N, kWide>(static_cast<const float*>(it.grad) + mat.first, mat, places, u);
  }
  if (!it.momentum) return;
  typename Shape<N>::Blocks v;
  float* const momentum = static_cast<float*>(it.momentum) + mat.first;
  const float mu = static_cast<float>(st.mu);
  load_f32<N, kWide>(momentum, mat, places, v);
  if constexpr (kMomentum) {
    each_result<N>([&](int e, int f, int q, int, int) { v[e][f][q] = mu * v[e][f][q] + u[e][f][q]; });
    store_f32<N, kWide>(momentum, mat, places, v);
  }
  const bool nesterov = st.nesterov;
  each_result<N>([&](int e, int f, int q, int, int) { u[e][f][q] = direction(u[e][f][q], static_cast<float>(v[e][f][q]), mu, nesterov); });
}

template <int N, bool kWide>
__device__ __forceinline__ void store_results(const Item& it, const Step& st, const Matrix& mat, const Places<N>& places, const typename Shape<N>::Blocks& x) {
  if (it.update) {
    if (it.dtype == SC_BF16) {
      const __amdgpu_buffer_rsrc_t d = descriptor(static_cast<const __bf16*>(it.update) + mat.first, mat);
      if constexpr (kWide)
        each_four<N>(places, [&](int e, int f, int q, unsigned at) {
          auto bits = [&](int k) { return static_cast<unsigned>(__builtin_bit_cast(unsigned short, static_cast<__bf16>(static_cast<float>(x[e][f][q + k])))); };
          __builtin_amdgcn_raw_buffer_store_b64(U2{bits(0) | bits(1) << 16, bits(2) | bits(3) << 16}, d, static_cast<int>(at * 2u), 0, 0);
        });
      else each_result<N>([&](int e, int f, int q, int, int) {
        const unsigned short bits = __builtin_bit_cast(unsigned short, static_cast<__bf16>(static_cast<float>(x[e][f][q])));
        __builtin_amdgcn_raw_buffer_store_b16(bits, d, static_cast<int>(places.at[e][f][q] * 2u), 0, 0);
      });
    } else {
      store_f32<N, kWide>(static_cast<float*>(it.update) + mat.first, mat, places, x);
    }
  }
  if (it.weight) {
    typename Shape<N>::Blocks w;
    float* const weight = static_cast<float*>(it.weight) + mat.first;
    load_f32<N, kWide>(weight, mat, places, w);
    each_result<N>([&](int e, int f, int q, int, int) { w[e][f][q] = new_weight(it, st, static_cast<float>(w[e][f][q]), static_cast<float>(x[e][f][q])); });
    store_f32<N, kWide>(weight, mat, places, w);
  }
}

// P = b S + c S S; its parts are left in `square`.  Begins and ends with the workgroup in step.
template <int N>
__device__ __forceinline__ void make_p(const Step& st, const Scales& sc, int m, int deep, _Float16* square, const typename Shape<N>::Blocks& s) {
  typename Shape<N>::Blocks r;
  put<N, true, false>(s, sc.s_up, m, m, square, nullptr);   // (symmetric)
  __syncthreads();
  multiply<N>(square, square, m, m, deep, r);
  __syncthreads();
  const float cb = static_cast<float>(st.b), scale = static_cast<float>(st.c) * sc.ss_down;
#pragma unroll
  for (int e = 0; e < Shape<N>::kSide; ++e)
#pragma unroll
    for (int f = 0; f < Shape<N>::kSide; ++f) r[e][f] = cb * s[e][f] + scale * r[e][f];
  put<N, true, false>(r, sc.p_up, m, m, square, nullptr);
  __syncthreads();
}

template <int N>
__device__ __forceinline__ void next_x(float a, float scale, const typename Shape<N>::Blocks& r, typename Shape<N>::Blocks& x) {
#pragma unroll
  for (int e = 0; e < Shape<N>::kSide; ++e)
#pragma unroll
    for (int f = 0; f < Shape<N>::kSide; ++f) x[e][f] = a * x[e][f] + scale * r[e][f];
}

// A matrix of m, l <= N.  Rows and columns of parts up to the next multiple of 32 are zeros, those beyond are never used.
template <int N>
__device__ __forceinline__ void whole(const Item* __restrict__ items, int n, int64_t unit, const Step& st, int steps, const AllScales& all) {
  using S = Shape<N>;
  extern __shared__ __attribute__((aligned(16))) _Float16 lds[];
  _Float16* const square = lds;
  _Float16* const turned_x = lds + 2 * S::kPart;
  const Item& it = items[item_of(items, n, kBlocks, unit)];
  const Matrix mat = matrix_of(it, unit - it.unit[kBlocks]);
  const bool wide = wide_of(it, mat);
  const int m = mat.m, l = mat.l, deep_l = (l + 31) / 32 * 32, deep_m = (m + 31) / 32 * 32;
  typename S::Blocks x, s, r;
  {
    Places<N> places;
    places_of<N>(mat, mat.turned, 0, places);
    if (wide) load_direction<N, true, true>(it, st, mat, places, x);
    else load_direction<N, true, false>(it, st, mat, places, x);
  }
  double sum = 0;
  each_result<N>([&](int e, int f, int q, int, int) { sum = fma(static_cast<double>(x[e][f][q]), static_cast<double>(x[e][f][q]), sum); });
  const double down = down_from(workgroup_sum(sum, reinterpret_cast<double*>(lds)), st.eps);
  each_result<N>([&](int e, int f, int q, int, int) { x[e][f][q] = static_cast<float>(static_cast<double>(x[e][f][q]) * down); });
  const float ca = static_cast<float>(st.a);
  Scales next = all.step[0];
  for (int step = 0; step < steps; ++step) {
    const Scales sc = next;
    next = all.step[min(step + 1, OU_MAX_STEPS - 1)];   // (asked for a step ahead)
    put<N, true, true>(x, sc.x_up, m, l, turned_x, square);
    __syncthreads();
    multiply<N>(square, square, m, m, deep_l, s);
    __syncthreads();
#pragma unroll
    for (int e = 0; e < S::kSide; ++e)
#pragma unroll
      for (int f = 0; f < S::kSide; ++f) s[e][f] *= sc.xx_down;
    make_p<N>(st, sc, m, deep_m, square, s);
    multiply<N>(square, turned_x, m, l, deep_m, r);
    next_x<N>(ca, sc.px_down, r, x);
    __syncthreads();
  }
  Places<N> places;
  places_of<N>(mat, mat.turned, 0, places);
  if (wide) store_results<N, true>(it, st, mat, places, x);
  else store_results<N, false>(it, st, mat, places, x);
}

template <int N>
__global__ __launch_bounds__(kThreads) void whole_kernel(const Item* __restrict__ items, int n, const Step st, int steps, const AllScales sc) {
  whole<N>(items, n, blockIdx.x, st, steps, sc);
}

// Matrices of up to 128 (`large` of them) and, after them, of up to 64.
__global__ __launch_bounds__(kThreads) void both_kernel(const Item* __restrict__ items128, int n128, int large, const Item* __restrict__ items64, int n64, const Step st,
                                                        int steps, const AllScales sc) {
  const int unit = blockIdx.x;
  if (unit < large) whole<128>(items128, n128, unit, st, steps, sc);
  else whole<64>(items64, n64, unit - large, st, steps, sc);
}

// Slices of `width` columns (a multiple of N) of a matrix of m <= N.  step 0: X from the gradient; then the step before `step` of the iteration; the last one leaves the
// results.  X and the slices' shares of S (partial) are kept in the order of the registers.  sc: of that step; next_up, next_down: x_up and xx_down of the one after it.
template <int N>
__global__ __launch_bounds__(kThreads) void slice_kernel(const Item* __restrict__ items, int n, const Step st, int step, bool last, const Scales sc, float next_up, float next_down,
                                                         const double* __restrict__ squares, float* __restrict__ X, const float* __restrict__ partial,
                                                         float* __restrict__ next_partial) {
  using S = Shape<N>;
  constexpr int kSide = S::kSide;
  extern __shared__ __attribute__((aligned(16))) _Float16 lds[];
  _Float16* const square = lds;
  _Float16* const slice = lds + 2 * S::kPart;
  const Item& it = items[item_of(items, n, kBlocks, blockIdx.x)];
  const int width = it.width, long_side = max(it.rows, it.cols), slices = (long_side + width - 1) / width;
  const int64_t unit = blockIdx.x - it.unit[kBlocks], index = unit / slices;
  const int own = static_cast<int>(unit % slices);
  const Matrix mat = matrix_of(it, index);
  const bool wide = wide_of(it, mat);
  const int m = mat.m, l = mat.l, deep_m = (m + 31) / 32 * 32, end = min(l, (own + 1) * width);
  float* const x_of = X + it.x + index * ((l + N - 1) / N) * S::kResults;   // squares of N columns
  typename S::Blocks x, s, r;
  double down = 0;
#pragma unroll
  for (int e = 0; e < kSide; ++e)
#pragma unroll
    for (int f = 0; f < kSide; ++f)
#pragma unroll
      for (int q = 0; q < 16; ++q) s[e][f][q] = 0;
  if (step == 0) {
    const int64_t per = chunks_of(static_cast<int64_t>(m) * l);
    down = down_of(squares + it.unit[kChunks] + index * per, per, st.eps, reinterpret_cast<double*>(lds));
  } else {
    const float* from = partial + (blockIdx.x - own) * static_cast<int64_t>(S::kResults);
#pragma unroll 4 / kSide
    for (int k = 0; k < slices; ++k, from += S::kResults) load_square<N>(from, [&](int e, int f, int q, float v) { s[e][f][q] += v; });
    make_p<N>(st, sc, m, deep_m, square, s);
#pragma unroll
    for (int e = 0; e < kSide; ++e)
#pragma unroll
      for (int f = 0; f < kSide; ++f)
#pragma unroll
        for (int q = 0; q < 16; ++q) s[e][f][q] = 0;
  }
  for (int j0 = own * width; j0 < end; j0 += N) {
    const int columns = min(l - j0, N);
    float* const x_here = x_of + static_cast<int64_t>(j0 / N) * S::kResults;
    Places<N> places;
    if (step == 0 || last) places_of<N>(mat, mat.turned, j0, places);
    if (step == 0) {
      if (wide) load_direction<N, false, true>(it, st, mat, places, x);
      else load_direction<N, false, false>(it, st, mat, places, x);
      each_result<N>([&](int e, int f, int q, int, int) { x[e][f][q] = static_cast<float>(static_cast<double>(x[e][f][q]) * down); });
    } else {
      load_square<N>(x_here, [&](int e, int f, int q, float v) { x[e][f][q] = v; });
      put<N, true, false>(x, sc.x_up, m, columns, slice, nullptr);
      __syncthreads();
      multiply<N>(square, slice, m, columns, deep_m, r);
      next_x<N>(static_cast<float>(st.a), sc.px_down, r, x);
      __syncthreads();
    }
    if (last) {
      if (wide) store_results<N, true>(it, st, mat, places, x);
      else store_results<N, false>(it, st, mat, places, x);
      continue;
    }
    store_square<N>(x_here, x);   // (zeros up to the next multiples of 32, beyond whatever the products were)
    // (the columns up to the next multiple of 32 are read too: they hold zeros, made of the parts' zeros)
    put<N, false, true>(x, next_up, m, columns, nullptr, slice);
    __syncthreads();
    multiply<N>(slice, slice, m, m, (columns + 31) / 32 * 32, r);
#pragma unroll
    for (int e = 0; e < kSide; ++e)
#pragma unroll
      for (int f = 0; f < kSide; ++f) s[e][f] += next_down * r[e][f];
    __syncthreads();
  }
  if (last) return;
  store_square<N>(next_partial + blockIdx.x * static_cast<int64_t>(S::kResults), s);
}

template <typename Kernel, typename... Args>
hipError_t launch(Kernel kernel, int bytes, int64_t grid, hipStream_t stream, Args... args) {
  if (bytes > 64 * 1024) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(grid)), dim3(kThreads), bytes, stream, args...);
  return hipGetLastError();
}

AllScales scales_of(const ou_config* cfg) {
  AllScales all{};
  double top = 1;
  for (int i = 0; i < cfg->steps; ++i) {
    const double square = top * top;
    const int x = exponent_of(top), s = exponent_of(square), p = exponent_of(std::fabs(cfg->b) * square + std::fabs(cfg->c) * square * square);
    all.step[i] = {std::ldexp(1.f, x), std::ldexp(1.f, s), std::ldexp(1.f, p), std::ldexp(1.f, -2 * x), std::ldexp(1.f, -2 * s), std::ldexp(1.f, -p - x)};
    top = growth(cfg, top);
  }
  return all;
}

template <int N>
hipError_t slices(const Part& p, const ou_config* cfg, const Step& st, char* base, const Item* items, hipStream_t stream) {
  const AllScales sc = scales_of(cfg);
  float* const partial[2] = {reinterpret_cast<float*>(base + p.at[0]), reinterpret_cast<float*>(base + p.at[1])};
  const double* const squares = reinterpret_cast<const double*>(base + p.at_partial);
  hipError_t e = hipSuccess;
  for (int step = 0; step <= cfg->steps && e == hipSuccess; ++step) {
    const Scales& next = sc.step[std::min(step, OU_MAX_STEPS - 1)];
    e = launch(&slice_kernel<N>, Shape<N>::kBytes, p.units[kBlocks], stream, items, static_cast<int>(p.items.size()), st, step, step == cfg->steps, sc.step[std::max(step - 1, 0)],
               next.x_up, next.xx_down, squares,
               reinterpret_cast<float*>(base + p.at_x), static_cast<const float*>(partial[(step + 1) & 1]), partial[step & 1]);
  }
  return e;
}

}  // namespace

// Every slice adds up the shares of all and makes P again, so there are fewer where a list has many matrices: as many as fill the chip, two workgroups of the smaller size a
// compute unit.  Five steps of 89 x 64 x 1024: 138 us with five slices, 159 with eleven, 164 with two; of 89 x 128 x 512: 192 with two, 271 with four; of one 64 x 8192: 117
// with 64, 147 with 16.  In the tiles of ou_parts.hip those take 274, 247 and 437, one 128 x 512 116 (here 102), 500 x 64 x 256 385 (here 136).
void slice_place(Part& p, Item& it, int64_t count, int64_t matrices, bool large) {
  const int64_t n = large ? 128 : 64, l = std::max(it.rows, it.cols);
  const int64_t slices = std::clamp<int64_t>((large ? kUnits : 2 * kUnits) / matrices, 1, kSlices);
  it.width = static_cast<int32_t>(n * ceil_div(l, n * slices));
  it.x = p.x;
  p.units[kBlocks] += count * ceil_div(l, it.width);
  p.x += count * ceil_div(l, n) * n * n;
}

void slice_layout(Part& p, Room& room, int steps, bool large) {
  if (steps == 0) return;
  const size_t square = large ? Shape<128>::kResults : Shape<64>::kResults;
  p.at_x = room(p.x * sizeof(float));
  p.at[0] = room(p.units[kBlocks] * square * sizeof(float));
  p.at[1] = room(p.units[kBlocks] * square * sizeof(float));
}

hipError_t slice_run(const Part& p, const ou_config* cfg, const Step& st, bool large, char* base, hipStream_t stream) {
  const Item* const items = reinterpret_cast<const Item*>(base + p.at_items);
  return large ? slices<128>(p, cfg, st, base, items, stream) : slices<64>(p, cfg, st, base, items, stream);
}

// A matrix of up to 64 takes a quarter of the LDS that one of up to 128 takes, so four of them share a compute unit.  Where a unit for each
// of both sizes is there, they have one launch (10 matrices of 128 and 6 of 64, five steps: 61 us, the launches of their own take 60 and 19).
hipError_t whole_run(const Part& p64, const Part& p128, const ou_config* cfg, const Step& st, char* base, hipStream_t stream) {
  const AllScales sc = scales_of(cfg);
  const Item* const items[2] = {reinterpret_cast<const Item*>(base + p64.at_items), reinterpret_cast<const Item*>(base + p128.at_items)};
  const int n[2] = {static_cast<int>(p64.items.size()), static_cast<int>(p128.items.size())};
  const int64_t units[2] = {p64.units[kBlocks], p128.units[kBlocks]};
  if (units[0] && units[1] && units[0] + units[1] <= kUnits)
    return launch(&both_kernel, Shape<128>::kBytes, units[0] + units[1], stream, items[1], n[1], static_cast<int>(units[1]), items[0], n[0], st, cfg->steps, sc);
  hipError_t e = hipSuccess;
  if (units[0]) e = launch(&whole_kernel<64>, Shape<64>::kBytes, units[0], stream, items[0], n[0], st, cfg->steps, sc);
  if (units[1] && e == hipSuccess) e = launch(&whole_kernel<128>, Shape<128>::kBytes, units[1], stream, items[1], n[1], st, cfg->steps, sc);
  return e;
}

}  // namespace ou
