// The orthogonalised update of matrices whose shorter side one workgroup can hold (m <= 64 or 128).
//
// S = X X^T, P = b S + c S S and P X are products of rows with rows on fp16 parts (ou_parts.hip has the arithmetic).  A workgroup keeps the parts of a square
// matrix (X, S or P) in one half of its LDS and those of X transposed in the other; X and S in fp32 stay in registers, where the matrix instruction leaves its
// results: four waves, each with every second 32 x 32 block of every second row of blocks, so that a matrix of half the size keeps all of them busy.
//
// Up to 64 or 128 columns (whole_kernel) everything from the gradient to the weight is one launch.  Wider matrices are cut along their columns into at most
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

constexpr int kSlices = 32;

// The powers of two of every step: they travel as kernel arguments.
struct Exponents {
  int8_t x[OU_MAX_STEPS + 1], s[OU_MAX_STEPS], p[OU_MAX_STEPS];
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
#pragma unroll
  for (int e = 0; e < kSide; ++e)
#pragma unroll
    for (int f = 0; f < kSide; ++f)
#pragma unroll
      for (int r = 0; r < 16; ++r) sum[e][f][r] = small[e][f][r] = other[e][f][r] = 0;
  const _Float16* const pa = a + (wave / 2 * 32 + (lane & 31)) * S::kPitch + lane / 32 * 8;
  const _Float16* const pb = b + (wave % 2 * 32 + (lane & 31)) * S::kPitch + lane / 32 * 8;
  bool in_row[kSide], in_col[kSide];
#pragma unroll
  for (int e = 0; e < kSide; ++e) {
    in_row[e] = 32 * (wave / 2 + 2 * e) < rows;
    in_col[e] = 32 * (wave % 2 + 2 * e) < cols;
  }
  if (!in_row[0] || !in_col[0]) return;
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
  auto mma = [&](int at, int p, int q, typename S::Blocks& to) {
#pragma unroll
    for (int e = 0; e < kSide; ++e)
#pragma unroll
      for (int f = 0; f < kSide; ++f)
        if (in_row[e] && in_col[f]) to[e][f] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x[at][e][p], y[at][f][q], to[e][f], 0, 0, 0);
  };
  auto products = [&](int at) {
    mma(at, 1, 0, small);
    mma(at, 0, 0, sum);
    if constexpr (kSide == 1) mma(at, 0, 1, other);   // (one block: a sum of its own, so that no instruction waits for the one before it)
    else mma(at, 0, 1, small);
  };
  load(0, 0);
  for (int k = 0; k < depth; k += 32) {
    load(1, k + 16);
    products(0);
    if (k + 32 < depth) load(0, k + 32);
    products(1);
  }
#pragma unroll
  for (int e = 0; e < kSide; ++e)
#pragma unroll
    for (int f = 0; f < kSide; ++f) {
      if constexpr (kSide == 1) small[e][f] += other[e][f];
      sum[e][f] += small[e][f];
    }
}

// Parts of the wave's blocks that begin inside rows x cols, transposed: a lane's four consecutive rows are neighbours there.
template <int N>
__device__ __forceinline__ void put_turned(const typename Shape<N>::Blocks& v, float up, int rows, int cols, _Float16* to) {
  using S = Shape<N>;
  const int lane = threadIdx.x & (kLanes - 1), wave = wave_of();
#pragma unroll
  for (int e = 0; e < S::kSide; ++e)
#pragma unroll
    for (int f = 0; f < S::kSide; ++f) {
      const int i = 32 * (wave / 2 + 2 * e), j = 32 * (wave % 2 + 2 * f);
      if (i >= rows || j >= cols) continue;
      _Float16* const at = to + (j + (lane & 31)) * S::kPitch + i + lane / 32 * 4;
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        H4 h, l;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          _Float16 x, y;
          split(v[e][f][4 * g + k] * up, x, y);
          h[k] = x;
          l[k] = y;
        }
        *reinterpret_cast<H4*>(at + 8 * g) = h;
        *reinterpret_cast<H4*>(at + S::kPart + 8 * g) = l;
      }
    }
}
// And as they are: neighbouring lanes (columns) exchange halves, so that each writes two columns of one of two rows.
template <int N>
__device__ __forceinline__ void put_straight(const typename Shape<N>::Blocks& v, float up, int rows, int cols, _Float16* to) {
  using S = Shape<N>;
  typedef _Float16 H2 __attribute__((ext_vector_type(2)));
  const int lane = threadIdx.x & (kLanes - 1), wave = wave_of();
  const unsigned select = lane & 1 ? 0x03020706u : 0x05040100u;   // odd: upper halves of the neighbour's and its own; even: lower halves of its own and the neighbour's
#pragma unroll
  for (int e = 0; e < S::kSide; ++e)
#pragma unroll
    for (int f = 0; f < S::kSide; ++f) {
      const int i = 32 * (wave / 2 + 2 * e), j = 32 * (wave % 2 + 2 * f);
      if (i >= rows || j >= cols) continue;
      _Float16* const at = to + (i + lane / 32 * 4 + (lane & 1)) * S::kPitch + j + (lane & 30);
#pragma unroll
      for (int r = 0; r < 16; r += 2) {
        _Float16 h0, l0, h1, l1;
        split(v[e][f][r] * up, h0, l0);
        split(v[e][f][r + 1] * up, h1, l1);
        const unsigned h = __builtin_bit_cast(unsigned, H2{h0, h1}), l = __builtin_bit_cast(unsigned, H2{l0, l1});
        const unsigned hn = __builtin_amdgcn_update_dpp(0u, h, 0xB1, 0xf, 0xf, true), ln = __builtin_amdgcn_update_dpp(0u, l, 0xB1, 0xf, 0xf, true);
        _Float16* const row = at + (8 * (r / 4) + r % 4) * S::kPitch;
        *reinterpret_cast<unsigned*>(row) = __builtin_amdgcn_perm(hn, h, select);
        *reinterpret_cast<unsigned*>(row + S::kPart) = __builtin_amdgcn_perm(ln, l, select);
      }
    }
}

// A matrix m x l and where its element (i, j) stands in the tensor.
struct Matrix {
  int m, l;
  bool turned;
  int64_t first;   // of the matrix in the tensor
  __device__ __forceinline__ int64_t at(int i, int j) const { return first + (turned ? static_cast<int64_t>(j) * m + i : static_cast<int64_t>(i) * l + j); }
};
__device__ __forceinline__ Matrix matrix_of(const Item& it, int64_t index) {
  const bool turned = it.rows > it.cols;
  return {turned ? it.cols : it.rows, turned ? it.rows : it.cols, turned, index * it.rows * it.cols};
}

// U of the lane's elements of columns j0 on, zero outside.  kMomentum: the momentum takes its step too.  (All requests before the first store.)
template <int N, bool kMomentum>
__device__ __forceinline__ void load_direction(const Item& it, const Step& st, const Matrix& mat, int j0, typename Shape<N>::Blocks& u) {
  typename Shape<N>::Blocks old;
  each_result<N>([&](int e, int f, int q, int i, int j) { u[e][f][q] = i < mat.m && j0 + j < mat.l ? gradient<float>(it, mat.at(i, j0 + j)) : 0.f; });
  if (!it.momentum) return;
  float* const momentum = static_cast<float*>(it.momentum);
  const float mu = static_cast<float>(st.mu);
  each_result<N>([&](int e, int f, int q, int i, int j) { old[e][f][q] = i < mat.m && j0 + j < mat.l ? momentum[mat.at(i, j0 + j)] : 0.f; });
  each_result<N>([&](int e, int f, int q, int i, int j) {
    float v = old[e][f][q];
    if constexpr (kMomentum) {
      v = mu * v + u[e][f][q];
      if (i < mat.m && j0 + j < mat.l) momentum[mat.at(i, j0 + j)] = v;
    }
    u[e][f][q] = direction(u[e][f][q], v, mu, st.nesterov);
  });
}

template <int N>
__device__ __forceinline__ void store_results(const Item& it, const Step& st, const Matrix& mat, int j0, const typename Shape<N>::Blocks& x) {
  if (it.update) {
    each_result<N>([&](int e, int f, int q, int i, int j) {
      if (i < mat.m && j0 + j < mat.l) put_update<float>(it, mat.at(i, j0 + j), x[e][f][q]);
    });
  }
  if (it.weight) {
    typename Shape<N>::Blocks old;
    float* const weight = static_cast<float*>(it.weight);
    each_result<N>([&](int e, int f, int q, int i, int j) { old[e][f][q] = i < mat.m && j0 + j < mat.l ? weight[mat.at(i, j0 + j)] : 0.f; });
    each_result<N>([&](int e, int f, int q, int i, int j) {
      if (i < mat.m && j0 + j < mat.l) weight[mat.at(i, j0 + j)] = new_weight(it, st, old[e][f][q], x[e][f][q]);
    });
  }
}

// P = b S + c S S from the sums of parts in s; its parts are left in `square`.  Begins and ends with the workgroup in step.
template <int N>
__device__ __forceinline__ void make_p(const Step& st, const Exponents& ex, int step, int m, int deep, _Float16* square, typename Shape<N>::Blocks& s) {
  constexpr int kSide = Shape<N>::kSide;
  typename Shape<N>::Blocks r;
  put_turned<N>(s, __builtin_ldexpf(1.f, ex.s[step]), m, m, square);   // (symmetric)
  __syncthreads();
  multiply<N>(square, square, m, m, deep, r);
  __syncthreads();
  const float cb = static_cast<float>(st.b), scale = static_cast<float>(st.c) * __builtin_ldexpf(1.f, -2 * ex.s[step]);
#pragma unroll
  for (int e = 0; e < kSide; ++e)
#pragma unroll
    for (int f = 0; f < kSide; ++f) r[e][f] = cb * s[e][f] + scale * r[e][f];
  put_turned<N>(r, __builtin_ldexpf(1.f, ex.p[step]), m, m, square);
  __syncthreads();
}

template <int N>
__device__ __forceinline__ void scale_by(float v, typename Shape<N>::Blocks& s) {
#pragma unroll
  for (int e = 0; e < Shape<N>::kSide; ++e)
#pragma unroll
    for (int f = 0; f < Shape<N>::kSide; ++f) s[e][f] *= v;
}
template <int N>
__device__ __forceinline__ void next_x(float a, float scale, const typename Shape<N>::Blocks& r, typename Shape<N>::Blocks& x) {
#pragma unroll
  for (int e = 0; e < Shape<N>::kSide; ++e)
#pragma unroll
    for (int f = 0; f < Shape<N>::kSide; ++f) x[e][f] = a * x[e][f] + scale * r[e][f];
}

// A matrix of m, l <= N.  Rows and columns of parts up to the next multiple of 32 are zeros, those beyond are never read.
template <int N>
__global__ __launch_bounds__(kThreads) void whole_kernel(const Item* __restrict__ items, int n, const Step st, int steps, const Exponents ex) {
  using S = Shape<N>;
  extern __shared__ __attribute__((aligned(16))) _Float16 lds[];
  _Float16* const square = lds;
  _Float16* const turned_x = lds + 2 * S::kPart;
  const Item& it = items[item_of(items, n, kBlocks, blockIdx.x)];
  const Matrix mat = matrix_of(it, blockIdx.x - it.unit[kBlocks]);
  const int m = mat.m, l = mat.l, deep_l = (l + 31) / 32 * 32, deep_m = (m + 31) / 32 * 32;
  typename S::Blocks x, s, r;
  load_direction<N, true>(it, st, mat, 0, x);
  double sum = 0;
  each_result<N>([&](int e, int f, int q, int, int) { sum = fma(static_cast<double>(x[e][f][q]), static_cast<double>(x[e][f][q]), sum); });
  const double down = 1.0 / (sqrt(workgroup_sum(sum, reinterpret_cast<double*>(lds))) + st.eps);
  each_result<N>([&](int e, int f, int q, int, int) { x[e][f][q] = static_cast<float>(static_cast<double>(x[e][f][q]) * down); });
  for (int step = 0; step < steps; ++step) {
    const float up = __builtin_ldexpf(1.f, ex.x[step]);
    put_straight<N>(x, up, m, l, square);
    put_turned<N>(x, up, m, l, turned_x);
    __syncthreads();
    multiply<N>(square, square, m, m, deep_l, s);
    __syncthreads();
    scale_by<N>(__builtin_ldexpf(1.f, -2 * ex.x[step]), s);
    make_p<N>(st, ex, step, m, deep_m, square, s);
    multiply<N>(square, turned_x, m, l, deep_m, r);
    next_x<N>(static_cast<float>(st.a), __builtin_ldexpf(1.f, -ex.p[step] - ex.x[step]), r, x);
    __syncthreads();
  }
  store_results<N>(it, st, mat, 0, x);
}

// Slices of `width` columns (a multiple of N) of a matrix of m <= N.  step 0: X from the gradient; then the step before `step` of the iteration; the last one leaves the
// results.  partial: the slices' shares of S, in the order of the registers.
template <int N>
__global__ __launch_bounds__(kThreads) void slice_kernel(const Item* __restrict__ items, int n, const Step st, int step, bool last, const Exponents ex,
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
  const int m = mat.m, l = mat.l, deep_m = (m + 31) / 32 * 32, end = min(l, (own + 1) * width);
  float* const x_of = X + it.x + mat.first;
  typename S::Blocks x, s, r;
  double down = 0;
  if (step == 0) {
    const int64_t per = chunks_of(static_cast<int64_t>(m) * l);
    down = down_of(squares + it.unit[kChunks] + index * per, per, st.eps, reinterpret_cast<double*>(lds));
  } else {
    const float* from = partial + (blockIdx.x - own) * static_cast<int64_t>(S::kResults) + threadIdx.x;
#pragma unroll
    for (int e = 0; e < kSide; ++e)
#pragma unroll
      for (int f = 0; f < kSide; ++f)
#pragma unroll
        for (int q = 0; q < 16; ++q) s[e][f][q] = 0;
#pragma unroll 2
    for (int k = 0; k < slices; ++k, from += S::kResults) {
#pragma unroll
      for (int e = 0; e < kSide; ++e)
#pragma unroll
        for (int f = 0; f < kSide; ++f)
#pragma unroll
          for (int q = 0; q < 16; ++q) s[e][f][q] += from[((e * kSide + f) * 16 + q) * kThreads];
    }
    make_p<N>(st, ex, step - 1, m, deep_m, square, s);
  }
#pragma unroll
  for (int e = 0; e < kSide; ++e)
#pragma unroll
    for (int f = 0; f < kSide; ++f)
#pragma unroll
      for (int q = 0; q < 16; ++q) s[e][f][q] = 0;
  for (int j0 = own * width; j0 < end; j0 += N) {
    const int columns = min(l - j0, N);
    if (step == 0) {
      load_direction<N, false>(it, st, mat, j0, x);
      each_result<N>([&](int e, int f, int q, int, int) { x[e][f][q] = static_cast<float>(static_cast<double>(x[e][f][q]) * down); });
    } else {
      each_result<N>([&](int e, int f, int q, int i, int j) { x[e][f][q] = i < m && j0 + j < l ? x_of[static_cast<int64_t>(i) * l + j0 + j] : 0.f; });
      put_turned<N>(x, __builtin_ldexpf(1.f, ex.x[step - 1]), m, columns, slice);
      __syncthreads();
      multiply<N>(square, slice, m, columns, deep_m, r);
      next_x<N>(static_cast<float>(st.a), __builtin_ldexpf(1.f, -ex.p[step - 1] - ex.x[step - 1]), r, x);
      __syncthreads();
    }
    if (last) {
      store_results<N>(it, st, mat, j0, x);
      continue;
    }
    each_result<N>([&](int e, int f, int q, int i, int j) {
      if (i < m && j0 + j < l) x_of[static_cast<int64_t>(i) * l + j0 + j] = x[e][f][q];
    });
    // (columns beyond the last one of the matrix hold zeros or what came of the parts' zeros; they are inside the multiple of 32 that is read)
    put_straight<N>(x, __builtin_ldexpf(1.f, ex.x[step]), m, columns, slice);
    __syncthreads();
    multiply<N>(slice, slice, m, m, (columns + 31) / 32 * 32, r);
    const float scale = __builtin_ldexpf(1.f, -2 * ex.x[step]);
#pragma unroll
    for (int e = 0; e < kSide; ++e)
#pragma unroll
      for (int f = 0; f < kSide; ++f) s[e][f] += scale * r[e][f];
    __syncthreads();
  }
  if (last) return;
  float* const to = next_partial + blockIdx.x * static_cast<int64_t>(S::kResults) + threadIdx.x;
#pragma unroll
  for (int e = 0; e < kSide; ++e)
#pragma unroll
    for (int f = 0; f < kSide; ++f)
#pragma unroll
      for (int q = 0; q < 16; ++q) to[((e * kSide + f) * 16 + q) * kThreads] = s[e][f][q];
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

Exponents exponents_of(const ou_config* cfg) {
  Exponents ex{};
  double top = 1;
  for (int i = 0; i < cfg->steps; ++i) {
    const double square = top * top;
    ex.x[i] = static_cast<int8_t>(exponent_of(top));
    ex.s[i] = static_cast<int8_t>(exponent_of(square));
    ex.p[i] = static_cast<int8_t>(exponent_of(std::fabs(cfg->b) * square + std::fabs(cfg->c) * square * square));
    top = growth(cfg, top);
  }
  ex.x[cfg->steps] = static_cast<int8_t>(exponent_of(top));
  return ex;
}

template <int N>
hipError_t slices(const Part& p, const ou_config* cfg, const Step& st, char* base, const Item* items, hipStream_t stream) {
  const Exponents ex = exponents_of(cfg);
  float* const partial[2] = {reinterpret_cast<float*>(base + p.at[0]), reinterpret_cast<float*>(base + p.at[1])};
  const double* const squares = reinterpret_cast<const double*>(base + p.at_partial);
  hipError_t e = hipSuccess;
  for (int step = 0; step <= cfg->steps && e == hipSuccess; ++step)
    e = launch(&slice_kernel<N>, Shape<N>::kBytes, p.units[kBlocks], stream, items, static_cast<int>(p.items.size()), st, step, step == cfg->steps, ex, squares,
               reinterpret_cast<float*>(base + p.at_x), static_cast<const float*>(partial[(step + 1) & 1]), partial[step & 1]);
  return e;
}

}  // namespace

void slice_place(Part& p, Item& it, int64_t count, bool large) {
  const int64_t n = large ? 128 : 64, l = std::max(it.rows, it.cols);
  it.width = static_cast<int32_t>(n * ceil_div(l, n * kSlices));
  it.x = p.x;
  p.units[kBlocks] += count * ceil_div(l, it.width);
  p.x += count * it.rows * it.cols;
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

hipError_t whole_run(const Part& p, const ou_config* cfg, const Step& st, bool large, char* base, hipStream_t stream) {
  const Exponents ex = exponents_of(cfg);
  const Item* const items = reinterpret_cast<const Item*>(base + p.at_items);
  const int n = static_cast<int>(p.items.size());
  return large ? launch(&whole_kernel<128>, Shape<128>::kBytes, p.units[kBlocks], stream, items, n, st, cfg->steps, ex)
               : launch(&whole_kernel<64>, Shape<64>::kBytes, p.units[kBlocks], stream, items, n, st, cfg->steps, ex);
}

}  // namespace ou
