// The orthogonalised update of matrices that one workgroup can hold: everything from the gradient to the weight in one launch.
//
// X, S = X X^T and P = b S + c S S are products of rows with rows on fp16 parts (ou_parts.hip has the arithmetic).  The workgroup keeps the parts of X
// transposed in one half of its LDS and, one after the other, those of X, S and P in the other; X and S in fp32 stay in registers, where the matrix
// instruction leaves its results.  With at most 128 reduced indices the products of the first parts have one sum and the smaller ones another.
#include <cmath>

#include "ou_internal.h"

namespace ou {
namespace {

typedef _Float16 H8 __attribute__((ext_vector_type(8)));
typedef _Float16 H4 __attribute__((ext_vector_type(4)));
typedef float F16 __attribute__((ext_vector_type(16)));

// The powers of two of every step: they travel as kernel arguments.
struct Exponents {
  int8_t x[OU_MAX_STEPS + 1], s[OU_MAX_STEPS], p[OU_MAX_STEPS];
};

template <int N>
struct Shape {
  static constexpr int kThreads = N == 128 ? 512 : 256;
  static constexpr int kWaves = kThreads / kLanes;
  static constexpr int kBlocks = N / 32;                     // 32 x 32 blocks along a side
  static constexpr int kMine = kBlocks * kBlocks / kWaves;   // blocks of a wave: neighbours in a row
  static constexpr int kPitch = N + 8;                       // halfs of a row: 16-byte accesses of neighbouring rows meet different banks
  static constexpr int kPart = N * kPitch;
  static constexpr int kWide = N + 1;                        // floats of a row where X is in fp32
  static constexpr int kBytes = 4 * kPart * 2;
  static_assert(N * kWide * 4 <= 2 * kPart * 2, "X in fp32 fits the half of the parts of X");
};

// sum over k of A[i][k] B[j][k] for the wave's blocks; the parts of A and B at a and b, `depth` a multiple of 32.
template <int N, int kMine>
__device__ __forceinline__ void multiply(const _Float16* a, const _Float16* b, int rb, int cb, int depth, F16 (&sum)[kMine]) {
  using S = Shape<N>;
  const int lane = threadIdx.x & (kLanes - 1);
  F16 small[kMine];
#pragma unroll
  for (int e = 0; e < kMine; ++e)
#pragma unroll
    for (int r = 0; r < 16; ++r) sum[e][r] = small[e][r] = 0;
  const _Float16* const pa = a + (rb * 32 + (lane & 31)) * S::kPitch + lane / 32 * 8;
  const _Float16* const pb = b + (cb * 32 + (lane & 31)) * S::kPitch + lane / 32 * 8;
  for (int k = 0; k < depth; k += 16) {
    H8 x[2], y[kMine][2];
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      x[q] = *reinterpret_cast<const H8*>(pa + q * S::kPart + k);
#pragma unroll
      for (int e = 0; e < kMine; ++e) y[e][q] = *reinterpret_cast<const H8*>(pb + q * S::kPart + e * 32 * S::kPitch + k);
    }
#pragma unroll
    for (int e = 0; e < kMine; ++e) small[e] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x[1], y[e][0], small[e], 0, 0, 0);
#pragma unroll
    for (int e = 0; e < kMine; ++e) sum[e] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x[0], y[e][0], sum[e], 0, 0, 0);
#pragma unroll
    for (int e = 0; e < kMine; ++e) small[e] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x[0], y[e][1], small[e], 0, 0, 0);
  }
#pragma unroll
  for (int e = 0; e < kMine; ++e) sum[e] += small[e];
}

// Parts of a block's results, transposed: a lane's four consecutive rows are neighbours there.
template <int N>
__device__ __forceinline__ void put_turned(const F16& v, float up, int rb, int cb, _Float16* to) {
  using S = Shape<N>;
  const int lane = threadIdx.x & (kLanes - 1);
  _Float16* const at = to + (cb * 32 + (lane & 31)) * S::kPitch + rb * 32 + lane / 32 * 4;
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    H4 h, l;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      _Float16 x, y;
      split(v[4 * g + i] * up, x, y);
      h[i] = x;
      l[i] = y;
    }
    *reinterpret_cast<H4*>(at + 8 * g) = h;
    *reinterpret_cast<H4*>(at + S::kPart + 8 * g) = l;
  }
}
// And as they are.
template <int N>
__device__ __forceinline__ void put_straight(const F16& v, float up, int rb, int cb, _Float16* to) {
  using S = Shape<N>;
  const int lane = threadIdx.x & (kLanes - 1);
  _Float16* const at = to + (rb * 32 + lane / 32 * 4) * S::kPitch + cb * 32 + (lane & 31);
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    _Float16 x, y;
    split(v[r] * up, x, y);
    at[(8 * (r / 4) + r % 4) * S::kPitch] = x;
    at[S::kPart + (8 * (r / 4) + r % 4) * S::kPitch] = y;
  }
}

template <int N>
__global__ __launch_bounds__(Shape<N>::kThreads) void small_kernel(const Item* __restrict__ items, int n, const Step st, int steps, const Exponents ex) {
  using S = Shape<N>;
  constexpr int kMine = S::kMine, kEach = N * N / S::kThreads;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  _Float16* const square = reinterpret_cast<_Float16*>(lds);              // X, S, P
  _Float16* const turned_x = square + 2 * S::kPart;
  float* const wide = reinterpret_cast<float*>(lds);                      // X in fp32, [m][kWide]
  double* const slots = reinterpret_cast<double*>(turned_x);              // (before the parts come)
  const Item& it = items[item_of(items, n, kBlocks, blockIdx.x)];
  const bool turned = it.rows > it.cols;
  const int m = turned ? it.cols : it.rows, l = turned ? it.rows : it.cols, size = m * l;
  const int64_t first = (blockIdx.x - it.unit[kBlocks]) * size;
  const int lane = threadIdx.x & (kLanes - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kLanes);

  // U and its norm
  float u[kEach];
  double sum = 0;
  const float mu = static_cast<float>(st.mu);
#pragma unroll
  for (int e = 0; e < kEach; ++e) {
    const int i = threadIdx.x + e * S::kThreads;
    u[e] = 0;
    if (i < size) {
      float g = gradient<float>(it, first + i);
      if (it.momentum) {
        float* const p = static_cast<float*>(it.momentum) + first + i;
        const float v = mu * *p + g;
        *p = v;
        g = direction(g, v, mu, st.nesterov);
      }
      u[e] = g;
    }
    sum = fma(static_cast<double>(u[e]), static_cast<double>(u[e]), sum);
  }
#pragma unroll
  for (int d = 32; d > 0; d /= 2) sum += __shfl_xor(sum, d);
  if (lane == 0) slots[wave] = sum;
  __syncthreads();
  sum = slots[0];
#pragma unroll
  for (int w = 1; w < S::kWaves; ++w) sum += slots[w];
  const double down = 1.0 / (sqrt(sum) + st.eps);
#pragma unroll
  for (int e = 0; e < kEach; ++e) u[e] = static_cast<float>(static_cast<double>(u[e]) * down);
  if (steps == 0) {
#pragma unroll
    for (int e = 0; e < kEach; ++e)
      if (threadIdx.x + e * S::kThreads < size) finish(it, st, first + threadIdx.x + e * S::kThreads, u[e]);
    return;
  }

  // X in fp32 through LDS to where the matrix instruction will have its results
  const int columns = it.cols;
#pragma unroll
  for (int e = 0; e < kEach; ++e) {
    const int i = threadIdx.x + e * S::kThreads;
    if (i < size) wide[turned ? i % columns * S::kWide + i / columns : i / columns * S::kWide + i % columns] = u[e];
  }
  __syncthreads();
  const int rb = wave * kMine / S::kBlocks, cb = wave * kMine % S::kBlocks;
  const bool rows_inside = rb * 32 < m;
  F16 x[kMine], s[kMine], r[kMine];
#pragma unroll
  for (int e = 0; e < kMine; ++e)
#pragma unroll
    for (int q = 0; q < 16; ++q) {
      const int i = rb * 32 + 8 * (q / 4) + 4 * (lane / 32) + q % 4, j = (cb + e) * 32 + (lane & 31);
      x[e][q] = i < m && j < l ? wide[i * S::kWide + j] : 0.f;
    }
  __syncthreads();
  // rows and columns up to the next multiple of 32 are zeros, the others are never read
  auto put_x = [&](int step) {
    const float up = __builtin_ldexpf(1.f, ex.x[step]);
#pragma unroll
    for (int e = 0; e < kMine; ++e)
      if (rows_inside && (cb + e) * 32 < l) {
        put_straight<N>(x[e], up, rb, cb + e, square);
        put_turned<N>(x[e], up, rb, cb + e, turned_x);
      }
  };
  put_x(0);
  const int deep_l = (l + 31) / 32 * 32, deep_m = (m + 31) / 32 * 32;
  const bool in_square = rows_inside && cb * 32 < m, in_x = rows_inside && cb * 32 < l;
  const float ca = static_cast<float>(st.a), cb_ = static_cast<float>(st.b), cc = static_cast<float>(st.c);
  for (int step = 0; step < steps; ++step) {
    __syncthreads();
    if (in_square) multiply<N, kMine>(square, square, rb, cb, deep_l, s);
    __syncthreads();
    if (in_square) {
      const float scale = __builtin_ldexpf(1.f, -2 * ex.x[step]), up = __builtin_ldexpf(1.f, ex.s[step]);
#pragma unroll
      for (int e = 0; e < kMine; ++e) {
        s[e] *= scale;
        if ((cb + e) * 32 < m) put_turned<N>(s[e], up, rb, cb + e, square);
      }
    }
    __syncthreads();
    if (in_square) multiply<N, kMine>(square, square, rb, cb, deep_m, r);
    __syncthreads();
    if (in_square) {
      const float scale = cc * __builtin_ldexpf(1.f, -2 * ex.s[step]), up = __builtin_ldexpf(1.f, ex.p[step]);
#pragma unroll
      for (int e = 0; e < kMine; ++e) {
        r[e] = cb_ * s[e] + scale * r[e];
        if ((cb + e) * 32 < m) put_turned<N>(r[e], up, rb, cb + e, square);
      }
    }
    __syncthreads();
    if (in_x) {
      multiply<N, kMine>(square, turned_x, rb, cb, deep_m, r);
      const float scale = __builtin_ldexpf(1.f, -ex.p[step] - ex.x[step]);
#pragma unroll
      for (int e = 0; e < kMine; ++e) x[e] = ca * x[e] + scale * r[e];
    }
    __syncthreads();
    if (step + 1 < steps) put_x(step + 1);
  }

  // results in the tensor's order
#pragma unroll
  for (int e = 0; e < kMine; ++e)
#pragma unroll
    for (int q = 0; q < 16; ++q) {
      const int i = rb * 32 + 8 * (q / 4) + 4 * (lane / 32) + q % 4, j = (cb + e) * 32 + (lane & 31);
      if (i < m && j < l) wide[i * S::kWide + j] = x[e][q];
    }
  __syncthreads();
#pragma unroll 4
  for (int e = 0; e < kEach; ++e) {
    const int i = threadIdx.x + e * S::kThreads;
    if (i < size) finish(it, st, first + i, wide[turned ? i % columns * S::kWide + i / columns : i / columns * S::kWide + i % columns]);
  }
}

template <int N>
hipError_t launch(const Part& p, const ou_config* cfg, const Step& st, const Exponents& ex, const Item* items, hipStream_t stream) {
  using S = Shape<N>;
  if (S::kBytes > 64 * 1024) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(&small_kernel<N>), hipFuncAttributeMaxDynamicSharedMemorySize, S::kBytes);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(small_kernel<N>, dim3(static_cast<unsigned>(p.units[kBlocks])), dim3(S::kThreads), S::kBytes, stream, items,
                     static_cast<int>(p.items.size()), st, cfg->steps, ex);
  return hipGetLastError();
}

}  // namespace

hipError_t small_run(const Part& p, const ou_config* cfg, const Step& st, bool wide, const Item* items, hipStream_t stream) {
  Exponents ex{};
  double top = 1;
  for (int i = 0; i < cfg->steps; ++i) {
    const double square = top * top;
    ex.x[i] = static_cast<int8_t>(exponent_of(top));
    ex.s[i] = static_cast<int8_t>(exponent_of(square));
    ex.p[i] = static_cast<int8_t>(exponent_of(std::fabs(cfg->b) * square + std::fabs(cfg->c) * square * square));
    top = growth(cfg, top);
  }
  return wide ? launch<128>(p, cfg, st, ex, items, stream) : launch<64>(p, cfg, st, ex, items, stream);
}

}  // namespace ou
