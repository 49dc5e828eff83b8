// The products by element on the bfloat16 matrix cores, for widths from 2 on.
//
// An fp32 value is the sum of three bfloat16 parts h + m + l (el::split_pair), a bfloat16 row its own only part.  Rows of fp32: h h' and the five products
// h m', m h', m m', h l', l h' (what is left out is below 2^-24 of the product); rows of bfloat16 with W: three products; dW of bfloat16 rows: one.  An instruction cuts
// off what is below the last bit of the sum it adds to, so a sum of fp32 results goes over 32 indices, smaller products first, and then joins an fp32
// sum; results that are rounded to bfloat16 take one sum throughout.  Values that the parts do not stand for (not finite, beyond the largest bfloat16,
// below 2^-110) are noted, and the tile is computed by the blocks of gp_blocks.h.
//
// A workgroup: 128 rows of a bucket x 128 columns, or 128 x 128 of an element's dW over a chunk of rows, four waves of 64 x 64.  32 reduced indices of both
// operands are requested while the 32 before are multiplied, and pass through registers, where they are split, to LDS.  One set of LDS and two barriers a
// stage: the two or, of bfloat16 rows, three workgroups of a compute unit fill each other's waits (200 000 rows of bfloat16, 128 x 128: with three a tenth less than with two
// that request their rows two stages ahead).
//
// Medians of a trace, inputs from memory.  149 997 rows of fp32, 128 x 128: Y 62 us (160 MB, 2.6 TB/s; the products are 27 at the rate of a large product), dX 57, dW 64 and 16 for the
// chunks' sums; 200 000 of bfloat16: 47, 42, 37 and 16.  What bounds them is the splitting beside loads and products in turn: the matrix cores work a fifth of the cycles.  16 384 rows, 64
// elements, 1024 x 2048: Y of bfloat16 289 us (710 TFLOP/s; called in turn 285, of fp32 522: 790), dX 272, dW 341; matrix cores two fifths of the cycles in Y and dX, a tenth in dW.
#include <algorithm>
#include <type_traits>

#include "gp_blocks.h"

namespace gp {
namespace {

typedef __bf16 B8 __attribute__((ext_vector_type(8)));
typedef float F16 __attribute__((ext_vector_type(16)));
typedef float F4 __attribute__((ext_vector_type(4), aligned(4)));
typedef float F4Tight __attribute__((ext_vector_type(4)));
typedef float F2 __attribute__((ext_vector_type(2), aligned(4)));
typedef unsigned U4 __attribute__((ext_vector_type(4)));
typedef unsigned U4Loose __attribute__((ext_vector_type(4), aligned(2)));
typedef unsigned ULoose __attribute__((aligned(2)));

constexpr int kTile = 128, kStage = 32;
constexpr int kPlane = kTile * kStage;   // elements of one part of one operand: rows of 64 bytes

template <typename T>
constexpr int parts() { return sizeof(T) == 2 ? 1 : 3; }

// Rows 0..7, and the even and the odd ones of 16, have their four pieces at different places.
__device__ __forceinline__ int swizzle(int row) { return ((row >> 1) & 3) ^ ((row >> 3) & 1); }

// Eight reduced indices of one row of an operand: raw elements (request_some: the first n, zeros behind them), and as its parts in LDS.
template <typename T>
struct Eight;
template <>
struct Eight<float> {
  F4 v[2];
  __device__ __forceinline__ void request(const float* p) {
    v[0] = *reinterpret_cast<const F4*>(p);
    v[1] = *reinterpret_cast<const F4*>(p + 4);
  }
  __device__ __forceinline__ void clear() { v[0] = v[1] = F4{0, 0, 0, 0}; }
  __device__ __forceinline__ void request_some(const float* p, int n) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i / 4][i % 4] = i < n ? p[i] : 0.f;
  }
  __device__ __forceinline__ void put(__bf16* to, int plane, unsigned& low) const {
    U4 p[3];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const el::SplitPair s = el::split_pair(v[i / 2][2 * (i % 2)], v[i / 2][2 * (i % 2) + 1], low);
      p[0][i] = s.h;
      p[1][i] = s.m;
      p[2][i] = s.l;
    }
#pragma unroll
    for (int q = 0; q < 3; ++q) *reinterpret_cast<U4*>(to + q * plane) = p[q];
  }
};
template <>
struct Eight<__bf16> {
  U4 v;
  __device__ __forceinline__ void request(const __bf16* p) { v = *reinterpret_cast<const U4Loose*>(p); }
  __device__ __forceinline__ void clear() { v = U4{0, 0, 0, 0}; }
  __device__ __forceinline__ void request_some(const __bf16* p, int n) {
    const unsigned short* const bits = reinterpret_cast<const unsigned short*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const unsigned x = 2 * i < n ? bits[2 * i] : 0u, y = 2 * i + 1 < n ? bits[2 * i + 1] : 0u;
      v[i] = x | y << 16;
    }
  }
  __device__ __forceinline__ void put(__bf16* to, int, unsigned&) const { *reinterpret_cast<U4*>(to) = v; }
};

// Eight reduced indices of two neighbouring columns, from eight rows of an operand whose rows are the reduced index.
template <typename T>
struct TwoColumns;
template <>
struct TwoColumns<float> {
  F2 v[8];
  __device__ __forceinline__ void request(int i, const float* p) { v[i] = *reinterpret_cast<const F2*>(p); }
  __device__ __forceinline__ void clear_from(int n) {   // of the eight
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < n ? v[i] : F2{0, 0};
  }
  // the first column where the second one was requested as the last of the row
  __device__ __forceinline__ void shift(bool alone) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i][0] = alone ? v[i][1] : v[i][0];
  }
  __device__ __forceinline__ void put(int piece, int row, __bf16* to, unsigned& low) const {
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      U4 p[3];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const el::SplitPair s = el::split_pair(v[2 * i][c], v[2 * i + 1][c], low);
        p[0][i] = s.h;
        p[1][i] = s.m;
        p[2][i] = s.l;
      }
#pragma unroll
      for (int q = 0; q < 3; ++q) *reinterpret_cast<U4*>(to + q * kPlane + (row + c) * kStage + (piece ^ swizzle(row + c)) * 8) = p[q];
    }
  }
};
template <>
struct TwoColumns<__bf16> {
  unsigned v[8];
  __device__ __forceinline__ void request(int i, const __bf16* p) { v[i] = *reinterpret_cast<const ULoose*>(p); }
  __device__ __forceinline__ void clear_from(int n) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < n ? v[i] : 0u;
  }
  __device__ __forceinline__ void shift(bool alone) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = alone ? v[i] >> 16 : v[i];
  }
  __device__ __forceinline__ void put(int piece, int row, __bf16* to, unsigned&) const {
    U4 p[2];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const unsigned x = v[2 * i], y = v[2 * i + 1];
      p[0][i] = __builtin_amdgcn_perm(y, x, 0x05040100);
      p[1][i] = __builtin_amdgcn_perm(y, x, 0x07060302);
    }
#pragma unroll
    for (int c = 0; c < 2; ++c) *reinterpret_cast<U4*>(to + (row + c) * kStage + (piece ^ swizzle(row + c)) * 8) = p[c];
  }
};

// Sums of a wave: kR x 2 blocks of 32 x 32.
template <int kR>
using SumsOf = F16[kR][2];

template <int kR>
__device__ __forceinline__ void clear(SumsOf<kR>& s) {
#pragma unroll
  for (int e = 0; e < kR; ++e)
#pragma unroll
    for (int f = 0; f < 2; ++f)
#pragma unroll
      for (int r = 0; r < 16; ++r) s[e][f][r] = 0;
}

// Adds the products of a stage, a and b in LDS, NA and NB parts, to sum (of the blocks that begin inside `rows`): at once (kOneSum), or, a row of blocks after the other, by a sum of the stage's own.
template <int NA, int NB, int kR, bool kOneSum>
__device__ __forceinline__ void multiply(const __bf16* a, const __bf16* b, int rows, SumsOf<kR>& sum) {
  constexpr int kPlaneA = 64 * kR * kStage;
  const int lane = threadIdx.x & (kLanes - 1), wave = threadIdx.x / kLanes;
  const int first = __builtin_amdgcn_readfirstlane(wave / 2 * 32 * kR);
  const int wi = wave / 2 * 32 * kR + (lane & 31), wj = wave % 2 * 64 + (lane & 31);
  auto a_part = [&](int e, int s, int p) {
    const int i = wi + 32 * e;
    return *reinterpret_cast<const B8*>(a + p * kPlaneA + i * kStage + ((2 * s + lane / 32) ^ swizzle(i)) * 8);
  };
  auto b_part = [&](int f, int s, int p) {
    const int j = wj + 32 * f;
    return *reinterpret_cast<const B8*>(b + p * kPlane + j * kStage + ((2 * s + lane / 32) ^ swizzle(j)) * 8);
  };
  // the smallest products first; of two operands of three parts, their second parts' product too
  auto products = [&](auto&& body) {
#pragma unroll
    for (int order = (NA > NB ? NA : NB) - 1; order >= 0; --order)
#pragma unroll
      for (int p = NA - 1; p >= 0; --p)
        if (order - p >= 0 && order - p < NB) body(p, order - p);
  };
  if constexpr (kOneSum) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      if (first >= rows) return;
      B8 x[kR][NA], y[2][NB];
#pragma unroll
      for (int e = 0; e < kR; ++e)
#pragma unroll
        for (int p = 0; p < NA; ++p) x[e][p] = a_part(e, s, p);
#pragma unroll
      for (int f = 0; f < 2; ++f)
#pragma unroll
        for (int p = 0; p < NB; ++p) y[f][p] = b_part(f, s, p);
      products([&](int p, int q) {
#pragma unroll
        for (int e = 0; e < kR; ++e)
#pragma unroll
          for (int f = 0; f < 2; ++f) sum[e][f] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[e][p], y[f][q], sum[e][f], 0, 0, 0);
      });
    }
  } else {
#pragma unroll
    for (int e = 0; e < kR; ++e) {
      F16 part[2];
#pragma unroll
      for (int f = 0; f < 2; ++f)
#pragma unroll
        for (int r = 0; r < 16; ++r) part[f][r] = 0;
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        B8 x[NA], y[2][NB];
#pragma unroll
        for (int p = 0; p < NA; ++p) x[p] = a_part(e, s, p);
#pragma unroll
        for (int f = 0; f < 2; ++f)
#pragma unroll
          for (int p = 0; p < NB; ++p) y[f][p] = b_part(f, s, p);
        products([&](int p, int q) {
#pragma unroll
          for (int f = 0; f < 2; ++f) part[f] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[p], y[f][q], part[f], 0, 0, 0);
        });
      }
#pragma unroll
      for (int f = 0; f < 2; ++f) sum[e][f] += part[f];
    }
  }
}

// Has a thread of the workgroup met a value that the parts do not stand for?  (One that is not finite leaves a NaN in the sums.)
template <int kR>
__device__ __forceinline__ bool unserved(const SumsOf<kR>& sum, unsigned low, unsigned* flags) {
  float mark = 0;
#pragma unroll
  for (int e = 0; e < kR; ++e)
#pragma unroll
    for (int f = 0; f < 2; ++f)
#pragma unroll
      for (int r = 0; r < 16; ++r) mark = fmaf(sum[e][f][r], 0.f, mark);
  const bool mine = __builtin_amdgcn_ballot_w64((low & 0xffffu) != 0 || mark != 0.f) != 0;
  __syncthreads();
  if ((threadIdx.x & (kLanes - 1)) == 0) flags[threadIdx.x / kLanes] = mine;
  __syncthreads();
  return (flags[0] | flags[1] | flags[2] | flags[3]) != 0;
}

// The results, a wave's 32 x 32 after the other through its corner of LDS, which turns them so that neighbouring lanes have the pieces of 16 bytes of a row:
// f(row, column, values of a piece).  The workgroup has left the LDS.
constexpr int kPitchOut = 36;   // floats
template <typename T>
constexpr int piece_of() { return 16 / sizeof(T); }
template <typename T, int kR, typename F>
__device__ __forceinline__ void each_result(const SumsOf<kR>& sum, float* lds, F&& body) {
  constexpr int kN = piece_of<T>(), kLanesOfRow = 32 / kN;
  const int lane = threadIdx.x & (kLanes - 1), wave = threadIdx.x / kLanes;
  float* const corner = lds + wave * 32 * kPitchOut;
  const int column = lane % kLanesOfRow * kN;
#pragma unroll
  for (int e = 0; e < kR; ++e)
#pragma unroll
    for (int f = 0; f < 2; ++f) {
#pragma unroll
      for (int r = 0; r < 16; ++r) corner[(8 * (r / 4) + 4 * (lane / 32) + r % 4) * kPitchOut + (lane & 31)] = sum[e][f][r];
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      float v[16 / kN][kN];
#pragma unroll
      for (int i = 0; i < 16 / kN; ++i)
#pragma unroll
        for (int k = 0; k < kN; k += 4) {
          const F4Tight x = *reinterpret_cast<const F4Tight*>(corner + (lane / kLanesOfRow + i * (kLanes / kLanesOfRow)) * kPitchOut + column + k);
#pragma unroll
          for (int j = 0; j < 4; ++j) v[i][k + j] = x[j];
        }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
      for (int i = 0; i < 16 / kN; ++i) body(wave / 2 * 32 * kR + 32 * e + lane / kLanesOfRow + i * (kLanes / kLanesOfRow), wave % 2 * 64 + 32 * f + column, v[i]);
    }
}

// A piece of results to p, with what stands at `residual` (NULL: nothing); `inside` of its elements are there.
template <typename T, int kN>
__device__ __forceinline__ void store_piece(T* p, const T* residual, int inside, float (&v)[kN]) {
  static_assert(kN * sizeof(T) == 16, "a piece is 16 bytes");
  if (inside >= kN) {
    if constexpr (sizeof(T) == 4) {
      if (residual) {
        const F4 x = *reinterpret_cast<const F4*>(residual);
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] += x[k];
      }
      *reinterpret_cast<F4*>(p) = F4{v[0], v[1], v[2], v[3]};
    } else {
      if (residual) {
        const U4 x = *reinterpret_cast<const U4Loose*>(residual);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          v[2 * k] += el::low_half(x[k]);
          v[2 * k + 1] += el::high_half(x[k]);
        }
      }
      *reinterpret_cast<U4Loose*>(p) = U4Loose{el::pack_bf16(v[0], v[1]), el::pack_bf16(v[2], v[3]), el::pack_bf16(v[4], v[5]), el::pack_bf16(v[6], v[7])};
    }
  } else {
#pragma unroll
    for (int k = 0; k < kN; ++k)
      if (k < inside) p[k] = static_cast<T>(residual ? v[k] + static_cast<float>(residual[k]) : v[k]);
  }
}

// Tiles of 64 kR rows.  kEights: widths are multiples of 8, so a piece is all there or not at all, and no request needs a test of its own (vectors of 128: 53 us, 58
// with the tests).
template <typename T, bool kBack, int kR, bool kEights>
__global__ __launch_bounds__(kThreads, sizeof(T) == 4 ? 2 : 3) void rows_parts_kernel(const Rows a) {
  constexpr int kTileRows = 64 * kR, kPlaneX = kTileRows * kStage;
  constexpr int NX = parts<T>(), NW = 3;
  constexpr bool kOneSum = NX == 1;
  __shared__ __attribute__((aligned(16))) __bf16 lds[NX * kPlaneX + NW * kPlane];
  __shared__ int64_t offsets[kTileRows];
  __shared__ unsigned flags[kWaves];
  static_assert(sizeof(lds) >= sizeof(BlockSpace<float>), "the blocks use the same space");
  __bf16* const xs = lds;
  __bf16* const ws = lds + NX * kPlaneX;
  const int lane = threadIdx.x & (kLanes - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kLanes);
  const int columns = (a.columns + kTile - 1) / kTile;
  for (int64_t block = blockIdx.x;; block += gridDim.x) {
    int which;
    const Place p = place_of(a.group.offsets, a.elements + 1, a.n, block, columns, [&](int atoms) { return (atoms * a.components + kTileRows - 1) / kTileRows; }, &which);
    if (p.bucket < 0) return;
    const int rows = p.atoms * a.components, first = p.local * kTileRows, c0 = which * kTile;
    __syncthreads();   // (the offsets of the tile before)
    if (threadIdx.x < kTileRows) {
      const int r = min(first + static_cast<int>(threadIdx.x), rows - 1);
      offsets[threadIdx.x] = row_offset(a.group.order, a.n, p.begin, r, a.components, a.ld_dst, a.columns);
    }
    SumsOf<kR> sum;
    clear<kR>(sum);
    unsigned low = 0;
    if (p.bucket < a.elements) {
      const float* const W = static_cast<const float*>(a.W) + static_cast<int64_t>(p.bucket) * a.reduced * a.columns;
      // kR rows of X and (kBack) two of W a thread, a piece of eight of each
      const int piece = threadIdx.x % 4;
      const T* x[kR];
      int to[2];
      const float* w[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int r = i * 64 + threadIdx.x / 4;
        if (i < kR) x[i] = row_at(static_cast<const T*>(a.src), a.group.order, a.n, p.begin, min(first + r, rows - 1), a.components, a.ld_src, a.reduced);
        to[i] = r * kStage + (piece ^ swizzle(r)) * 8;
        w[i] = W + static_cast<int64_t>(min(c0 + r, a.columns - 1)) * a.reduced;
      }
      const int pair = 2 * lane;                                                   // forward: columns c0 + pair, + 1 of rows 8 wave on
      const float* const w_rows = W + min(c0 + pair, a.columns - 2);
      constexpr int kAhead = kR == 1 ? 2 : 1;   // stages of rows under way, as registers allow (of W one)
      Eight<T> xv[kAhead][kR];
      Eight<float> wv[2];
      TwoColumns<float> wc;
      auto request_rows = [&](int k, Eight<T> (&v)[kR]) {
        const int at = kEights ? min(k + 8 * piece, a.reduced - 8) : k + 8 * piece;
#pragma unroll
        for (int i = 0; i < kR; ++i) {
          if (kEights || k + kStage <= a.reduced) v[i].request(x[i] + at);
          else v[i].request_some(x[i] + at, a.reduced - at);
        }
      };
      auto request_weights = [&](int k) {
        if constexpr (kBack) {
          const int at = kEights ? min(k + 8 * piece, a.reduced - 8) : k + 8 * piece;
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            if (kEights || k + kStage <= a.reduced) wv[i].request(w[i] + at);
            else wv[i].request_some(w[i] + at, a.reduced - at);
          }
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) wc.request(i, w_rows + static_cast<int64_t>(min(k + 8 * wave + i, a.reduced - 1)) * a.columns);
        }
      };
      auto stage = [&](int k, Eight<T> (&v)[kR]) {
        if (k > 0) barrier();   // the stage before has been read
        if (k + kStage > a.reduced) {
          const bool inside = k + 8 * piece < a.reduced;
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            if (kEights && i < kR && !inside) v[i].clear();
            if (kEights && kBack && !inside) wv[i].clear();
          }
          if (!kBack) wc.clear_from(a.reduced - k - 8 * wave);
        }
        if (!kEights && !kBack && a.columns % 2) wc.shift(c0 + pair == a.columns - 1);
#pragma unroll
        for (int i = 0; i < kR; ++i) v[i].put(xs + to[i], kPlaneX, low);
        if constexpr (kBack) {
#pragma unroll
          for (int i = 0; i < 2; ++i) wv[i].put(ws + to[i], kPlane, low);
        } else {
          wc.put(wave, pair, ws, low);
        }
        if (k + kStage < a.reduced) request_weights(k + kStage);
        if (k + kAhead * kStage < a.reduced) request_rows(k + kAhead * kStage, v);
        barrier();
        multiply<NX, NW, kR, kOneSum>(xs, ws, rows - first, sum);
      };
      request_rows(0, xv[0]);
      request_weights(0);
      if (kAhead > 1 && kStage < a.reduced) request_rows(kStage, xv[kAhead - 1]);
      for (int k = 0; k < a.reduced; k += kAhead * kStage) {
        stage(k, xv[0]);
        if (kAhead > 1 && k + kStage < a.reduced) stage(k + kStage, xv[kAhead - 1]);
      }
      if (unserved<kR>(sum, low, flags)) {
        BlockSpace<float>& space = *reinterpret_cast<BlockSpace<float>*>(lds);
        for (int q = 0; q < 2 * kR; ++q)
          if (first + q / 2 * kBlock < rows && c0 + q % 2 * kBlock < a.columns)
            rows_block<T, float, kBack>(a, p.bucket, p.begin, rows, first + q / 2 * kBlock, c0 + q % 2 * kBlock, space);
        continue;
      }
    } else {
      __syncthreads();   // the offsets
    }
    T* const dst = static_cast<T*>(a.dst);
    const T* const residual = static_cast<const T*>(a.residual);
    each_result<T, kR>(sum, reinterpret_cast<float*>(lds), [&](int row, int column, float (&v)[piece_of<T>()]) {
      if (first + row >= rows || c0 + column >= a.columns) return;
      const int64_t at = offsets[row] + c0 + column;
      store_piece(dst + at, residual ? residual + at : nullptr, kEights ? 8 : a.columns - c0 - column, v);
    });
  }
}

template <typename T>
__global__ __launch_bounds__(kThreads, 2) void outer_parts_kernel(const Outer a) {
  constexpr int N = parts<T>();
  __shared__ __attribute__((aligned(16))) __bf16 lds[2 * N * kPlane < 9216 ? 9216 : 2 * N * kPlane];
  __shared__ unsigned flags[kWaves];
  static_assert(sizeof(lds) >= sizeof(BlockSpace<float>), "the blocks use the same space");
  __bf16* const xs = lds;
  __bf16* const gs = lds + N * kPlane;
  const int lane = threadIdx.x & (kLanes - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kLanes);
  const int col_tiles = (a.k_out + kTile - 1) / kTile, tiles = (a.k_in + kTile - 1) / kTile * col_tiles;
  for (int64_t block = blockIdx.x;; block += gridDim.x) {
    int which;
    Chunk c;
    if (!chunk_of(a, block, tiles, &c, &which)) return;
    const int k0 = which / col_tiles * kTile, c0 = which % col_tiles * kTile;
    float* const out = static_cast<float*>(c.partial ? a.partial : a.dW) + c.matrix * a.k_in * a.k_out;
    const int pair = 2 * lane;
    const T* const x_at = static_cast<const T*>(a.X) + min(k0 + pair, a.k_in - 2);
    const T* const g_at = static_cast<const T*>(a.dY) + min(c0 + pair, a.k_out - 2);
    TwoColumns<T> xv, gv;
    // Lane i holds where the wave's row 8 wave + i of a stage begins (i < 8); it is looked up a stage before the row is requested.
    int64_t x_row, g_row;
    auto look_up = [&](int r) {
      const int row = min(r + 8 * wave + (lane & 7), c.last - 1);
      const int atom_of = a.components == 1 ? row : static_cast<int>(static_cast<unsigned>(row) / static_cast<unsigned>(a.components));
      const int64_t atom = min(static_cast<unsigned>(a.group.order[c.begin + atom_of]), static_cast<unsigned>(a.n - 1));
      const int component = row - atom_of * a.components;
      x_row = atom * a.ld_in + static_cast<int64_t>(component) * a.k_in;
      g_row = atom * a.ld_out + static_cast<int64_t>(component) * a.k_out;
    };
    auto of_lane = [](int64_t v, int i) {
      const unsigned low_word = __builtin_amdgcn_readlane(static_cast<unsigned>(v), i), high_word = __builtin_amdgcn_readlane(static_cast<unsigned>(v >> 32), i);
      return static_cast<int64_t>(static_cast<uint64_t>(high_word) << 32 | low_word);
    };
    auto request = [&] {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        xv.request(i, x_at + of_lane(x_row, i));
        gv.request(i, g_at + of_lane(g_row, i));
      }
    };
    SumsOf<2> sum;
    clear<2>(sum);
    unsigned low = 0;
    __syncthreads();
    if (c.first < c.last) {
      look_up(c.first);
      request();
      look_up(c.first + kStage);
    }
    for (int r = c.first; r < c.last; r += kStage) {
      if (r > c.first) barrier();
      if (r + kStage > c.last) {
        xv.clear_from(c.last - r - 8 * wave);
        gv.clear_from(c.last - r - 8 * wave);
      }
      if (a.k_in % 2) xv.shift(k0 + pair == a.k_in - 1);
      if (a.k_out % 2) gv.shift(c0 + pair == a.k_out - 1);
      xv.put(wave, pair, xs, low);
      gv.put(wave, pair, gs, low);
      if (r + kStage < c.last) {
        request();
        look_up(r + 2 * kStage);
      }
      barrier();
      multiply<N, N, 2, false>(xs, gs, a.k_in - k0, sum);
    }
    if (unserved<2>(sum, low, flags)) {
      BlockSpace<float>& space = *reinterpret_cast<BlockSpace<float>*>(lds);
      for (int q = 0; q < 4; ++q)
        if (k0 + q / 2 * kBlock < a.k_in && c0 + q % 2 * kBlock < a.k_out)
          outer_block<T, float>(a, a.group.order, c.begin, c.first, c.last, k0 + q / 2 * kBlock, c0 + q % 2 * kBlock, out, space);
      continue;
    }
    each_result<float, 2>(sum, reinterpret_cast<float*>(lds), [&](int k, int column, float (&v)[4]) {
      if (k0 + k < a.k_in && c0 + column < a.k_out)
        store_piece<float>(out + static_cast<int64_t>(k0 + k) * a.k_out + c0 + column, nullptr, a.k_out - c0 - column, v);
    });
  }
}

}  // namespace

bool parts_serve(const gp_config* c) { return c->dtype != SC_F64 && c->k_in >= 2 && c->k_out >= 2; }

namespace {

template <typename T, int kR>
hipError_t launch_rows_of(const gp_config* c, const Rows& a, bool back, hipStream_t stream) {
  const int64_t tiles = ceil_div(a.n * c->components, 64 * kR) + std::min<int64_t>(c->num_elements + 1, a.n);
  const dim3 grid(static_cast<unsigned>(std::min(kMaxGrid, ceil_div(tiles * ceil_div(a.columns, kTile), kXcds) * kXcds)));
  const bool eights = a.reduced % 8 == 0 && a.columns % 8 == 0;
  auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, stream, a); };
  if (back) eights ? launch(&rows_parts_kernel<T, true, kR, true>) : launch(&rows_parts_kernel<T, true, kR, false>);
  else eights ? launch(&rows_parts_kernel<T, false, kR, true>) : launch(&rows_parts_kernel<T, false, kR, false>);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rows_parts(const gp_config* c, const Rows& a, bool back, hipStream_t stream) {
  // Tiles of half the height where the others would not fill the compute units (10 000 rows, 128 x 128: 11 us instead of 14, 1000 rows, 512 x 512: 26 instead of 36;
  // 30 000 rows, 128 x 128: 23 instead of 20).
  const int64_t tiles = (ceil_div(a.n * c->components, 128) + std::min<int64_t>(c->num_elements + 1, a.n)) * ceil_div(a.columns, kTile);
  const bool half = tiles <= 256;
  if (c->dtype == SC_F32) return half ? launch_rows_of<float, 1>(c, a, back, stream) : launch_rows_of<float, 2>(c, a, back, stream);
  return half ? launch_rows_of<__bf16, 1>(c, a, back, stream) : launch_rows_of<__bf16, 2>(c, a, back, stream);
}

hipError_t launch_outer_parts(const gp_config* c, const Outer& a, hipStream_t stream) {
  const int64_t chunks = c->num_elements + a.n * c->components / a.per, tiles = ceil_div(c->k_in, kTile) * ceil_div(c->k_out, kTile);
  const dim3 grid(static_cast<unsigned>(std::min(kMaxGrid, ceil_div(chunks * tiles, kXcds) * kXcds)));
  if (c->dtype == SC_F32) hipLaunchKernelGGL(outer_parts_kernel<float>, grid, dim3(kThreads), 0, stream, a);
  else hipLaunchKernelGGL(outer_parts_kernel<__bf16>, grid, dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace gp
