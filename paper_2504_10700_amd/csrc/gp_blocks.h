// 64 x 64 blocks of the products by element in fp32 and fp64 matrix instructions (el_tile.h has their operand layout): what serves every width and every value.
#pragma once
#include "el_tile.h"
#include "gp_internal.h"

namespace gp {

using el::Mma;

constexpr int kBlock = 64;
constexpr int kDepth = 16;
constexpr int kPitch = kBlock + 4;

template <typename TA>
struct BlockSpace {
  TA a[kDepth][kPitch], b[kDepth][kPitch];
};

__device__ __forceinline__ void barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }   // (requests to memory stay under way)

// Rows `first` on of a bucket, columns c0 on, of Y or (kBack: W is read transposed) dX.
template <typename T, typename TA, bool kBack>
__device__ __forceinline__ void rows_block(const Rows& a, int bucket, int begin, int rows, int first, int c0, BlockSpace<TA>& space) {
  typedef typename Mma<TA>::acc_t Acc;
  const int lane = threadIdx.x & (kLanes - 1), wave = threadIdx.x / kLanes;
  Acc acc[4];
#pragma unroll
  for (int t = 0; t < 4; ++t) acc[t] = Acc{0, 0, 0, 0};
  if (bucket < a.elements) {
    const TA* const W = static_cast<const TA*>(a.W) + static_cast<int64_t>(bucket) * a.reduced * a.columns;
    const int xr = threadIdx.x / 4, xk = threadIdx.x % 4 * 4;   // 64 rows x 4 pieces of 4
    const T* const x = row_at(static_cast<const T*>(a.src), a.group.order, a.n, begin, min(first + xr, rows - 1), a.components, a.ld_src, a.reduced);
    TA xv[4], wv[4];   // 16 reduced indices, requested while the 16 before are multiplied
    auto request = [&](int k) {
#pragma unroll
      for (int i = 0; i < 4; ++i) xv[i] = k + xk + i < a.reduced ? static_cast<TA>(x[k + xk + i]) : TA(0);
      if constexpr (kBack) {   // W [column][reduced]
        const int c = min(c0 + static_cast<int>(threadIdx.x) / 4, a.columns - 1);
#pragma unroll
        for (int i = 0; i < 4; ++i) wv[i] = k + xk + i < a.reduced ? W[static_cast<int64_t>(c) * a.reduced + k + xk + i] : TA(0);
      } else {                 // W [reduced][column]
        const int r = k + threadIdx.x / 16, c = c0 + threadIdx.x % 16 * 4;
#pragma unroll
        for (int i = 0; i < 4; ++i) wv[i] = r < a.reduced && c + i < a.columns ? W[static_cast<int64_t>(r) * a.columns + c + i] : TA(0);
      }
    };
    request(0);
    for (int k = 0; k < a.reduced; k += kDepth) {
      barrier();
#pragma unroll
      for (int i = 0; i < 4; ++i) space.a[xk + i][xr] = xv[i];
      if constexpr (kBack) {
#pragma unroll
        for (int i = 0; i < 4; ++i) space.b[xk + i][threadIdx.x / 4] = wv[i];
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) space.b[threadIdx.x / 16][threadIdx.x % 16 * 4 + i] = wv[i];
      }
      if (k + kDepth < a.reduced) request(k + kDepth);
      barrier();
#pragma unroll
      for (int s = 0; s < kDepth / 4; ++s) {
        const TA xo = space.a[4 * s + lane / 16][16 * wave + (lane & 15)];
#pragma unroll
        for (int t = 0; t < 4; ++t) acc[t] = Mma<TA>::mma(xo, space.b[4 * s + lane / 16][16 * t + (lane & 15)], acc[t]);
      }
    }
  }
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int row = first + 16 * wave + Mma<TA>::row(lane, r);
    if (row >= rows) continue;
    T* const y = row_at(static_cast<T*>(a.dst), a.group.order, a.n, begin, row, a.components, a.ld_dst, a.columns);
    const T* const base = a.residual ? static_cast<const T*>(a.residual) + (y - static_cast<T*>(a.dst)) : nullptr;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const int c = c0 + 16 * t + (lane & 15);
      if (c < a.columns) y[c] = static_cast<T>(base ? acc[t][r] + static_cast<TA>(base[c]) : acc[t][r]);
    }
  }
}

// The block (k0, c0) of an element's matrix, of its rows first..last - 1, to `out`.
template <typename T, typename TA>
__device__ __forceinline__ void outer_block(const Outer& a, const int32_t* order, int begin, int first, int last, int k0, int c0, TA* out, BlockSpace<TA>& space) {
  typedef typename Mma<TA>::acc_t Acc;
  const int lane = threadIdx.x & (kLanes - 1), wave = threadIdx.x / kLanes;
  Acc acc[4];
#pragma unroll
  for (int t = 0; t < 4; ++t) acc[t] = Acc{0, 0, 0, 0};
  const int lr = threadIdx.x / 16, lc = threadIdx.x % 16 * 4;
  TA xv[4], gv[4];   // 16 rows, requested while the 16 before are multiplied
  auto request = [&](int r) {
    const int row = min(r + lr, last - 1);
    const bool inside = r + lr < last;
    const T* const x = row_at(static_cast<const T*>(a.X), order, a.n, begin, row, a.components, a.ld_in, a.k_in);
    const T* const g = row_at(static_cast<const T*>(a.dY), order, a.n, begin, row, a.components, a.ld_out, a.k_out);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      xv[i] = inside && k0 + lc + i < a.k_in ? static_cast<TA>(x[k0 + lc + i]) : TA(0);
      gv[i] = inside && c0 + lc + i < a.k_out ? static_cast<TA>(g[c0 + lc + i]) : TA(0);
    }
  };
  if (first < last) request(first);
  for (int r = first; r < last; r += kDepth) {
    barrier();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      space.a[lr][lc + i] = xv[i];
      space.b[lr][lc + i] = gv[i];
    }
    if (r + kDepth < last) request(r + kDepth);
    barrier();
#pragma unroll
    for (int s = 0; s < kDepth / 4; ++s) {
      const TA xo = space.a[4 * s + lane / 16][16 * wave + (lane & 15)];
#pragma unroll
      for (int t = 0; t < 4; ++t) acc[t] = Mma<TA>::mma(xo, space.b[4 * s + lane / 16][16 * t + (lane & 15)], acc[t]);
    }
  }
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int k = k0 + 16 * wave + Mma<TA>::row(lane, r);
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const int c = c0 + 16 * t + (lane & 15);
      if (k < a.k_in && c < a.k_out) out[static_cast<int64_t>(k) * a.k_out + c] = acc[t][r];
    }
  }
}

// What a chunk's workgroup sums and where it goes.
struct Chunk {
  int begin, first, last;
  int64_t matrix;      // of the partial ones or of dW
  bool partial;
};
__device__ __forceinline__ bool chunk_of(const Outer& a, int64_t block, int each, Chunk* c, int* which) {
  const Place p = place_of(a.group.offsets, a.elements, a.n, block, each, [&](int atoms) { return chunks_of(atoms * a.components, a.per); }, which);
  if (p.bucket < 0) return false;
  c->begin = p.begin;
  c->first = p.local * a.per;
  c->last = min(p.atoms * a.components, c->first + a.per);
  c->partial = p.units > 1;
  c->matrix = c->partial ? p.slots + p.local : p.bucket;
  return !c->partial || c->matrix < a.slots;   // (with a grouping of something else there can be more: they stay out of memory)
}

}  // namespace gp
