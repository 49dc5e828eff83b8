// The dense layer of include/dl.h: products with bias, activation and residual, their gradients and the second-order pass.
//
// Every step is a product C[m][n] = sum_k A[m][k] B[k][n] whose operands are made while they are staged
// (G = dY act'(Z) never exists in memory) and whose result is finished where it stands in the accumulators:
//
//   forward   rows x k_out   A = X    B = W      epilogue + b, act, + residual -> Y, Z
//   dX        rows x k_in    A = G    B = W^T
//   dW, db    k_in x k_out   A = X^T  B = G      the rows cut into ranges, partial results summed by a second launch in order
//   V         rows x k_out   A = HX   B = W      epilogue V act'(Z) -> ddY, S = V dY act''(Z) -> workspace
//   X2        rows x k_in    A = S    B = W^T
//   W2, b2    k_in x k_out   A = X^T  B = S, then A = HX^T  B = G on the same accumulators
#include <algorithm>
#include <cstring>

#include "dl_gate.h"
#include "el_tile.h"

namespace dl {
namespace {

using el::Mma;
using sc::align_up;
using sc::DeviceGuard;
using sc::kLanes;
using sc::misaligned;
using sc::set_error;

constexpr int kThreads = 256;
constexpr int kTile = 64;      // rows and columns of a workgroup's tile: four waves of 32 x 32
constexpr int kDepth = 16;     // reduction index per staged step
constexpr int kPad = kTile + 4;
constexpr int kXcds = 8;

// One row-major tensor as an operand: element (r, c) at p[r * ld + c].
template <typename T>
struct Matrix {
  const T* p;
  int64_t ld;
};

enum Source { kPlain, kGated };   // kGated: dY act'(Z)

template <typename T, typename TA>
__device__ __forceinline__ void load4(const Matrix<T>& m, int64_t r, int64_t c, int64_t rows, int64_t cols, TA (&v)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = TA(0);
  if (r >= rows || c >= cols) return;
  const T* p = m.p + r * m.ld + c;
  if (c + 4 <= cols) {
    typedef T Vec __attribute__((ext_vector_type(4), aligned(sizeof(T))));   // wide accesses need element alignment only
    const Vec x = *reinterpret_cast<const Vec*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = static_cast<TA>(x[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (c + i < cols) v[i] = static_cast<TA>(p[i]);
  }
}

template <typename TA, typename T, Source kSource>
struct Operand {
  Matrix<T> x, z;   // z: pre-activations beside x = dY (kGated)
  int act;
  __device__ __forceinline__ void load(int64_t r, int64_t c, int64_t rows, int64_t cols, TA (&v)[4]) const {
    load4(x, r, c, rows, cols, v);
    if constexpr (kSource == kGated) {
      TA g[4];
      load4(z, r, c, rows, cols, g);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] *= Gate<TA>::first(act, g[i]);
    }
  }
};

// Adds to acc the product over k in [k0, k1) of the 64 x 64 tile at (m0, n0).  kAlongM: A is stored [k][m], otherwise [m][k];
// kAlongN: B is stored [k][n], otherwise [n][k].  sum: column sums of B, per staging thread, if wanted.
template <typename TA, bool kAlongM, bool kAlongN, bool kSum, typename A, typename B>
__device__ __forceinline__ void tile_product(const A& a, const B& b, int64_t m0, int64_t n0, int64_t m_end, int64_t n_end,
                                             int64_t k0, int64_t k1, TA* as, TA* bs, typename Mma<TA>::acc_t (&acc)[2][2],
                                             TA (&sum)[4]) {
  const int t = threadIdx.x, lane = t & (kLanes - 1), wave = t / kLanes;
  const int wm = (wave / 2) * 32, wn = (wave % 2) * 32;
  TA va[4], vb[4];
  auto fetch = [&](int64_t k) {
    if constexpr (kAlongM)
      a.load(k + t / 16, m0 + (t % 16) * 4, k1, m_end, va);
    else
      a.load(m0 + t / 4, k + (t % 4) * 4, m_end, k1, va);
    if constexpr (kAlongN)
      b.load(k + t / 16, n0 + (t % 16) * 4, k1, n_end, vb);
    else
      b.load(n0 + t / 4, k + (t % 4) * 4, n_end, k1, vb);
  };
  auto stage = [&]() {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (kAlongM) as[(t / 16) * kPad + (t % 16) * 4 + i] = va[i];
      else as[((t % 4) * 4 + i) * kPad + t / 4] = va[i];
      if constexpr (kAlongN) bs[(t / 16) * kPad + (t % 16) * 4 + i] = vb[i];
      else bs[((t % 4) * 4 + i) * kPad + t / 4] = vb[i];
      if constexpr (kSum) sum[i] += vb[i];
    }
  };
  if (k0 < k1) fetch(k0);
  for (int64_t k = k0; k < k1; k += kDepth) {
    __syncthreads();
    stage();
    __syncthreads();
    if (k + kDepth < k1) fetch(k + kDepth);
#pragma unroll
    for (int s = 0; s < kDepth / 4; ++s) {
      const int row = (s * 4 + lane / 16) * kPad + (lane & 15);
      TA fa[2], fb[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        fa[i] = as[row + wm + i * 16];
        fb[i] = bs[row + wn + i * 16];
      }
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) acc[i][j] = Mma<TA>::mma(fa[i], fb[j], acc[i][j]);
    }
  }
}

// Calls f(m, n, value) for the elements of the tile that lie inside the result.
template <typename TA, typename F>
__device__ __forceinline__ void each_result(int64_t m0, int64_t n0, int64_t m_end, int64_t n_end,
                                            const typename Mma<TA>::acc_t (&acc)[2][2], F&& f) {
  const int lane = threadIdx.x & (kLanes - 1), wave = threadIdx.x / kLanes;
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int64_t m = m0 + (wave / 2) * 32 + i * 16 + Mma<TA>::row(lane, r);
        const int64_t n = n0 + (wave % 2) * 32 + j * 16 + (lane & 15);
        if (m < m_end && n < n_end) f(m, n, acc[i][j][r]);
      }
}

// The tiles of a result with many rows: all column tiles of a row tile go to one XCD (workgroups are dealt out to the XCDs in turn), whose
// L2 then holds the rows that they share.
struct TileWalk {
  int64_t row_tiles, col_tiles;
  __host__ __device__ int64_t count() const { return (row_tiles + kXcds - 1) / kXcds * kXcds * col_tiles; }
  __device__ bool at(int64_t t, int64_t* row, int64_t* col) const {
    const int64_t local = t / kXcds;
    *row = local / col_tiles * kXcds + t % kXcds;
    *col = local % col_tiles;
    return *row < row_tiles;
  }
};

template <typename TA>
struct Zero {
  typename Mma<TA>::acc_t acc[2][2];
  __device__ Zero() {
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) acc[i][j] = typename Mma<TA>::acc_t{0, 0, 0, 0};
  }
};

template <typename TS, typename TA>
__global__ __launch_bounds__(kThreads) void forward_kernel(TileWalk walk, int64_t rows, int k_in, int k_out, int64_t ld_out, int act,
                                                           Matrix<TS> X, Matrix<TA> W, const TA* __restrict__ bias,
                                                           const TS* __restrict__ residual, TS* __restrict__ Y, TS* __restrict__ Z) {
  __shared__ TA as[kDepth * kPad], bs[kDepth * kPad];
  const Operand<TA, TS, kPlain> a{X, X, 0};
  const Operand<TA, TA, kPlain> b{W, W, 0};
  for (int64_t t = blockIdx.x; t < walk.count(); t += gridDim.x) {
    int64_t row, col;
    if (!walk.at(t, &row, &col)) continue;
    Zero<TA> c;
    TA none[4];
    tile_product<TA, false, true, false>(a, b, row * kTile, col * kTile, rows, k_out, 0, k_in, as, bs, c.acc, none);
    each_result<TA>(row * kTile, col * kTile, rows, k_out, c.acc, [&](int64_t m, int64_t n, TA z) {
      const int64_t at = m * ld_out + n;
      if (bias) z += bias[n];
      if (Z) Z[at] = static_cast<TS>(z);
      TA y = Gate<TA>::value(act, z);
      if (residual) y += static_cast<TA>(residual[at]);
      Y[at] = static_cast<TS>(y);
    });
  }
}

// dX (and X2, whose source is S): A = the source, B = W transposed.
template <typename TS, typename TA, typename TG, Source kSource>
__global__ __launch_bounds__(kThreads) void dx_kernel(TileWalk walk, int64_t rows, int k_in, int k_out, int64_t ld_in,
                                                      Operand<TA, TG, kSource> g, Matrix<TA> W, TS* __restrict__ dX) {
  __shared__ TA as[kDepth * kPad], bs[kDepth * kPad];
  const Operand<TA, TA, kPlain> b{W, W, 0};
  for (int64_t t = blockIdx.x; t < walk.count(); t += gridDim.x) {
    int64_t row, col;
    if (!walk.at(t, &row, &col)) continue;
    Zero<TA> c;
    TA none[4];
    tile_product<TA, false, false, false>(g, b, row * kTile, col * kTile, rows, k_in, 0, k_out, as, bs, c.acc, none);
    each_result<TA>(row * kTile, col * kTile, rows, k_in, c.acc,
                    [&](int64_t m, int64_t n, TA v) { dX[m * ld_in + n] = static_cast<TS>(v); });
  }
}

template <typename TS, typename TA>
__global__ __launch_bounds__(kThreads) void v_kernel(TileWalk walk, int64_t rows, int k_in, int k_out, int64_t ld_out, int act,
                                                     Matrix<TS> HX, Matrix<TA> W, const TS* __restrict__ Z, const TS* __restrict__ dY,
                                                     TS* __restrict__ ddY, TA* __restrict__ S) {
  __shared__ TA as[kDepth * kPad], bs[kDepth * kPad];
  const Operand<TA, TS, kPlain> a{HX, HX, 0};
  const Operand<TA, TA, kPlain> b{W, W, 0};
  for (int64_t t = blockIdx.x; t < walk.count(); t += gridDim.x) {
    int64_t row, col;
    if (!walk.at(t, &row, &col)) continue;
    Zero<TA> c;
    TA none[4];
    tile_product<TA, false, true, false>(a, b, row * kTile, col * kTile, rows, k_out, 0, k_in, as, bs, c.acc, none);
    each_result<TA>(row * kTile, col * kTile, rows, k_out, c.acc, [&](int64_t m, int64_t n, TA v) {
      const int64_t at = m * ld_out + n;
      if (Z) {
        TA first, second;
        Gate<TA>::both(act, static_cast<TA>(Z[at]), &first, &second);
        if (S) S[m * k_out + n] = v * static_cast<TA>(dY[at]) * second;
        v *= first;
      }
      ddY[at] = static_cast<TS>(v);
    });
  }
}

// Partial dW (and db) of one range of rows per workgroup: tile (m, n) of the range's row of `part`, [k_in][k_out] then [k_out].
// kTwo: A2, B2 are added on the same accumulators (the second-order pass); column sums are those of the first pair.
template <typename TA, typename TX, typename TB, Source kB, typename TB2, Source kB2, bool kTwo>
__global__ __launch_bounds__(kThreads) void dw_kernel(int64_t rows, int64_t per, int k_in, int k_out, int want_dw, int want_db,
                                                      Matrix<TX> X, Operand<TA, TB, kB> B, Matrix<TX> X2, Operand<TA, TB2, kB2> B2,
                                                      TA* __restrict__ dW, TA* __restrict__ db, int64_t stride) {
  __shared__ TA as[kDepth * kPad], bs[kDepth * kPad];
  __shared__ TA sums[16][kTile];
  const int col_tiles = (k_out + kTile - 1) / kTile, row_tiles = (k_in + kTile - 1) / kTile;
  const int64_t tiles = static_cast<int64_t>(col_tiles) * row_tiles;
  const int64_t range = blockIdx.x / tiles, tile = blockIdx.x % tiles;
  const int64_t m0 = tile / col_tiles * kTile, n0 = tile % col_tiles * kTile;
  const int64_t k0 = range * per, k1 = min(rows, k0 + per);
  const Operand<TA, TX, kPlain> a{X, X, 0}, a2{X2, X2, 0};
  Zero<TA> c;
  TA sum[4] = {0, 0, 0, 0}, none[4];
  tile_product<TA, true, true, true>(a, B, m0, n0, k_in, k_out, k0, k1, as, bs, c.acc, sum);
  if constexpr (kTwo) tile_product<TA, true, true, false>(a2, B2, m0, n0, k_in, k_out, k0, k1, as, bs, c.acc, none);
  if (want_dw)
    each_result<TA>(m0, n0, k_in, k_out, c.acc, [&](int64_t m, int64_t n, TA v) { dW[range * stride + m * k_out + n] = v; });
  if (want_db && m0 == 0) {
    const int t = threadIdx.x;
#pragma unroll
    for (int i = 0; i < 4; ++i) sums[t / 16][(t % 16) * 4 + i] = sum[i];
    __syncthreads();
    if (t < kTile && n0 + t < k_out) {
      TA s = 0;
      for (int i = 0; i < 16; ++i) s += sums[i][t];
      db[range * stride + n0 + t] = s;
    }
  }
}

// out[i] = sum over the ranges of part[range][i], in order: [0, n_dw) to dW, the rest to db.  No range at all: zeros.
template <typename TA>
__global__ __launch_bounds__(kThreads) void sum_ranges_kernel(const TA* __restrict__ part, int64_t ranges, int64_t stride, int64_t n_dw,
                                                              int64_t n_db, TA* __restrict__ dW, TA* __restrict__ db) {
  for (int64_t i = blockIdx.x * static_cast<int64_t>(kThreads) + threadIdx.x; i < n_dw + n_db; i += static_cast<int64_t>(gridDim.x) * kThreads) {
    TA s = 0;
    for (int64_t r = 0; r < ranges; ++r) s += part[r * stride + i];
    if (i < n_dw) {
      if (dW) dW[i] = s;
    } else if (db) {
      db[i - n_dw] = s;
    }
  }
}

template <typename TS>
__global__ __launch_bounds__(kThreads) void zero_rows_kernel(int64_t rows, int cols, int64_t ld, TS* __restrict__ p) {
  for (int64_t i = blockIdx.x * static_cast<int64_t>(kThreads) + threadIdx.x; i < rows * cols; i += static_cast<int64_t>(gridDim.x) * kThreads)
    p[i / cols * ld + i % cols] = static_cast<TS>(0.f);
}

// ---- host side

size_t row_size(const dl_config* c) { return c->dtype == SC_F64 ? 8 : c->dtype == SC_F32 ? 4 : 2; }
size_t weight_size(const dl_config* c) { return c->dtype == SC_F64 ? 8 : 4; }
int64_t ld_in(const dl_config* c) { return c->ld_in ? c->ld_in : c->k_in; }
int64_t ld_out(const dl_config* c) { return c->ld_out ? c->ld_out : c->k_out; }

sc_status check_config(const char* fn, const dl_config* cfg, int64_t n) {
  auto bad = [&](sc_status st, const char* what) { return set_error(st, std::string(fn) + ": " + what); };
  if (!cfg) return bad(SC_ERR_INVALID_ARG, "cfg is NULL");
  if (cfg->struct_size != static_cast<int32_t>(sizeof(dl_config)))
    return bad(SC_ERR_INVALID_ARG, "struct_size does not match this library's dl_config");
  if (cfg->k_in < 1 || cfg->k_out < 1) return bad(SC_ERR_INVALID_ARG, "k_in or k_out < 1");
  if (cfg->k_in > DL_MAX_WIDTH || cfg->k_out > DL_MAX_WIDTH) return bad(SC_ERR_UNSUPPORTED, "k_in or k_out above DL_MAX_WIDTH");
  if (cfg->activation < DL_NONE || cfg->activation > DL_GELU) return bad(SC_ERR_INVALID_ARG, "bad activation");
  if (cfg->dtype != SC_F32 && cfg->dtype != SC_F64 && cfg->dtype != SC_BF16) return bad(SC_ERR_INVALID_ARG, "bad dtype");
  const int64_t most = int64_t(1) << 32;
  if (cfg->ld_in != 0 && (cfg->ld_in < cfg->k_in || cfg->ld_in > most)) return bad(SC_ERR_INVALID_ARG, "ld_in below k_in or above 2^32");
  if (cfg->ld_out != 0 && (cfg->ld_out < cfg->k_out || cfg->ld_out > most))
    return bad(SC_ERR_INVALID_ARG, "ld_out below k_out or above 2^32");
  if (n < 0 || n > (int64_t(1) << 30)) return bad(SC_ERR_INVALID_ARG, "n_rows outside 0..2^30");
  return SC_OK;
}

int64_t tiles_of(int64_t n) { return (n + kTile - 1) / kTile; }

// Rows per range of the dW launch: about four workgroups per CU together, no range below 256 rows.
int64_t rows_per_range(const dl_config* c, int64_t n) {
  const int64_t tiles = tiles_of(c->k_in) * tiles_of(c->k_out);
  const int64_t ranges = std::max<int64_t>(1, 1024 / tiles);
  const int64_t per = std::max<int64_t>(256, (n + ranges - 1) / ranges);
  return (per + kDepth - 1) / kDepth * kDepth;
}

int64_t range_count(const dl_config* c, int64_t n) {
  const int64_t per = rows_per_range(c, n);
  return (n + per - 1) / per;
}

int64_t range_stride(const dl_config* c) { return static_cast<int64_t>(c->k_in) * c->k_out + c->k_out; }

// Workspace: [ S of the second-order pass ][ partial dW and db per range of rows ].
size_t s_bytes(const dl_config* c, int64_t n) {
  return c->activation == DL_NONE || c->activation == DL_RELU ? 0 : align_up(static_cast<size_t>(n) * c->k_out * weight_size(c), 256);
}

size_t workspace_bytes(const dl_config* c, int64_t n) {
  if (n == 0) return 256;
  return s_bytes(c, n) + align_up(static_cast<size_t>(range_count(c, n)) * range_stride(c) * weight_size(c), 256) + 256;
}

template <typename T>
Matrix<T> matrix(const void* p, int64_t ld) {
  return {static_cast<const T*>(p), ld};
}

unsigned grid_of(int64_t n) { return static_cast<unsigned>(std::min<int64_t>(std::max<int64_t>(n, 1), 1 << 22)); }

template <typename TS, typename TA>
struct Calls {
  const dl_config* c;
  int64_t n;
  hipStream_t stream;

  hipError_t forward(const void* X, const void* W, const void* b, const void* residual, void* Y, void* Z) const {
    const TileWalk walk{tiles_of(n), tiles_of(c->k_out)};
    hipLaunchKernelGGL((forward_kernel<TS, TA>), dim3(grid_of(walk.count())), dim3(kThreads), 0, stream, walk, n, c->k_in, c->k_out,
                       ld_out(c), c->activation, matrix<TS>(X, ld_in(c)), matrix<TA>(W, c->k_out), static_cast<const TA*>(b),
                       static_cast<const TS*>(residual), static_cast<TS*>(Y), static_cast<TS*>(Z));
    return hipGetLastError();
  }

  template <typename TG, Source kSource>
  hipError_t dx(const Operand<TA, TG, kSource>& g, const void* W, void* dX) const {
    const TileWalk walk{tiles_of(n), tiles_of(c->k_in)};
    hipLaunchKernelGGL((dx_kernel<TS, TA, TG, kSource>), dim3(grid_of(walk.count())), dim3(kThreads), 0, stream, walk, n, c->k_in, c->k_out,
                       ld_in(c), g, matrix<TA>(W, c->k_out), static_cast<TS*>(dX));
    return hipGetLastError();
  }

  template <bool kTwo, typename TB, Source kB, typename TB2, Source kB2>
  hipError_t dw(const void* X, const Operand<TA, TB, kB>& B, const void* X2, const Operand<TA, TB2, kB2>& B2, void* dW, void* db,
                void* partial) const {
    const int64_t per = rows_per_range(c, n), ranges = range_count(c, n), stride = range_stride(c);
    const int64_t n_dw = static_cast<int64_t>(c->k_in) * c->k_out;
    TA* part = static_cast<TA*>(partial);
    TA* to_dw = ranges == 1 ? static_cast<TA*>(dW) : part;
    TA* to_db = ranges == 1 ? static_cast<TA*>(db) : part + n_dw;
    const int64_t tiles = (dW ? tiles_of(c->k_in) : 1) * tiles_of(c->k_out);
    hipLaunchKernelGGL((dw_kernel<TA, TS, TB, kB, TB2, kB2, kTwo>), dim3(static_cast<unsigned>(tiles * ranges)), dim3(kThreads), 0, stream, n,
                       per, dW ? c->k_in : std::min(c->k_in, kTile), c->k_out, dW != nullptr, db != nullptr, matrix<TS>(X, ld_in(c)), B,
                       matrix<TS>(X2, ld_in(c)), B2, to_dw, to_db, stride);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || ranges == 1) return e;
    return sum_ranges(part, ranges, dW, db);
  }

  hipError_t sum_ranges(const TA* part, int64_t ranges, void* dW, void* db) const {
    const int64_t n_dw = static_cast<int64_t>(c->k_in) * c->k_out;
    hipLaunchKernelGGL((sum_ranges_kernel<TA>), dim3(grid_of(std::min<int64_t>((n_dw + c->k_out + kThreads - 1) / kThreads, 1 << 16))),
                       dim3(kThreads), 0, stream, part, ranges, range_stride(c), n_dw, static_cast<int64_t>(c->k_out),
                       static_cast<TA*>(dW), static_cast<TA*>(db));
    return hipGetLastError();
  }

  template <Source kSource>
  Operand<TA, TS, kSource> g(const void* dY, const void* Z) const {
    return {matrix<TS>(dY, ld_out(c)), matrix<TS>(Z, ld_out(c)), c->activation};
  }

  template <Source kSource>
  hipError_t backward_as(const void* X, const void* W, const void* Z, const void* dY, void* dX, void* dW, void* db, void* ws) const {
    const auto G = g<kSource>(dY, Z);
    if (dX) {
      const hipError_t e = dx(G, W, dX);
      if (e != hipSuccess) return e;
    }
    return dW || db ? dw<false>(X, G, X, G, dW, db, ws) : hipSuccess;
  }

  hipError_t backward(const void* X, const void* W, const void* Z, const void* dY, void* dX, void* dW, void* db, void* ws) const {
    return c->activation == DL_NONE ? backward_as<kPlain>(X, W, Z, dY, dX, dW, db, ws) : backward_as<kGated>(X, W, Z, dY, dX, dW, db, ws);
  }

  hipError_t zero_rows(void* p, int cols, int64_t ld) const {
    if (!p) return hipSuccess;
    hipLaunchKernelGGL((zero_rows_kernel<TS>), dim3(grid_of(std::min<int64_t>((n * cols + kThreads - 1) / kThreads, 2048))), dim3(kThreads),
                       0, stream, n, cols, ld, static_cast<TS*>(p));
    return hipGetLastError();
  }

  hipError_t double_backward(const void* X, const void* W, const void* Z, const void* dY, const void* HX, void* ddY, void* X2, void* W2,
                             void* b2, void* ws) const {
    const bool curved = s_bytes(c, n) != 0;
    TA* S = curved ? static_cast<TA*>(ws) : nullptr;
    void* part = static_cast<char*>(ws) + s_bytes(c, n);
    const TileWalk walk{tiles_of(n), tiles_of(c->k_out)};
    hipLaunchKernelGGL((v_kernel<TS, TA>), dim3(grid_of(walk.count())), dim3(kThreads), 0, stream, walk, n, c->k_in, c->k_out, ld_out(c),
                       c->activation, matrix<TS>(HX, ld_in(c)), matrix<TA>(W, c->k_out),
                       c->activation == DL_NONE ? nullptr : static_cast<const TS*>(Z), static_cast<const TS*>(dY), static_cast<TS*>(ddY), S);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (!curved) {   // act'' = 0: W2 is dW of HX, X2 and b2 are zero
      e = zero_rows(X2, c->k_in, ld_in(c));
      if (e != hipSuccess) return e;
      if (b2) {
        e = sum_ranges(nullptr, 0, nullptr, b2);
        if (e != hipSuccess) return e;
      }
      if (!W2) return hipSuccess;
      if (c->activation == DL_NONE) return dw<false>(HX, g<kPlain>(dY, Z), HX, g<kPlain>(dY, Z), W2, nullptr, part);
      return dw<false>(HX, g<kGated>(dY, Z), HX, g<kGated>(dY, Z), W2, nullptr, part);
    }
    const Operand<TA, TA, kPlain> s{matrix<TA>(S, c->k_out), matrix<TA>(S, c->k_out), 0};
    if (X2) {
      e = dx(s, W, X2);
      if (e != hipSuccess) return e;
    }
    return W2 || b2 ? dw<true>(X, s, HX, g<kGated>(dY, Z), W2, b2, part) : hipSuccess;
  }
};

template <typename F>
hipError_t by_type(const dl_config* c, int64_t n, hipStream_t stream, F&& f) {
  switch (c->dtype) {
    case SC_F64: return f(Calls<double, double>{c, n, stream});
    case SC_BF16: return f(Calls<__bf16, float>{c, n, stream});
    default: return f(Calls<float, float>{c, n, stream});
  }
}

sc_status check_tensors(const char* fn, std::initializer_list<const void*> needed, std::initializer_list<const void*> optional) {
  for (const void* p : needed)
    if (!p) return set_error(SC_ERR_INVALID_ARG, std::string(fn) + ": NULL tensor argument");
  for (auto list : {needed, optional})
    for (const void* p : list)
      if (misaligned(p, 16)) return set_error(SC_ERR_INVALID_ARG, std::string(fn) + ": tensor pointer not 16-byte aligned");
  return SC_OK;
}

sc_status check_workspace(const char* fn, const dl_config* cfg, int64_t n, const void* workspace, size_t given) {
  if (!workspace || given < workspace_bytes(cfg, n))
    return set_error(SC_ERR_WORKSPACE, std::string(fn) + ": workspace missing or smaller than dl_workspace_bytes()");
  if (misaligned(workspace, 256)) return set_error(SC_ERR_WORKSPACE, std::string(fn) + ": workspace not 256-byte aligned");
  return SC_OK;
}

sc_status launched(const char* fn, hipError_t e) {
  return e == hipSuccess ? SC_OK : set_error(SC_ERR_HIP, std::string(fn) + ": kernel launch: " + hipGetErrorString(e));
}

}  // namespace
}  // namespace dl

extern "C" {

sc_status dl_forward(const dl_config* cfg, int64_t n_rows, const void* X, const void* W, const void* b, const void* residual, void* Y,
                     void* Z, void* hip_stream) {
  using namespace dl;
  sc_status st = check_config("dl_forward", cfg, n_rows);
  if (st != SC_OK || n_rows == 0) return st;
  st = check_tensors("dl_forward", {X, W, Y}, {b, residual, Z});
  if (st != SC_OK) return st;
  DeviceGuard guard(cfg->device);
  if (!guard.ok) return set_error(SC_ERR_HIP, "dl_forward: cannot make cfg->device current");
  return launched("dl_forward", by_type(cfg, n_rows, static_cast<hipStream_t>(hip_stream),
                                        [&](const auto& calls) { return calls.forward(X, W, b, residual, Y, Z); }));
}

sc_status dl_workspace_bytes(const dl_config* cfg, int64_t n_rows, size_t* bytes) {
  using namespace dl;
  const sc_status st = check_config("dl_workspace_bytes", cfg, n_rows);
  if (st != SC_OK) return st;
  if (!bytes) return set_error(SC_ERR_INVALID_ARG, "dl_workspace_bytes: bytes is NULL");
  *bytes = workspace_bytes(cfg, n_rows);
  return SC_OK;
}

sc_status dl_backward(const dl_config* cfg, int64_t n_rows, const void* X, const void* W, const void* Z, const void* dY, void* dX, void* dW,
                      void* db, void* workspace, size_t workspace_bytes_given, void* hip_stream) {
  using namespace dl;
  sc_status st = check_config("dl_backward", cfg, n_rows);
  if (st != SC_OK) return st;
  if (!dX && !dW && !db) return set_error(SC_ERR_INVALID_ARG, "dl_backward: dX, dW and db are all NULL");
  st = check_tensors("dl_backward", {}, {X, W, Z, dY, dX, dW, db});
  if (st != SC_OK) return st;
  if (n_rows > 0) {
    st = check_tensors("dl_backward", {X, W, dY}, {});
    if (st == SC_OK && cfg->activation != DL_NONE) st = check_tensors("dl_backward", {Z}, {});
    if (st == SC_OK) st = check_workspace("dl_backward", cfg, n_rows, workspace, workspace_bytes_given);
    if (st != SC_OK) return st;
  }
  DeviceGuard guard(cfg->device);
  if (!guard.ok) return set_error(SC_ERR_HIP, "dl_backward: cannot make cfg->device current");
  return launched("dl_backward", by_type(cfg, n_rows, static_cast<hipStream_t>(hip_stream), [&](const auto& calls) {
                    if (n_rows == 0) return dW || db ? calls.sum_ranges(nullptr, 0, dW, db) : hipSuccess;
                    return calls.backward(X, W, Z, dY, dX, dW, db, workspace);
                  }));
}

sc_status dl_double_backward(const dl_config* cfg, int64_t n_rows, const void* X, const void* W, const void* Z, const void* dY,
                             const void* HX, void* ddY, void* X2, void* W2, void* b2, void* workspace, size_t workspace_bytes_given,
                             void* hip_stream) {
  using namespace dl;
  sc_status st = check_config("dl_double_backward", cfg, n_rows);
  if (st != SC_OK) return st;
  st = check_tensors("dl_double_backward", {}, {X, W, Z, dY, HX, ddY, X2, W2, b2});
  if (st != SC_OK) return st;
  if (n_rows > 0) {
    st = check_tensors("dl_double_backward", {X, W, dY, HX, ddY}, {});
    if (st == SC_OK && cfg->activation != DL_NONE) st = check_tensors("dl_double_backward", {Z}, {});
    if (st == SC_OK) st = check_workspace("dl_double_backward", cfg, n_rows, workspace, workspace_bytes_given);
    if (st != SC_OK) return st;
  }
  DeviceGuard guard(cfg->device);
  if (!guard.ok) return set_error(SC_ERR_HIP, "dl_double_backward: cannot make cfg->device current");
  return launched("dl_double_backward", by_type(cfg, n_rows, static_cast<hipStream_t>(hip_stream), [&](const auto& calls) {
                    if (n_rows == 0) return W2 || b2 ? calls.sum_ranges(nullptr, 0, W2, b2) : hipSuccess;
                    return calls.double_backward(X, W, Z, dY, HX, ddY, X2, W2, b2, workspace);
                  }));
}

}  // extern "C"
