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
#include <initializer_list>
#include <string>
#include <type_traits>

#include "dl_product.h"

namespace dl {
namespace {

using sc::align_up;
using sc::DeviceGuard;
using sc::misaligned;
using sc::set_error;

constexpr int kXcds = 8;

// Waves that share one result where rows are few (the registers of an fp64 wave leave room for four).
template <typename TA>
__host__ __device__ constexpr int split_waves() { return sizeof(TA) == 8 ? 4 : 8; }
template <bool kSplit, typename TA>
constexpr int threads() { return kSplit ? split_waves<TA>() * kLanes : kThreads; }
// LDS of a product of rows: the waves' corners, or their results where they share one.
template <bool kSplit, int kRT, typename TA>
constexpr int lds_elements() { return kSplit ? split_waves<TA>() * 16 * kLanes : kWaves * kRT * Corner<TA>::kBlock; }

// How a workgroup's waves stand: wc side by side along the columns, the others along the rows.
struct Shape {
  int wc, wr;
};

// Row groups x column groups of workgroups.  All column groups of a row group go to one XCD (workgroups are dealt out to the XCDs in turn), whose
// L2 then holds the rows that they share.
struct Walk {
  int64_t row_groups;
  int col_groups;
  __host__ __device__ int64_t count() const { return (row_groups + kXcds - 1) / kXcds * kXcds * col_groups; }
  __device__ bool at(int64_t t, int64_t* row, int* col) const {
    const int64_t local = t / kXcds;
    *row = local / col_groups * kXcds + t % kXcds;
    *col = static_cast<int>(local % col_groups);
    return *row < row_groups;
  }
};

// The results of 16 kRT rows and 64 columns, by this wave alone or (kSplit) by all waves of the workgroup, each over its part of the reduced
// index, joined in LDS in the order of the waves.  f as in each_four.
template <typename TA, int kRT, bool kSplit, bool kFours, typename Rows, typename Weights, typename T, int N, typename F>
__device__ __forceinline__ void finish_rows(const Rows& a, const Weights& w, int64_t row0, int64_t rows, int n0, TA* lds,
                                            const TA* __restrict__ bias, const Beside<T, N>& beside, F&& f) {
  typename Mma<TA>::acc_t acc[kRT][4];
  const int lane = threadIdx.x & (kLanes - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kLanes);
  TA* const corner = lds + wave * (kRT * Corner<TA>::kBlock);
  if constexpr (!kSplit) {
    rows_product<TA, kRT, kFours>(a, w, row0, rows, n0, 0, w.k_end, corner, acc);
    each_four<TA, kRT, kFours>(row0, rows, n0, w.n_end, acc, bias, beside, f);
  } else {
    static_assert(kRT == 1, "one row tile");
    constexpr int kN = split_waves<TA>();
    const int per = ((w.k_end + kN - 1) / kN + kDepth - 1) / kDepth * kDepth;
    const int from = min(w.k_end, wave * per), to = min(w.k_end, from + per);
    if (from < to) {
      rows_product<TA, 1, kFours>(a, w, row0, rows, n0, from, to, corner, acc);
    } else {
#pragma unroll
      for (int u = 0; u < 4; ++u) acc[0][u] = typename Mma<TA>::acc_t{0, 0, 0, 0};
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int u = 0; u < 4; ++u) lds[((wave * 4 + r) * 4 + u) * kLanes + lane] = acc[0][u][r];
    __syncthreads();
    const int64_t row = row0 + Mma<TA>::row(lane, wave & 3);   // wave w < 4 finishes the lanes' result r = w
    const int c = n0 + 4 * (lane & 15);
    if (wave < 4 && row < rows && c < w.n_end) {
      TA x[N > 0 ? N : 1][4], v[4] = {0, 0, 0, 0}, sum[4] = {0, 0, 0, 0};
      if (bias) load4<kFours>(bias, c, w.n_end, v);
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (beside.m[e].p) load4<kFours>(beside.m[e].p + row * beside.m[e].ld, c, w.n_end, x[e]);
      for (int p = 0; p < kN; ++p)
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[i] += lds[((p * 4 + wave) * 4 + i) * kLanes + lane];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] += sum[i];
      f(row, c, v, x);
    }
    __syncthreads();
  }
}

// Calls f(first row, first column) for the tiles of this wave (kSplit: of the workgroup).
template <int kRT, bool kSplit, typename F>
__device__ __forceinline__ void each_tile(const Walk& walk, const Shape& shape, int64_t rows, int n_end, F&& f) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kLanes);
  for (int64_t t = blockIdx.x; t < walk.count(); t += gridDim.x) {
    int64_t rg;
    int cg;
    if (!walk.at(t, &rg, &cg)) continue;
    const int64_t row0 = kSplit ? rg * 16 : (rg * shape.wr + wave / shape.wc) * (16 * kRT);
    const int n0 = (kSplit ? cg : cg * shape.wc + wave % shape.wc) * kCols;
    if (row0 < rows && n0 < n_end) f(row0, n0);
  }
}

template <typename TS, typename TA, int kRT, bool kSplit, bool kFours>
__global__ __launch_bounds__((threads<kSplit, TA>())) void forward_kernel(Walk walk, Shape shape, int64_t rows, Gate<TA> gate, int64_t ld_out,
                                                                    Operand<TA, TS, kPlain> X, AlongRows<TA> W, const TA* __restrict__ bias,
                                                                    const TS* __restrict__ residual, TS* __restrict__ Y,
                                                                    TS* __restrict__ Z) {
  __shared__ TA lds[lds_elements<kSplit, kRT, TA>()];
  const int n_end = W.n_end;
  const Beside<TS, 1> beside{{{residual, ld_out}}};
  each_tile<kRT, kSplit>(walk, shape, rows, n_end, [&](int64_t row0, int n0) {
    finish_rows<TA, kRT, kSplit, kFours>(X, W, row0, rows, n0, lds, bias, beside, [&](int64_t row, int c, const TA (&z)[4], const TA (&x)[1][4]) {
      const int64_t at = row * ld_out;
      TA y[4];
      if (Z) store4<kFours>(Z + at, c, n_end, z);
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = z[i];
      if (gate.on) {
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = gate.value(z[i]);
      }
      if (residual) {
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] += x[0][i];
      }
      store4<kFours>(Y + at, c, n_end, y);
    });
  });
}

// V = HX W, ddY = V act'(Z), S = V dY act''(Z).  Z NULL: no activation; S NULL: no curvature.
template <typename TS, typename TA, int kRT, bool kSplit, bool kFours>
__global__ __launch_bounds__((threads<kSplit, TA>())) void v_kernel(Walk walk, Shape shape, int64_t rows, Gate<TA> gate, int64_t ld_out,
                                                              Operand<TA, TS, kPlain> HX, AlongRows<TA> W, const TS* __restrict__ Z,
                                                              const TS* __restrict__ dY, TS* __restrict__ ddY, TA* __restrict__ S) {
  __shared__ TA lds[lds_elements<kSplit, kRT, TA>()];
  const int n_end = W.n_end;
  const Beside<TS, 2> beside{{{Z, ld_out}, {S ? dY : nullptr, ld_out}}};
  each_tile<kRT, kSplit>(walk, shape, rows, n_end, [&](int64_t row0, int n0) {
    const TA* const none = nullptr;
    finish_rows<TA, kRT, kSplit, kFours>(HX, W, row0, rows, n0, lds, none, beside, [&](int64_t row, int c, const TA (&v)[4], const TA (&x)[2][4]) {
      TA out[4], s[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        TA first = TA(1), second = TA(0);
        if (Z) gate.both(x[0][i], &first, &second);
        out[i] = v[i] * first;
        s[i] = v[i] * x[1][i] * second;
      }
      if (S) store4<kFours>(S + row * n_end, c, n_end, s);
      store4<kFours>(ddY + row * ld_out, c, n_end, out);
    });
  });
}

// What a launch of the backward does: the rows in chunks, of each chunk first dx_groups workgroups of dX, then dw_groups of the chunk's partial dW and
// db.  A chunk stays on one XCD and its two halves run at about the same time: the second reading of dY (and Z) comes from the caches.
struct Plan {
  int64_t rows, per;    // per: rows of a chunk, a multiple of 64
  int64_t chunks;
  int64_t dx_groups, dw_groups;   // workgroups of a chunk
  int dx_col_groups, dw_col_groups;
  Shape dx, dw;
  int64_t stride;       // elements between the chunks' partial results
};

template <typename TA, int kRT, bool kSplit, bool kFours, typename TS, typename G, typename Weights>
__device__ __forceinline__ void dx_role(const Plan& p, int64_t chunk, int64_t i, const G& g, const Weights& W, int64_t ld_in,
                                        TS* __restrict__ dX, TA* lds) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kLanes);
  const int64_t end = min(p.rows, (chunk + 1) * p.per);
  const int64_t rg = i / p.dx_col_groups;
  const int cg = static_cast<int>(i % p.dx_col_groups);
  const int64_t row0 = chunk * p.per + (kSplit ? rg * 16 : (rg * p.dx.wr + wave / p.dx.wc) * (16 * kRT));
  const int n0 = (kSplit ? cg : cg * p.dx.wc + wave % p.dx.wc) * kCols;
  if (row0 >= end || n0 >= W.n_end) return;   // for kSplit the same in all waves
  const TA* const none = nullptr;
  finish_rows<TA, kRT, kSplit, kFours>(g, W, row0, end, n0, lds, none, Beside<TS, 0>{}, [&](int64_t row, int c, const TA (&v)[4], const TA (&)[1][4]) {
    store4<kFours>(dX + row * ld_in, c, W.n_end, v);
  });
}

// Partial dW of one 64 x 64 wc block: the chunk's rows are shared by dw.wr waves, joined in LDS in order.
template <typename TA, bool kTwo, bool kFours, typename X, typename B, typename B2>
__device__ __forceinline__ void dw_role(const Plan& p, int64_t chunk, int i, int k_in, int k_out, const X& x, const B& b, const X& x2,
                                        const B2& b2, TA* __restrict__ dW, TA* __restrict__ db, TA* lds) {
  const int lane = threadIdx.x & (kLanes - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kLanes);
  const int q = lane / 16, j = lane & 15;
  const int wc = wave % p.dw.wc, wr = wave / p.dw.wc;
  const int m0 = i / p.dw_col_groups * kCols, n0 = (i % p.dw_col_groups * p.dw.wc + wc) * kCols;
  const int64_t begin = chunk * p.per, end = min(p.rows, begin + p.per);
  const int64_t share = (p.per / p.dw.wr + 15) / 16 * 16;
  const int64_t from = min(end, begin + wr * share), to = min(end, from + share);
  typename Mma<TA>::acc_t acc[4][4];
#pragma unroll
  for (int t = 0; t < 4; ++t)
#pragma unroll
    for (int u = 0; u < 4; ++u) acc[t][u] = typename Mma<TA>::acc_t{0, 0, 0, 0};
  TA sum[4] = {0, 0, 0, 0}, none[4];
  if (n0 < k_out) {
    outer_product<TA, kFours>(x, b, m0, k_in, n0, k_out, from, to, acc, sum);
    if constexpr (kTwo) outer_product<TA, kFours>(x2, b2, m0, k_in, n0, k_out, from, to, acc, none);
  }
  TA* const to_dw = dW ? dW + chunk * p.stride : nullptr;
  TA* const to_db = db && m0 == 0 ? db + chunk * p.stride : nullptr;
  // column sums: over the four q of the wave, then over the waves
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    sum[u] += __shfl_xor(sum[u], 16);
    sum[u] += __shfl_xor(sum[u], 32);
  }
  const int n = n0 + 4 * j;
  if (p.dw.wr == 1) {
    if (n0 >= k_out) return;
    if (to_db && q == 0) store4<kFours>(to_db, n, k_out, sum);
    if (to_dw) {
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int m = m0 + 4 * Mma<TA>::row(lane, r) + t;
          const TA v[4] = {acc[t][0][r], acc[t][1][r], acc[t][2][r], acc[t][3][r]};
          if (m < k_in && n < k_out) store4<kFours>(to_dw + static_cast<int64_t>(m) * k_out, n, k_out, v);
        }
    }
    return;
  }
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    __syncthreads();
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int u = 0; u < 4; ++u) lds[((wave * 4 + r) * 4 + u) * kLanes + lane] = acc[t][u][r];
    __syncthreads();
    if (to_dw && n < k_out) {
      for (int r = wr; r < 4; r += p.dw.wr) {
        const int m = m0 + 4 * Mma<TA>::row(lane, r) + t;
        TA v[4] = {0, 0, 0, 0};
        for (int w = 0; w < p.dw.wr; ++w)
#pragma unroll
          for (int u = 0; u < 4; ++u) v[u] += lds[(((w * p.dw.wc + wc) * 4 + r) * 4 + u) * kLanes + lane];
        if (m < k_in) store4<kFours>(to_dw + static_cast<int64_t>(m) * k_out, n, k_out, v);
      }
    }
  }
  if (to_db) {
    __syncthreads();
    if (q == 0) {
#pragma unroll
      for (int u = 0; u < 4; ++u) lds[(wave * 4 + u) * 16 + j] = sum[u];
    }
    __syncthreads();
    if (wr == 0 && q == 0 && n < k_out) {
      TA v[4] = {0, 0, 0, 0};
      for (int w = 0; w < p.dw.wr; ++w)
#pragma unroll
        for (int u = 0; u < 4; ++u) v[u] += lds[((w * p.dw.wc + wc) * 4 + u) * 16 + j];
      store4<kFours>(to_db, n, k_out, v);
    }
  }
}

// G: the source of dX.  B, B2: those of dW (kTwo: the second-order pass, x2 B2 added to x B; the column sums are those of B).
template <typename TS, typename TA, int kRT, bool kSplit, bool kFours, bool kTwo, typename G, typename B, typename B2, typename Weights>
__global__ __launch_bounds__((threads<kSplit, TA>())) void backward_kernel(Plan p, int k_in, int k_out, int64_t ld_in, G g, Weights W,
                                                                     TS* __restrict__ dX, Operand<TA, TS, kPlain> x, B b,
                                                                     Operand<TA, TS, kPlain> x2, B2 b2, TA* __restrict__ dW,
                                                                     TA* __restrict__ db) {
  constexpr int kJoin = threads<kSplit, TA>() * 16, kRowsPart = lds_elements<kSplit, kRT, TA>();
  __shared__ TA lds[kJoin > kRowsPart ? kJoin : kRowsPart];
  const int64_t groups = p.dx_groups + p.dw_groups, total = (p.chunks + kXcds - 1) / kXcds * kXcds * groups;
  for (int64_t t = blockIdx.x; t < total; t += gridDim.x) {
    const int64_t local = t / kXcds, chunk = local / groups * kXcds + t % kXcds, i = local % groups;
    if (chunk >= p.chunks) continue;
    if (i < p.dx_groups)
      dx_role<TA, kRT, kSplit, kFours>(p, chunk, i, g, W, ld_in, dX, lds);
    else
      dw_role<TA, kTwo, kFours>(p, chunk, static_cast<int>(i - p.dx_groups), k_in, k_out, x, b, x2, b2, dW, db, lds);
    __syncthreads();   // LDS is the next tile's
  }
}

// out[i] = sum over the chunks of part[chunk][i], each of 16 groups of lanes over a stretch of the chunks, joined in order: [0, n_dw) to
// dW, the rest to db.  No chunk at all: zeros.
template <typename TA>
__global__ __launch_bounds__(kThreads) void sum_chunks_kernel(const TA* __restrict__ part, int64_t chunks, int64_t stride, int64_t n_dw,
                                                              int64_t n_db, TA* __restrict__ dW, TA* __restrict__ db) {
  constexpr int kGroups = 16, kAhead = 8;
  __shared__ TA lds[kGroups][64];
  const int group = threadIdx.x / 16, four = threadIdx.x % 16;
  const int64_t per = (chunks + kGroups - 1) / kGroups, from = min(chunks, group * per), to = min(chunks, from + per);
  const int64_t all = n_dw + n_db;
  for (int64_t i0 = blockIdx.x * static_cast<int64_t>(64); i0 < all; i0 += static_cast<int64_t>(gridDim.x) * 64) {
    const int64_t i = i0 + 4 * four;
    const int cols = static_cast<int>(min(static_cast<int64_t>(64), all - i0));
    TA s[4] = {0, 0, 0, 0};
    if (i < all) {
      for (int64_t c = from; c < to; c += kAhead) {
        TA v[kAhead][4];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) load4<false>(part + min(c + k, to - 1) * stride + i0, 4 * four, cols, v[k]);
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
          if (c + k < to)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[e] += v[k][e];
      }
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 4; ++e) lds[group][4 * four + e] = s[e];
    __syncthreads();
    if (threadIdx.x < 64 && i0 + threadIdx.x < all) {
      TA v = 0;
      for (int k = 0; k < kGroups; ++k) v += lds[k][threadIdx.x];
      const int64_t at = i0 + threadIdx.x;
      if (at < n_dw) {
        if (dW) dW[at] = v;
      } else if (db) {
        db[at - n_dw] = v;
      }
    }
  }
}

// WT [k_out][k_in] = W transposed, 32 x 32 elements at a time through LDS.
template <typename TA>
__global__ __launch_bounds__(kThreads) void transpose_kernel(int k_in, int k_out, const TA* __restrict__ W, TA* __restrict__ WT) {
  __shared__ TA tile[32][33];
  const int across = (k_out + 31) / 32, r0 = blockIdx.x / across * 32, c0 = blockIdx.x % across * 32;
  const int x = threadIdx.x % 32, y = threadIdx.x / 32;
#pragma unroll
  for (int i = 0; i < 32; i += kThreads / 32)
    if (r0 + y + i < k_in && c0 + x < k_out) tile[y + i][x] = W[static_cast<int64_t>(r0 + y + i) * k_out + c0 + x];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 32; i += kThreads / 32)
    if (c0 + y + i < k_out && r0 + x < k_in) WT[static_cast<int64_t>(c0 + y + i) * k_in + r0 + x] = tile[x][y + i];
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

int64_t blocks_of(int64_t n, int64_t size) { return (n + size - 1) / size; }

// Waves side by side along the columns: as many as there are column blocks, up to four.
Shape shape_of(int cols) {
  const int64_t blocks = blocks_of(cols, kCols);
  return blocks >= 3 ? Shape{4, 1} : blocks == 2 ? Shape{2, 2} : Shape{1, 4};
}

// Row tiles of a wave: the fewer the rows the fewer, so that there are two waves for every SIMD of 256 CUs as long as possible.
int row_tiles(int64_t rows, int cols, int most) {
  const int64_t waves = blocks_of(rows, 16) * blocks_of(cols, kCols);
  int rt = 1;
  while (rt < most && waves / (2 * rt) >= 2048) rt *= 2;
  return rt;
}

// Do all waves of a workgroup share one tile?  Where there is at most one row tile for every two SIMDs and the sum is long.
bool split_sum(int64_t rows, int cols, int k) { return k >= 128 && blocks_of(rows, 16) * blocks_of(cols, kCols) <= 512; }

Plan plan_of(const dl_config* c, int64_t n, bool want_dx, bool want_dw, bool split, int rt) {
  const int split_waves = c->dtype == SC_F64 ? dl::split_waves<double>() : dl::split_waves<float>();
  Plan p{};
  p.rows = n;
  p.dw = shape_of(c->k_out);
  if (split) p.dw = {1, split_waves};
  const int64_t blocks = blocks_of(c->k_in, kCols) * blocks_of(c->k_out, kCols);
  // about 2048 waves of dW, none with less than 64 rows
  const int64_t chunks = std::max<int64_t>(1, std::min(2048 / (blocks * p.dw.wr), n / (64 * p.dw.wr)));
  p.per = blocks_of(n, chunks);
  p.per = blocks_of(p.per, p.per < 256 ? 64 : 256) * (p.per < 256 ? 64 : 256);
  p.chunks = blocks_of(n, p.per);
  p.dx = split ? Shape{1, 1} : shape_of(c->k_in);
  p.dx_col_groups = static_cast<int>(blocks_of(c->k_in, kCols * p.dx.wc));
  p.dx_groups = want_dx ? blocks_of(p.per, split ? 16 : 16 * rt * p.dx.wr) * p.dx_col_groups : 0;
  p.dw_col_groups = static_cast<int>(blocks_of(c->k_out, kCols * p.dw.wc));
  p.dw_groups = want_dw ? blocks_of(c->k_in, kCols) * p.dw_col_groups : 0;
  p.stride = static_cast<int64_t>(c->k_in) * c->k_out + c->k_out;
  return p;
}

bool curved(const dl_config* c) { return c->activation == DL_SILU || c->activation == DL_GELU; }

// Does dX take W transposed (a launch of its own, 2 us)?  Where the reading of W as it is, four times the accesses, would take longer.
bool transposed(int64_t n, const dl_config* c, bool split) { return !split && n >= 4096; }

size_t wt_bytes(int64_t n, const dl_config* c) {
  return transposed(n, c, false) ? align_up(static_cast<size_t>(c->k_in) * c->k_out * weight_size(c), 256) : 0;
}

// Workspace: [ S of the second-order pass ][ W transposed ][ partial dW and db per chunk ].
size_t s_bytes(const dl_config* c, int64_t n) { return curved(c) ? align_up(static_cast<size_t>(n) * c->k_out * weight_size(c), 256) : 0; }

size_t workspace_bytes(const dl_config* c, int64_t n) {
  if (n == 0) return 256;
  size_t part = 0;
  for (bool split : {false, true}) {
    const Plan p = plan_of(c, n, true, true, split, 1);
    part = std::max(part, static_cast<size_t>(p.chunks) * p.stride * weight_size(c));
  }
  return s_bytes(c, n) + wt_bytes(n, c) + align_up(part, 256) + 256;
}

template <typename TS, typename TA>
struct Calls {
  const dl_config* c;
  int64_t n;
  hipStream_t stream;
  static constexpr int kMostTiles = sizeof(TA) == 8 ? 2 : 4;

  template <typename T>
  static Matrix<T> matrix(const void* p, int64_t ld) {
    return {static_cast<const T*>(p), ld};
  }
  Operand<TA, TS, kPlain> rows_in(const void* X) const { return {matrix<TS>(X, ld_in(c)), {}, {}}; }
  template <Source kSource>
  Operand<TA, TS, kSource> g(const void* dY, const void* Z) const {
    return {matrix<TS>(dY, ld_out(c)), matrix<TS>(Z, ld_out(c)), Gate<TA>::of(c->activation)};
  }

  // Launches a product of rows with W [k_in][k_out]: launch(row tiles, split, fours) with all three known at compile time.  Widths that are no
  // multiple of four test every element and are bound by that: one row tile does for them.
  template <typename F>
  hipError_t by_shape(int cols, int k, F&& launch) const {
    const std::integral_constant<int, 1> one{};
    const std::true_type yes{};
    const std::false_type no{};
    const bool fours = c->k_in % 4 == 0 && c->k_out % 4 == 0, split = split_sum(n, cols, k);
    if (!fours) return split ? launch(one, yes, no) : launch(one, no, no);
    if (split) return launch(one, yes, yes);
    const int rt = row_tiles(n, cols, kMostTiles);
    if constexpr (kMostTiles == 4) {
      if (rt == 4) return launch(std::integral_constant<int, 4>{}, no, yes);
    }
    if (rt >= 2) return launch(std::integral_constant<int, 2>{}, no, yes);
    return launch(one, no, yes);
  }

  Walk walk_of(int rt, bool split, const Shape& shape) const {
    if (split) return {blocks_of(n, 16), static_cast<int>(blocks_of(c->k_out, kCols))};
    return {blocks_of(n, 16 * rt * shape.wr), static_cast<int>(blocks_of(c->k_out, kCols * shape.wc))};
  }
  static unsigned grid_of(int64_t groups) { return static_cast<unsigned>(std::min<int64_t>(groups, 1 << 22)); }

  hipError_t forward(const void* X, const void* W, const void* b, const void* residual, void* Y, void* Z) const {
    return by_shape(c->k_out, c->k_in, [&](auto rt, auto split, auto fours) {
      const Shape shape = shape_of(c->k_out);
      const Walk walk = walk_of(rt, split, shape);
      hipLaunchKernelGGL((forward_kernel<TS, TA, rt.value, split.value, fours.value>), dim3(grid_of(walk.count())), dim3((threads<split.value, TA>())), 0, stream,
                         walk, shape, n, Gate<TA>::of(c->activation), ld_out(c), rows_in(X),
                         (AlongRows<TA>{static_cast<const TA*>(W), c->k_in, c->k_out}), static_cast<const TA*>(b),
                         static_cast<const TS*>(residual), static_cast<TS*>(Y), static_cast<TS*>(Z));
      return hipGetLastError();
    });
  }

  hipError_t v(const void* HX, const void* W, const void* Z, const void* dY, void* ddY, TA* S) const {
    return by_shape(c->k_out, c->k_in, [&](auto rt, auto split, auto fours) {
      const Shape shape = shape_of(c->k_out);
      const Walk walk = walk_of(rt, split, shape);
      hipLaunchKernelGGL((v_kernel<TS, TA, rt.value, split.value, fours.value>), dim3(grid_of(walk.count())), dim3((threads<split.value, TA>())), 0, stream, walk,
                         shape, n, Gate<TA>::of(c->activation), ld_out(c), rows_in(HX), (AlongRows<TA>{static_cast<const TA*>(W), c->k_in, c->k_out}),
                         c->activation == DL_NONE ? nullptr : static_cast<const TS*>(Z), static_cast<const TS*>(dY),
                         static_cast<TS*>(ddY), S);
      return hipGetLastError();
    });
  }

  // ws: [ W transposed ][ partial results ].
  template <bool kTwo, typename G, typename B, typename B2>
  hipError_t gradients(const G& source, const void* W, void* dX, const void* X, const B& b, const void* X2, const B2& b2, void* dW,
                       void* db, void* ws) const {
    return by_shape(c->k_in, c->k_out, [&](auto rt, auto split, auto fours) {
      const AlongColumns<TA> as_is{static_cast<const TA*>(W), c->k_out, c->k_in};
      if constexpr (!split.value && fours.value) {
        if (dX && transposed(n, c, split)) {
          const int64_t tiles = blocks_of(c->k_in, 32) * blocks_of(c->k_out, 32);
          hipLaunchKernelGGL((transpose_kernel<TA>), dim3(static_cast<unsigned>(tiles)), dim3(kThreads), 0, stream, c->k_in, c->k_out,
                             static_cast<const TA*>(W), static_cast<TA*>(ws));
          const hipError_t e = hipGetLastError();
          if (e != hipSuccess) return e;
          return gradients_with<kTwo>(rt, split, fours, source, AlongRows<TA>{static_cast<const TA*>(ws), c->k_out, c->k_in}, dX, X, b, X2,
                                      b2, dW, db, ws);
        }
      }
      return gradients_with<kTwo>(rt, split, fours, source, as_is, dX, X, b, X2, b2, dW, db, ws);
    });
  }

  template <bool kTwo, typename RT, typename Split, typename Fours, typename G, typename Weights, typename B, typename B2>
  hipError_t gradients_with(RT rt, Split split, Fours fours, const G& source, const Weights& w, void* dX, const void* X, const B& b,
                            const void* X2, const B2& b2, void* dW, void* db, void* ws) const {
    const Plan p = plan_of(c, n, dX != nullptr, dW || db, split, rt);
    const bool whole = p.chunks == 1;
    TA* part = reinterpret_cast<TA*>(static_cast<char*>(ws) + wt_bytes(n, c));
    const int64_t n_dw = static_cast<int64_t>(c->k_in) * c->k_out;
    TA* to_dw = !dW ? nullptr : whole ? static_cast<TA*>(dW) : part;
    TA* to_db = !db ? nullptr : whole ? static_cast<TA*>(db) : part + n_dw;
    const int64_t groups = blocks_of(p.chunks, kXcds) * kXcds * (p.dx_groups + p.dw_groups);
    hipLaunchKernelGGL((backward_kernel<TS, TA, RT::value, Split::value, Fours::value, kTwo, G, B, B2, Weights>), dim3(grid_of(groups)),
                       dim3((threads<Split::value, TA>())), 0, stream, p, c->k_in, c->k_out, ld_in(c), source, w, static_cast<TS*>(dX),
                       rows_in(X), b, rows_in(X2), b2, to_dw, to_db);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || whole || !(dW || db)) return e;
    return sum_chunks(part, p.chunks, dW, db);
  }

  hipError_t sum_chunks(const TA* part, int64_t chunks, void* dW, void* db) const {
    const int64_t n_dw = static_cast<int64_t>(c->k_in) * c->k_out;
    hipLaunchKernelGGL((sum_chunks_kernel<TA>), dim3(static_cast<unsigned>(std::min<int64_t>(blocks_of(n_dw + c->k_out, 64), 1 << 16))),
                       dim3(kThreads), 0, stream, part, chunks, n_dw + c->k_out, n_dw, static_cast<int64_t>(c->k_out),
                       static_cast<TA*>(dW), static_cast<TA*>(db));
    return hipGetLastError();
  }

  hipError_t backward(const void* X, const void* W, const void* Z, const void* dY, void* dX, void* dW, void* db, void* ws) const {
    if (c->activation == DL_NONE) return gradients<false>(g<kPlain>(dY, Z), W, dX, X, g<kPlain>(dY, Z), X, g<kPlain>(dY, Z), dW, db, ws);
    return gradients<false>(g<kGated>(dY, Z), W, dX, X, g<kGated>(dY, Z), X, g<kGated>(dY, Z), dW, db, ws);
  }

  hipError_t zero_rows(void* p, int cols, int64_t ld) const {
    if (!p) return hipSuccess;
    hipLaunchKernelGGL((zero_rows_kernel<TS>), dim3(grid_of(std::min<int64_t>(blocks_of(n * cols, kThreads), 2048))), dim3(kThreads), 0, stream,
                       n, cols, ld, static_cast<TS*>(p));
    return hipGetLastError();
  }

  hipError_t double_backward(const void* X, const void* W, const void* Z, const void* dY, const void* HX, void* ddY, void* X2, void* W2,
                             void* b2, void* ws) const {
    TA* S = curved(c) ? static_cast<TA*>(ws) : nullptr;
    void* part = static_cast<char*>(ws) + s_bytes(c, n);
    hipError_t e = v(HX, W, Z, dY, ddY, S);
    if (e != hipSuccess) return e;
    if (!S) {   // act'' = 0: W2 is dW of HX, X2 and b2 are zero
      e = zero_rows(X2, c->k_in, ld_in(c));
      if (e == hipSuccess && b2) e = sum_chunks(nullptr, 0, nullptr, b2);
      if (e != hipSuccess || !W2) return e;
      if (c->activation == DL_NONE)
        return gradients<false>(g<kPlain>(dY, Z), W, nullptr, HX, g<kPlain>(dY, Z), HX, g<kPlain>(dY, Z), W2, nullptr, part);
      return gradients<false>(g<kGated>(dY, Z), W, nullptr, HX, g<kGated>(dY, Z), HX, g<kGated>(dY, Z), W2, nullptr, part);
    }
    if (!X2 && !W2 && !b2) return hipSuccess;
    const Operand<TA, TA, kPlain> s{{S, c->k_out}, {}, {}};
    return gradients<true>(s, W, X2, X, s, HX, g<kGated>(dY, Z), W2, b2, part);
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
                    if (n_rows == 0) return dW || db ? calls.sum_chunks(nullptr, 0, dW, db) : hipSuccess;
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
                    if (n_rows == 0) return W2 || b2 ? calls.sum_chunks(nullptr, 0, W2, b2) : hipSuccess;
                    return calls.double_backward(X, W, Z, dY, HX, ddY, X2, W2, b2, workspace);
                  }));
}

}  // extern "C"
