// The dense layer of include/dl.h: products with bias, activation and residual, their gradients and the second-order pass.
//
// Every step is a product C[m][n] = sum_k A[m][k] B[k][n] whose operands are made while they are staged
// (G = dY act'(Z) exists in memory only where several column blocks of dX would each make it again) and whose result is finished where it stands
// in the accumulators:
//
//   forward   rows x k_out   A = X    B = W      epilogue + b, act, + residual -> Y, Z
//   dX        rows x k_in    A = G    B = W^T
//   dW, db    k_in x k_out   A = X^T  B = G      the rows cut into ranges, partial results summed by a second launch in order
//   V         rows x k_out   A = HX   B = W      epilogue V act'(Z) -> ddY, S = V dY act''(Z) -> workspace
//   X2        rows x k_in    A = S    B = W^T
//   W2, b2    k_in x k_out   A = X^T  B = S, then A = HX^T  B = G on the same accumulators
// Kernels and launches, instantiated for one type by each of dl_f32.hip, dl_f64.hip and dl_bf16.hip.
//
// Which kernel serves a product is a matter of its type and sizes (dl_plan.h):
//   rows_kernel, backward_kernel              the fp32 and fp64 instruction: fp64, small batches, widths that are no multiple of four.  Few rows and a long
//                                             sum: all waves of a workgroup share a tile, each a part of the sum.  Bound by the latency of the launch and of
//                                             a few dependent loads (380 rows, 8 -> 64: 4.9 us), fp64 also by act' (10 000 rows, 128 -> 16: 13 and 24 us).
//   kept_kernel                               sums of at most 64, many rows: W's parts in registers, the rows once through.  Bound by memory: 199 003 rows, 64 -> 64
//                                             fp32, forward 41 us and V 50 us at 4.9 and 5.1 TB/s, dX 35 us and X2 22 at 4.4 and 4.7, 64 -> 1280 215 to 262 us;
//                                             990 001 bfloat16 rows, 64 -> 1280, 630 to 665 us at 4 TB/s.
//   parts_rows_kernel, parts_backward_kernel  the other products of many rows or long sums.  64 x 64 blocks of dW: memory (64 -> 64 as above: 33 us at 4.7
//                                             TB/s, W2 60 us at 4.3).  Wide: the matrix cores and the splitting that feeds them (64 -> 1280 fp32 backward 520
//                                             us, the products of its parts alone 366; 8191 rows, 1024 -> 1024 bfloat16 197 us, 145).
#pragma once
#include "dl_plan.h"

namespace dl {
namespace {

// Parts of an operand on the bfloat16 matrix cores (dl_parts.h): an element that is stored in bfloat16 is one, whatever is computed or stored in fp32 three.
// (fp64: no parts.)
constexpr int kWeightParts = 3;
template <typename T, Source kSource>
constexpr int parts_of(const Operand<float, T, kSource>*) { return sizeof(T) == 2 && kSource == kPlain ? 1 : 3; }
template <typename T, Source kSource>
constexpr int parts_of(const Operand<double, T, kSource>*) { return 0; }
template <typename O>
constexpr int kPartsOf = parts_of(static_cast<O*>(nullptr));
template <typename TS>
constexpr int kRowParts = sizeof(TS) == 2 ? 1 : 3;
template <int kParts, typename T, Source kSource>
__device__ __forceinline__ PartsRows<T, kSource, kParts> as_rows(const Operand<float, T, kSource>& o) { return {o}; }
template <int kParts, typename T, Source kSource>
__device__ __forceinline__ PartsColumns<T, kSource, kParts> as_columns(const Operand<float, T, kSource>& o) { return {o}; }

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
    const int64_t row = row0 + base_row<TA>(wave & 3);   // wave w < 4 finishes the lanes' result r = w
    const int c = n0 + 4 * (lane & 15), lr = lane_row<TA>();
    if (wave < 4 && row + lr < rows && c < w.n_end) {
      TA x[N > 0 ? N : 1][4], v[4] = {0, 0, 0, 0}, sum[4] = {0, 0, 0, 0};
      if (bias) load4<kFours>(bias, c, w.n_end, v);
#pragma unroll
      for (int e = 0; e < N; ++e)
        load4<kFours>(beside.m[e].p + (row + lr) * beside.m[e].ld, c, w.n_end, x[e]);
      for (int p = 0; p < kN; ++p)
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[i] += lds[((p * 4 + wave) * 4 + i) * kLanes + lane];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] += sum[i];
      f(row, lr, c, v, x);
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

// What becomes of four neighbouring results v of a row.  The constructor takes what is the same for a lane's column.
template <typename TS, typename TA, bool kFours, int kResidual>
struct ForwardEnd {   // Z = v (bias added), Y = act(Z) + residual
  static constexpr bool kRounded = sizeof(TS) == 2;   // results go to bfloat16 and nowhere else
  Gate<TA> gate;
  int64_t ld_out;
  int n_end;
  const TS* residual;
  TS *Y, *Z;
  __device__ __forceinline__ Beside<TS, kResidual> beside() const { return {{{residual, ld_out}}}; }
  __device__ __forceinline__ void operator()(int64_t row, int lr, int c, const TA (&z)[4], const TA (&x)[1][4]) const {
    const Spot spot{row * ld_out, static_cast<unsigned>(lr) * static_cast<unsigned>(ld_out) + c};
    TA y[4];
    if (Z) store4<kFours>(at(Z, spot), c, n_end, z);
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = z[i];
    if (gate.on) {
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = gate.value(z[i]);
    }
    if constexpr (kResidual) {
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] += x[0][i];
    }
    store4<kFours>(at(Y, spot), c, n_end, y);
  }
};

// v = V: ddY = V act'(Z), S = V dY act''(Z).  kBeside 0: no activation; 1: no curvature (Z alone is read, no S); 2: Z and dY.
template <typename TS, typename TA, bool kFours, int kBeside>
struct SecondEnd {
  static constexpr bool kRounded = sizeof(TS) == 2 && kBeside < 2;   // (S goes into sums that stay fp32)
  Gate<TA> gate;
  int64_t ld_out;
  int n_end;
  const TS *Z, *dY;
  TS* ddY;
  TA *S, *G;   // G NULL, or where dY act'(Z) goes (g_first)
  __device__ __forceinline__ Beside<TS, kBeside> beside() const {
    if constexpr (kBeside == 2) return {{{Z, ld_out}, {dY, ld_out}}};
    else return {{{Z, ld_out}}};
  }
  __device__ __forceinline__ void operator()(int64_t row, int lr, int c, const TA (&v)[4], const TA (&x)[kBeside > 0 ? kBeside : 1][4]) const {
    TA out[4], s[4], g[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      TA first = TA(1), second = TA(0);
      if constexpr (kBeside > 0) gate.both(x[0][i], &first, &second);
      out[i] = v[i] * first;
      if constexpr (kBeside == 2) g[i] = x[1][i] * first;
      if constexpr (kBeside == 2) s[i] = v[i] * x[1][i] * second;
    }
    if constexpr (kBeside == 2) {
      const Spot spot{row * n_end, static_cast<unsigned>(lr * n_end + c)};
      store4<kFours>(at(S, spot), c, n_end, s);
      if (G) store4<kFours>(at(G, spot), c, n_end, g);
    }
    store4<kFours>(at(ddY, Spot{row * ld_out, static_cast<unsigned>(lr) * static_cast<unsigned>(ld_out) + c}), c, n_end, out);
  }
};

template <typename TS, typename TA, bool kFours>
struct StoreEnd {
  static constexpr bool kRounded = sizeof(TS) == 2;
  int64_t ld;
  int n_end;
  TS* out;
  __device__ __forceinline__ Beside<TS, 0> beside() const { return {}; }
  __device__ __forceinline__ void operator()(int64_t row, int lr, int c, const TA (&v)[4], const TA (&)[1][4]) const {
    store4<kFours>(at(out, Spot{row * ld, static_cast<unsigned>(lr) * static_cast<unsigned>(ld) + c}), c, n_end, v);
  }
};

// Forward and V: rows x W.
template <typename TS, typename TA, int kRT, bool kSplit, bool kFours, typename End>
__global__ __launch_bounds__((threads<kSplit, TA>())) void rows_kernel(Walk walk, Shape shape, int64_t rows, Operand<TA, TS, kPlain> X, AlongRows<TA> W,
                                                                       const TA* __restrict__ bias, End end) {
  __shared__ TA lds[lds_elements<kSplit, kRT, TA>()];
  each_tile<kRT, kSplit>(walk, shape, rows, W.n_end, [&](int64_t row0, int n0) {
    finish_rows<TA, kRT, kSplit, kFours>(X, W, row0, rows, n0, lds, bias, end.beside(), end);
  });
}

// Words of LDS of a product of rows on parts.
template <int kRT, int kX, int kW>
constexpr int rows_words() { return kWaves * kRT * kX * kPlane + shared_words<kW>(); }

// The results of 16 kRT kWaves rows from row0 and of 64 columns by a workgroup.
template <int kRT, int kX, int kW, typename Rows, typename T, int N, typename End>
__device__ __forceinline__ void finish_rows_parts(const Rows& a, const AlongRows<float>& w, int64_t row0, int64_t rows, int n0, unsigned* lds,
                                                  const float* __restrict__ bias, const Beside<T, N>& beside, const End& end) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kLanes);
  Acc acc[kRT][4];
  unsigned* const planes = lds + wave * (kRT * kX * kPlane);
  const Operand<float, float, kPlain> matrix{{w.W, w.n_end}, {}, {}};
  const int64_t first = row0 + wave * (16 * kRT);
  const bool done = rows_parts<kRT, kX, kW, kX == 1 && End::kRounded>(as_rows<kX>(a), SharedColumns<float, kPlain, kW>{matrix}, first, rows, n0, w.n_end,
                                                                      w.k_end, planes, lds + kWaves * kRT * kX * kPlane, acc);
  if (!done) rows_product<float, kRT, true>(a, w, first, rows, n0, 0, w.k_end, reinterpret_cast<float*>(planes), acc);
  unscale<Rows::source>(acc, done);
  each_four<float, kRT, true>(first, rows, n0, w.n_end, acc, bias, beside, end);
}

template <typename TS, int kRT, typename End>
__global__ __launch_bounds__(kThreads, 2) void parts_rows_kernel(Walk walk, int64_t rows, Operand<float, TS, kPlain> X, AlongRows<float> W,
                                                                 const float* __restrict__ bias, End end) {
  constexpr int kX = kRowParts<TS>, kW = kWeightParts;
  __shared__ unsigned lds[rows_words<kRT, kX, kW>()];
  for (int64_t t = blockIdx.x; t < walk.count(); t += gridDim.x) {
    int64_t rg;
    int cg;
    if (!walk.at(t, &rg, &cg)) continue;
    finish_rows_parts<kRT, kX, kW>(X, W, rg * (16 * kRT * kWaves), rows, cg * kCols, lds, bias, end.beside(), end);
    __syncthreads();
  }
}

// A product of rows with a matrix of at most 32 kRounds reduced indices that the waves keep (dl_parts.h).  Weights: W in place (forward, V) or
// transposed (dX), with the same matrix for the fp32 instruction; kX: parts of the rows.
template <typename TS, int kWc, int kRounds, int kX, typename Rows, typename Weights, typename Plain, typename End>
__global__ __launch_bounds__(kThreads, 2) void kept_kernel(Walk walk, int64_t turns, int64_t rows, Rows from, Weights weights, Plain plain,
                                                           const float* __restrict__ bias, End end) {
  constexpr int kW = kWeightParts, kWr = kWaves / kWc;
  constexpr int kTile = kRounds * kX * kPlane, kSlots = kWc > 1 ? 2 : 1;
  __shared__ unsigned lds[kWaves * kSlots * kTile];       // of each group of kWc waves: the planes of kWc tiles, a slot after the other
  __shared__ float corners[kWaves][Corner<float>::kBlock];
  __shared__ unsigned flags[kWr][2 * kWc];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kLanes), lane = threadIdx.x & (kLanes - 1);
  const int own = wave % kWc, group = wave / kWc;
  int64_t rg;
  int cg;
  if (!walk.at(blockIdx.x, &rg, &cg)) return;
  const int n0 = (cg * kWc + own) * kCols, n_end = plain.n_end, k_end = plain.k_end;   // (columns beyond the last are computed and not stored)
  Kept<kRounds, kW> kept;
  keep(weights, n0, n_end, k_end, kept);
  float b[4] = {0, 0, 0, 0};
  if (bias) load4<true>(bias, n0 + 4 * (lane & 15), n_end, b);
  walk_rows<kWc, kRounds, kX, kW, kX == 1 && End::kRounded>(
      as_rows<kX>(from), kept, (rg * kWr + group) * kWc, walk.row_groups * kWaves, turns, own, rows, n0, n_end, k_end, lds + group * kWc * kSlots * kTile,
      flags[group], end.beside(),
      [&](int64_t row0, Acc(&acc)[1][4]) { rows_product<float, 1, true>(from, plain, row0, rows, n0, 0, k_end, corners[wave], acc); },
      [&](int64_t row, int lr, int c, const float(&v)[4], const auto& x) {
        const float z[4] = {v[0] + b[0], v[1] + b[1], v[2] + b[2], v[3] + b[3]};
        end(row, lr, c, z, x);
      });
}

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
  finish_rows<TA, kRT, kSplit, kFours>(g, W, row0, end, n0, lds, none, Beside<TS, 0>{}, StoreEnd<TS, TA, kFours>{ld_in, W.n_end, dX});
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
  TA* const to_dw = dW ? dW + chunk * p.stride() : nullptr;
  TA* const to_db = db && m0 == 0 ? db + chunk * p.stride() : nullptr;
  // column sums: over the four q of the wave, then over the waves
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    sum[u] += __shfl_xor(sum[u], 16);
    sum[u] += __shfl_xor(sum[u], 32);
  }
  const int n = n0 + 4 * j;
  if (p.dw.wr == 1) {
    if (n0 >= k_out) return;
    if (to_db && q == 0 && n < k_out) store4<kFours>(to_db + n, n, k_out, sum);
    if (to_dw) {
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int m = m0 + 4 * Mma<TA>::row(lane, r) + t;
          const TA v[4] = {acc[t][0][r], acc[t][1][r], acc[t][2][r], acc[t][3][r]};
          if (m < k_in && n < k_out) store4<kFours>(to_dw + static_cast<int64_t>(m) * k_out + n, n, k_out, v);
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
        if (m < k_in) store4<kFours>(to_dw + static_cast<int64_t>(m) * k_out + n, n, k_out, v);
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
      store4<kFours>(to_db + n, n, k_out, v);
    }
  }
}

// G: the source of dX.  B, B2: those of dW (kTwo: the second-order pass, x2 B2 added to x B; the column sums are those of B).
template <typename TS, typename TA, int kRT, bool kSplit, bool kFours, bool kTwo, typename G, typename B, typename B2, typename Weights>
__global__ __launch_bounds__((threads<kSplit, TA>())) void backward_kernel(Plan p, int k_in, int k_out, int64_t ld_in, G g, Weights W, TS* __restrict__ dX,
                                                                           Operand<TA, TS, kPlain> x, B b, Operand<TA, TS, kPlain> x2, B2 b2,
                                                                           TA* __restrict__ dW, TA* __restrict__ db) {
  constexpr int kJoin = threads<kSplit, TA>() * 16, kRowsPart = lds_elements<kSplit, kRT, TA>();
  __shared__ TA lds[kJoin > kRowsPart ? kJoin : kRowsPart];
  const Deal deal = p.deal();
  const int64_t total = deal.count();
  for (int64_t t = blockIdx.x; t < total; t += gridDim.x) {
    int64_t chunk, i;
    if (!deal.at(t, &chunk, &i)) continue;
    if (i < p.dx_groups)
      dx_role<TA, kRT, kSplit, kFours>(p, chunk, i, g, W, ld_in, dX, lds);
    else
      dw_role<TA, kTwo, kFours>(p, chunk, static_cast<int>(i - p.dx_groups), k_in, k_out, x, b, x2, b2, dW, db, lds);
    __syncthreads();   // LDS is the next tile's
  }
}

template <int kParts, typename T, Source kSource>
__device__ __forceinline__ SharedColumns<T, kSource, kParts> as_shared(const Operand<float, T, kSource>& o) { return {o}; }

// Partial dW of the rows of a chunk on parts.  Wide: 64 x 256, a wave per 64 columns; otherwise 64 x 64, a wave per 16 rows of dW.
template <bool kWide, bool kTwo, int kX, int kB, int kB2, typename X, typename B, typename B2>
__device__ __forceinline__ void parts_dw_role(const Plan& p, int64_t chunk, int i, int k_in, int k_out, const X& x, const B& b, const X& x2,
                                              const B2& b2, float* __restrict__ dW, float* __restrict__ db, unsigned* lds) {
  constexpr int kT = kWide ? 4 : 1;   // tiles of 16 rows of dW a wave has
  const int lane = threadIdx.x & (kLanes - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kLanes);
  const int j = lane & 15;
  const int m0 = i / p.dw_col_groups * kCols, n0 = (i % p.dw_col_groups * p.dw.wc + (kWide ? wave : 0)) * kCols;
  const int64_t from = chunk * p.per, to = min(p.rows, from + p.per);
  unsigned* const shared_b = lds + shared_words<kX>();
  Acc acc[kT][4];
  float sum[4], none[4];
  auto clear = [&]() {
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      sum[u] = 0;
#pragma unroll
      for (int t = 0; t < kT; ++t) acc[t][u] = Acc{0, 0, 0, 0};
    }
  };
  clear();
  bool done;
  if constexpr (kWide) {
    done = db && m0 == 0 ? outer_parts<kX, kB, true>(as_shared<kX>(x), as_columns<kB>(b), m0, k_in, n0, k_out, from, to, lds, acc, sum)
                         : outer_parts<kX, kB, false>(as_shared<kX>(x), as_columns<kB>(b), m0, k_in, n0, k_out, from, to, lds, acc, sum);
    if constexpr (kTwo) done = outer_parts<kX, kB2, false>(as_shared<kX>(x2), as_columns<kB2>(b2), m0, k_in, n0, k_out, from, to, lds, acc, none) && done;
  } else {
    done = block_parts<kX, kB>(as_shared<kX>(x), as_shared<kB>(b), m0, k_in, n0, k_out, from, to, lds, shared_b, acc, sum);
    if constexpr (kTwo)
      done = block_parts<kX, kB2>(as_shared<kX>(x2), as_shared<kB2>(b2), m0, k_in, n0, k_out, from, to, lds, shared_b, acc, none) && done;
  }
  if (!done) {   // the same for all waves
    clear();
    if constexpr (kWide) {
      outer_product<float, true>(x, b, m0, k_in, n0, k_out, from, to, acc, sum);
      if constexpr (kTwo) outer_product<float, true>(x2, b2, m0, k_in, n0, k_out, from, to, acc, none);
    } else {   // every wave computes the block and keeps its own rows; the column sums are all there in every wave
      Acc whole[4][4];
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int u = 0; u < 4; ++u) whole[t][u] = Acc{0, 0, 0, 0};
      outer_product<float, true>(x, b, m0, k_in, n0, k_out, from, to, whole, sum);
      if constexpr (kTwo) outer_product<float, true>(x2, b2, m0, k_in, n0, k_out, from, to, whole, none);
#pragma unroll
      for (int t = 0; t < 4; ++t)
        if (t == wave) {
#pragma unroll
          for (int u = 0; u < 4; ++u) acc[0][u] = whole[t][u];
        }
      if (wave != 0) {
#pragma unroll
        for (int u = 0; u < 4; ++u) sum[u] = 0;
      }
    }
  }
  static_assert(!kTwo || kScale<B::source> == kScale<B2::source>, "both are in the same sums");
  unscale<B::source>(acc, done);
  const int n = n0 + 4 * j;
  if (dW && n < k_out) {
    float* const to_dw = dW + chunk * p.stride();
#pragma unroll
    for (int t = 0; t < kT; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int m = m0 + 4 * Mma<float>::row(lane, r) + (kWide ? t : wave);
        const float v[4] = {acc[t][0][r], acc[t][1][r], acc[t][2][r], acc[t][3][r]};
        if (m < k_in) store4<true>(to_dw + static_cast<int64_t>(m) * k_out + n, n, k_out, v);
      }
  }
  if (db && m0 == 0) {   // column sums: over the four q of a wave, then over the waves that shared the rows
    float* const to_db = db + chunk * p.stride();
    float* const joined = reinterpret_cast<float*>(lds);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      sum[u] += __shfl_xor(sum[u], 16);
      sum[u] += __shfl_xor(sum[u], 32);
    }
    if constexpr (!kWide) {
      if (lane < 16) {
#pragma unroll
        for (int u = 0; u < 4; ++u) joined[(wave * 4 + u) * 16 + j] = sum[u];
      }
      __syncthreads();
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        sum[u] = 0;
        for (int w = 0; w < kWaves; ++w) sum[u] += joined[(w * 4 + u) * 16 + j];
      }
    }
    if (lane < 16 && n < k_out && (kWide || wave == 0)) store4<true>(to_db + n, n, k_out, sum);
  }
}

// backward_kernel on parts.  WT: W transposed.  kDx: is there a dX here?  (Without it the 64 x 64 blocks leave room for more waves.)
template <typename TS, int kRT, bool kWide, bool kDx, bool kTwo, typename G, typename B, typename B2>
__global__ __launch_bounds__(kThreads, kWide || kDx ? 2 : 3) void parts_backward_kernel(Plan p, int k_in, int k_out, int64_t ld_in, G g, AlongRows<float> WT,
                                                                     TS* __restrict__ dX, Operand<float, TS, kPlain> x, B b,
                                                                     Operand<float, TS, kPlain> x2, B2 b2, float* __restrict__ dW,
                                                                     float* __restrict__ db) {
  constexpr int kX = kRowParts<TS>, kG = kPartsOf<G>, kB = kPartsOf<B>, kB2 = kPartsOf<B2>;
  constexpr int kDxWords = kDx ? rows_words<kRT, kG, kWeightParts>() : 0;
  constexpr int kDwWords = shared_words<kX>() + (kWide ? 0 : shared_words<(kB > kB2 ? kB : kB2)>());
  __shared__ unsigned lds[kDxWords > kDwWords ? kDxWords : kDwWords];
  const Deal deal = p.deal();
  const int64_t total = deal.count();
  for (int64_t t = blockIdx.x; t < total; t += gridDim.x) {
    int64_t chunk, i;
    if (!deal.at(t, &chunk, &i)) continue;
    if (kDx && i < p.dx_groups) {
      if constexpr (kDx) {
        const int64_t row0 = chunk * p.per + i / p.dx_col_groups * (16 * kRT * kWaves), end = min(p.rows, (chunk + 1) * p.per);
        const int n0 = static_cast<int>(i % p.dx_col_groups) * kCols;
        const float* const none = nullptr;
        if (row0 < end)
          finish_rows_parts<kRT, kG, kWeightParts>(g, WT, row0, end, n0, lds, none, Beside<TS, 0>{}, StoreEnd<TS, float, true>{ld_in, k_in, dX});
      }
    } else {
      parts_dw_role<kWide, kTwo, kX, kB, kB2>(p, chunk, static_cast<int>(i - p.dx_groups), k_in, k_out, x, b, x2, b2, dW, db, lds);
    }
    __syncthreads();
  }
}

// G = dY act'(Z) as a tensor of its own, in the arithmetic type: where several column blocks of dX would each make it again.
template <typename TS, typename TA, bool kFours>
__global__ __launch_bounds__(kThreads) void gate_kernel(int64_t rows, int cols, int64_t ld, Gate<TA> gate, const TS* __restrict__ dY,
                                                        const TS* __restrict__ Z, TA* __restrict__ G) {
  const int fours = (cols + 3) / 4;
  for (int64_t i = blockIdx.x * static_cast<int64_t>(kThreads) + threadIdx.x; i < rows * fours; i += static_cast<int64_t>(gridDim.x) * kThreads) {
    const int64_t row = i / fours;
    const int c = static_cast<int>(i - row * fours) * 4;
    TA g[4], z[4];
    load4<kFours>(dY + row * ld, c, cols, g);
    load4<kFours>(Z + row * ld, c, cols, z);
#pragma unroll
    for (int k = 0; k < 4; ++k) g[k] *= gate.first(z[k]);
    store4<kFours>(G + row * cols + c, c, cols, g);
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
      if (at < n_dw) dW[at] = v;
      else db[at - n_dw] = v;
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

  // Launches a product of rows with W [k_in][k_out] on the fp32 or fp64 instruction: launch(row tiles, split, fours), all known at compile time.
  // Widths that are no multiple of four test every element and are bound by that: one row tile does for them.
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

  // rows x W with an epilogue: make(fours) gives it.
  template <typename Make>
  hipError_t rows_times_w(const void* X, const void* W, const void* b, Make&& make) const {
    const AlongRows<TA> along{static_cast<const TA*>(W), c->k_in, c->k_out};
    if constexpr (sizeof(TA) == 4) {
      if (kept_ok(c, n, c->k_out, c->k_in)) {
        const auto end = make(std::true_type{});
        const PartsColumns<float, kPlain, kWeightParts> weights{{{along.W, c->k_out}, {}, {}}};
        return kept<kRowParts<TS>>(c->k_out, c->k_in, rows_in(X), weights, along, b, end);
      }
    }
    if constexpr (sizeof(TA) == 4) {
      if (in_parts(c, n, c->k_out, c->k_in, sizeof(TS) == 4 ? 2 * kFewBlocks : kFewBlocks)) {
        const int rt = parts_tiles(n, c->k_out);
        const Walk walk{blocks_of(n, 16 * rt * kWaves), static_cast<int>(blocks_of(c->k_out, kCols))};
        const auto end = make(std::true_type{});
        auto launch = [&](auto tiles) {
          hipLaunchKernelGGL((parts_rows_kernel<TS, tiles.value, std::decay_t<decltype(end)>>), dim3(grid_of(walk.count())), dim3(kThreads), 0, stream,
                             walk, n, rows_in(X), along, static_cast<const float*>(b), end);
          return hipGetLastError();
        };
        return rt == kPartsTiles ? launch(std::integral_constant<int, kPartsTiles>{}) : launch(std::integral_constant<int, 1>{});
      }
    }
    return by_shape(c->k_out, c->k_in, [&](auto rt, auto split, auto fours) {
      const Shape shape = shape_of(c->k_out);
      const Walk walk = walk_of(rt, split, shape);
      const auto end = make(fours);
      hipLaunchKernelGGL((rows_kernel<TS, TA, rt.value, split.value, fours.value, std::decay_t<decltype(end)>>),
                         dim3(grid_of(walk.count())), dim3((threads<split.value, TA>())), 0, stream, walk, shape, n, rows_in(X), along,
                         static_cast<const TA*>(b), end);
      return hipGetLastError();
    });
  }

  template <int kX, typename Rows, typename Weights, typename Plain, typename End>
  hipError_t kept(int cols, int k, const Rows& rows, const Weights& weights, const Plain& plain, const void* b, const End& end) const {
    const Shape shape = shape_of(cols);
    const int col_groups = static_cast<int>(blocks_of(cols, kCols * shape.wc));
    // two waves for every SIMD, all at once
    const int64_t groups = std::max<int64_t>(kXcds, std::min<int64_t>(512 / col_groups, blocks_of(n, 16 * kWaves)) / kXcds * kXcds);
    const Walk walk{groups, col_groups};
    const int64_t turns = blocks_of(blocks_of(n, 16), groups * kWaves);
    auto launch = [&](auto wc, auto rounds) {
      hipLaunchKernelGGL((kept_kernel<TS, wc.value, rounds.value, kX, Rows, Weights, Plain, End>), dim3(grid_of(walk.count())), dim3(kThreads), 0,
                         stream, walk, turns, n, rows, weights, plain, static_cast<const float*>(b), end);
      return hipGetLastError();
    };
    const std::integral_constant<int, 1> one{};
    const std::integral_constant<int, 2> two{};
    const std::integral_constant<int, 4> four{};
    if (k <= kRound) return shape.wc == 1 ? launch(one, one) : shape.wc == 2 ? launch(two, one) : launch(four, one);
    return shape.wc == 1 ? launch(one, two) : shape.wc == 2 ? launch(two, two) : launch(four, two);
  }

  template <int kResidual>
  hipError_t forward_with(const void* X, const void* W, const void* b, const void* residual, void* Y, void* Z) const {
    return rows_times_w(X, W, b, [&](auto fours) {
      return ForwardEnd<TS, TA, fours.value, kResidual>{Gate<TA>::of(c->activation), ld_out(c), c->k_out, static_cast<const TS*>(residual),
                                                        static_cast<TS*>(Y), static_cast<TS*>(Z)};
    });
  }
  hipError_t forward(const void* X, const void* W, const void* b, const void* residual, void* Y, void* Z) const {
    return residual ? forward_with<1>(X, W, b, residual, Y, Z) : forward_with<0>(X, W, b, residual, Y, Z);
  }

  template <int kBeside>
  hipError_t v_with(const void* HX, const void* W, const void* Z, const void* dY, void* ddY, TA* S, TA* G) const {
    return rows_times_w(HX, W, nullptr, [&](auto fours) {
      return SecondEnd<TS, TA, fours.value, kBeside>{Gate<TA>::of(c->activation), ld_out(c), c->k_out, static_cast<const TS*>(Z),
                                                     static_cast<const TS*>(dY), static_cast<TS*>(ddY), S, G};
    });
  }
  hipError_t v(const void* HX, const void* W, const void* Z, const void* dY, void* ddY, TA* S, TA* G) const {
    return S ? v_with<2>(HX, W, Z, dY, ddY, S, G)
             : c->activation == DL_NONE ? v_with<0>(HX, W, Z, dY, ddY, S, G) : v_with<1>(HX, W, Z, dY, ddY, S, G);
  }

  // ws: [ W transposed ][ partial results ].
  template <bool kTwo, typename G, typename B, typename B2>
  hipError_t gradients(const G& source, const void* W, void* dX, const void* X, const B& b, const void* X2, const B2& b2, void* dW,
                       void* db, void* ws) const {
    if constexpr (sizeof(TA) == 4) {
      if (dX && kept_ok(c, n, c->k_in, c->k_out)) {   // dX by itself, then dW
        const float* w = static_cast<const float*>(W);
        const PartsTransposed<kWeightParts> weights{{w, c->k_out}};
        const hipError_t e = kept<kPartsOf<G>>(c->k_in, c->k_out, source, weights, AlongColumns<float>{w, c->k_out, c->k_in},
                                                                                nullptr, StoreEnd<TS, float, true>{ld_in(c), c->k_in, static_cast<TS*>(dX)});
        return e != hipSuccess || !(dW || db) ? e : gradients<kTwo>(source, W, nullptr, X, b, X2, b2, dW, db, ws);
      }
    }
    if constexpr (sizeof(TA) == 4) {
      if (in_parts(c, n, c->k_in, c->k_out)) {
        if (dX) {
          const hipError_t e = transpose(W, ws);
          if (e != hipSuccess) return e;
        }
        auto with_tiles = [&](auto tiles) {
          if (wide_parts(c)) return parts_gradients<tiles.value, true, true, kTwo>(source, dX, X, b, X2, b2, dW, db, ws);
          return parts_gradients<tiles.value, false, true, kTwo>(source, dX, X, b, X2, b2, dW, db, ws);
        };
        if (dX) return parts_tiles(n, c->k_in) == kPartsTiles ? with_tiles(std::integral_constant<int, kPartsTiles>{}) : with_tiles(std::integral_constant<int, 1>{});
        return wide_parts(c) ? parts_gradients<1, true, false, kTwo>(source, dX, X, b, X2, b2, dW, db, ws)
                             : parts_gradients<1, false, false, kTwo>(source, dX, X, b, X2, b2, dW, db, ws);
      }
    }
    return by_shape(c->k_in, c->k_out, [&](auto rt, auto split, auto fours) {
      if constexpr (!split.value && fours.value) {
        if (dX && transposed(n, c)) {
          const hipError_t e = transpose(W, ws);
          if (e != hipSuccess) return e;
          return gradients_with<kTwo>(rt, split, fours, source, AlongRows<TA>{static_cast<const TA*>(ws), c->k_out, c->k_in}, dX, X, b, X2, b2, dW,
                                      db, ws);
        }
      }
      return gradients_with<kTwo>(rt, split, fours, source, AlongColumns<TA>{static_cast<const TA*>(W), c->k_out, c->k_in}, dX, X, b, X2, b2, dW, db,
                                  ws);
    });
  }

  hipError_t transpose(const void* W, void* wt) const {
    const int64_t tiles = blocks_of(c->k_in, 32) * blocks_of(c->k_out, 32);
    hipLaunchKernelGGL((transpose_kernel<TA>), dim3(static_cast<unsigned>(tiles)), dim3(kThreads), 0, stream, c->k_in, c->k_out,
                       static_cast<const TA*>(W), static_cast<TA*>(wt));
    return hipGetLastError();
  }

  // dW and db where a chunk's results go: the outputs themselves if there is one chunk.
  struct Target {
    TA *dw, *db, *part;
  };
  Target target(const Plan& p, void* dW, void* db, void* ws) const {
    TA* part = reinterpret_cast<TA*>(static_cast<char*>(ws) + wt_bytes(n, c));
    const bool whole = p.chunks == 1;
    return {!dW ? nullptr : whole ? static_cast<TA*>(dW) : part,
            !db ? nullptr : whole ? static_cast<TA*>(db) : part + p.n_dw, part};
  }
  hipError_t join(const Plan& p, const Target& to, void* dW, void* db) const {
    const hipError_t e = hipGetLastError();
    return e != hipSuccess || p.chunks == 1 || !(dW || db) ? e : sum_chunks(to.part, p.chunks, p.n_dw, dW, p.n_db, db);
  }

  template <bool kTwo, typename RT, typename Split, typename Fours, typename G, typename Weights, typename B, typename B2>
  hipError_t gradients_with(RT rt, Split split, Fours, const G& source, const Weights& w, void* dX, const void* X, const B& b, const void* X2,
                            const B2& b2, void* dW, void* db, void* ws) const {
    const Plan p = plan_of(c, n, Wanted{dX != nullptr, dW != nullptr, db != nullptr}, split, rt);
    const Target to = target(p, dW, db, ws);
    hipLaunchKernelGGL((backward_kernel<TS, TA, RT::value, Split::value, Fours::value, kTwo, G, B, B2, Weights>), dim3(grid_of(p.deal().count())),
                       dim3((threads<Split::value, TA>())), 0, stream, p, c->k_in, c->k_out, ld_in(c), source, w, static_cast<TS*>(dX), rows_in(X), b,
                       rows_in(X2), b2, to.dw, to.db);
    return join(p, to, dW, db);
  }

  // kRT: row tiles of a wave of dX
  template <int kRT, bool kWide, bool kDx, bool kTwo, typename G, typename B, typename B2>
  hipError_t parts_gradients(const G& source, void* dX, const void* X, const B& b, const void* X2, const B2& b2, void* dW, void* db, void* ws) const {
    const Plan p = parts_plan(c, n, Wanted{dX != nullptr, dW != nullptr, db != nullptr});
    const Target to = target(p, dW, db, ws);
    hipLaunchKernelGGL((parts_backward_kernel<TS, kRT, kWide, kDx, kTwo, G, B, B2>), dim3(grid_of(p.deal().count())), dim3(kThreads), 0, stream, p, c->k_in, c->k_out,
                       ld_in(c), source, (AlongRows<float>{static_cast<const float*>(ws), c->k_out, c->k_in}), static_cast<TS*>(dX), rows_in(X), b,
                       rows_in(X2), b2, to.dw, to.db);
    return join(p, to, dW, db);
  }

  // n_dw, n_db: what a chunk holds of each
  hipError_t sum_chunks(const TA* part, int64_t chunks, int64_t n_dw, void* dW, int64_t n_db, void* db) const {
    hipLaunchKernelGGL((sum_chunks_kernel<TA>), dim3(static_cast<unsigned>(std::min<int64_t>(blocks_of(n_dw + n_db, 64), 1 << 16))), dim3(kThreads), 0,
                       stream, part, chunks, n_dw + n_db, n_dw, n_db, static_cast<TA*>(dW), static_cast<TA*>(db));
    return hipGetLastError();
  }
  hipError_t zero(void* dW, void* db) const {
    if (!dW && !db) return hipSuccess;
    return sum_chunks(nullptr, 0, dW ? static_cast<int64_t>(c->k_in) * c->k_out : 0, dW, db ? c->k_out : 0, db);
  }

  hipError_t backward(const void* X, const void* W, const void* Z, const void* dY, void* dX, void* dW, void* db, void* ws) const {
    if (c->activation == DL_NONE) return gradients<false>(g<kPlain>(dY, Z), W, dX, X, g<kPlain>(dY, Z), X, g<kPlain>(dY, Z), dW, db, ws);
    if (g_first(c, n)) {
      const hipError_t e = make_g(dY, Z, static_cast<TA*>(ws));
      if (e != hipSuccess) return e;
      const Operand<TA, TA, kMade> made{{static_cast<const TA*>(ws), c->k_out}, {}, {}};
      return gradients<false>(made, W, dX, X, made, X, made, dW, db, static_cast<char*>(ws) + s_bytes(c, n));
    }
    return gradients<false>(g<kGated>(dY, Z), W, dX, X, g<kGated>(dY, Z), X, g<kGated>(dY, Z), dW, db, ws);
  }

  hipError_t make_g(const void* dY, const void* Z, TA* G) const {
    const dim3 grid(grid_of(std::min<int64_t>(blocks_of(n * blocks_of(c->k_out, 4), kThreads), 8192)));
    const Gate<TA> gate = Gate<TA>::of(c->activation);
    if (c->k_out % 4 == 0)
      hipLaunchKernelGGL((gate_kernel<TS, TA, true>), grid, dim3(kThreads), 0, stream, n, c->k_out, ld_out(c), gate, static_cast<const TS*>(dY),
                         static_cast<const TS*>(Z), G);
    else
      hipLaunchKernelGGL((gate_kernel<TS, TA, false>), grid, dim3(kThreads), 0, stream, n, c->k_out, ld_out(c), gate, static_cast<const TS*>(dY),
                         static_cast<const TS*>(Z), G);
    return hipGetLastError();
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
    TA* G = S && g_first(c, n) ? reinterpret_cast<TA*>(static_cast<char*>(ws) + s_bytes(c, n)) : nullptr;
    void* part = static_cast<char*>(ws) + (G ? 2 : 1) * s_bytes(c, n);
    hipError_t e = v(HX, W, Z, dY, ddY, S, G);
    if (e != hipSuccess) return e;
    if (!S) {   // act'' = 0: W2 is dW of HX, X2 and b2 are zero
      e = zero_rows(X2, c->k_in, ld_in(c));
      if (e == hipSuccess) e = zero(nullptr, b2);
      if (e != hipSuccess || !W2) return e;
      if (c->activation == DL_NONE)
        return gradients<false>(g<kPlain>(dY, Z), W, nullptr, HX, g<kPlain>(dY, Z), HX, g<kPlain>(dY, Z), W2, nullptr, part);
      return gradients<false>(g<kGated>(dY, Z), W, nullptr, HX, g<kGated>(dY, Z), HX, g<kGated>(dY, Z), W2, nullptr, part);
    }
    if (!X2 && !W2 && !b2) return hipSuccess;
    const Operand<TA, TA, kMade> s{{S, c->k_out}, {}, {}}, made{{G, c->k_out}, {}, {}};
    if (G) return gradients<true>(s, W, X2, X, s, HX, made, W2, b2, part);
    return gradients<true>(s, W, X2, X, s, HX, g<kGated>(dY, Z), W2, b2, part);
  }
};

template <typename TS, typename TA>
struct EntryOf {
  typedef Calls<TS, TA> C;
  static hipError_t forward(const dl_config* c, int64_t n, hipStream_t stream, const void* X, const void* W, const void* b, const void* residual,
                            void* Y, void* Z) {
    return C{c, n, stream}.forward(X, W, b, residual, Y, Z);
  }
  static hipError_t backward(const dl_config* c, int64_t n, hipStream_t stream, const void* X, const void* W, const void* Z, const void* dY, void* dX,
                             void* dW, void* db, void* ws) {
    return C{c, n, stream}.backward(X, W, Z, dY, dX, dW, db, ws);
  }
  static hipError_t double_backward(const dl_config* c, int64_t n, hipStream_t stream, const void* X, const void* W, const void* Z, const void* dY,
                                    const void* HX, void* ddY, void* X2, void* W2, void* b2, void* ws) {
    return C{c, n, stream}.double_backward(X, W, Z, dY, HX, ddY, X2, W2, b2, ws);
  }
  static hipError_t zero(const dl_config* c, hipStream_t stream, void* dW, void* db) {
    return C{c, 0, stream}.zero(dW, db);
  }
};

}  // namespace
}  // namespace dl
