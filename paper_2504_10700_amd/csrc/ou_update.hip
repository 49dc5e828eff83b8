// The orthogonalised update of include/ou.h: arguments, entry points, and the kernels that serve every case.
//
// The list goes to the workspace once.  Then, each for all tensors of a way together: momentum and sums of squares; X = U / norm; per step S = X X^T, P = b S + c S S,
// X = a X + P X; the last step's results go straight into the update and the weights.
#include <algorithm>
#include <cfloat>
#include <cmath>
#include <string>
#include <type_traits>

#include "el_tile.h"
#include "ou_internal.h"

namespace ou {
namespace {

using el::Mma;
using sc::DeviceGuard;
using sc::misaligned;
using sc::set_error;


__global__ __launch_bounds__(kLanes) void send_kernel(const Sent sent, Item* __restrict__ items) {
  const int i = threadIdx.x;
  if (i < sent.count) items[sent.first + i] = sent.item[i];
}

// Momentum of a chunk of elements, and the sum of their U's squares.  A matrix's sum is that of its chunks.  (A few elements of a thread are requested together: a store
// between two loads would make the second wait.)  Memory bounds it: 33 million elements with bfloat16 gradients 75 us, 4.4 TB/s.
constexpr int kAtOnce = 8;
template <typename TA>
__device__ __forceinline__ void gradients(const Item& it, int64_t at, int i0, int count, TA (&u)[kAtOnce]) {
  auto read = [&](auto* g) {
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) u[k] = i0 + k * kThreads < count ? static_cast<TA>(g[at + i0 + k * kThreads]) : TA(0);
  };
  if constexpr (sizeof(TA) == 8) read(static_cast<const double*>(it.grad));
  else if (it.dtype == SC_BF16) read(static_cast<const __bf16*>(it.grad));
  else read(static_cast<const float*>(it.grad));
}
template <typename TA>
__global__ __launch_bounds__(kThreads) void momentum_kernel(const Item* __restrict__ items, int n, const Step st, double* __restrict__ partial) {
  __shared__ double slots[kWaves];
  const Item& it = items[item_of(items, n, kChunks, blockIdx.x)];
  const int64_t size = static_cast<int64_t>(it.rows) * it.cols, per = chunks_of(size), unit = blockIdx.x - it.unit[kChunks];
  const int64_t matrix = unit / per, first = unit % per * kChunk, at = matrix * size + first;
  const int count = static_cast<int>(min(size - first, static_cast<int64_t>(kChunk)));
  const TA mu = static_cast<TA>(st.mu);
  TA* const momentum = it.momentum ? static_cast<TA*>(it.momentum) + at : nullptr;
  Squares sum{0, 0, 0};   // (fp32: one sum, of squares that fp64 holds)
  for (int i0 = threadIdx.x; i0 < count; i0 += kAtOnce * kThreads) {
    TA u[kAtOnce], v[kAtOnce];
    gradients(it, at, i0, count, u);
    if (momentum) {
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) v[k] = i0 + k * kThreads < count ? momentum[i0 + k * kThreads] : TA(0);
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) {
        v[k] = mu * v[k] + u[k];
        if (i0 + k * kThreads < count) momentum[i0 + k * kThreads] = v[k];
        u[k] = direction(u[k], v[k], mu, st.nesterov);
      }
    }
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      if constexpr (sizeof(TA) == 8) add_square(sum, u[k]);
      else sum.middle = fma(static_cast<double>(u[k]), static_cast<double>(u[k]), sum.middle);
    }
  }
  sum.middle = workgroup_sum(sum.middle, slots);
  if constexpr (sizeof(TA) == 8) {
    sum.small = workgroup_sum(sum.small, slots);
    sum.large = workgroup_sum(sum.large, slots);
    if (threadIdx.x == 0) reinterpret_cast<Squares*>(partial)[blockIdx.x] = sum;
  } else {
    if (threadIdx.x == 0) partial[blockIdx.x] = sum.middle;
  }
}

// ---- fp64, and fp32 where parts do not hold a step (parts_hold): X = U / (norm + eps), in the tensor's own orientation; last: no steps follow

template <typename TA>
using Sum = std::conditional_t<sizeof(TA) == 8, Squares, double>;   // of a chunk

template <typename TA>
__global__ __launch_bounds__(kThreads) void normalise_kernel(const Item* __restrict__ items, int n, const Step st, bool last, TA* __restrict__ X,
                                                             const Sum<TA>* __restrict__ partial) {
  __shared__ double slots[kWaves];
  const Item& it = items[item_of(items, n, kChunks, blockIdx.x)];
  const int64_t size = static_cast<int64_t>(it.rows) * it.cols, per = chunks_of(size), unit = blockIdx.x - it.unit[kChunks];
  const int64_t matrix = unit / per, first = unit % per * kChunk;
  const int count = static_cast<int>(min(size - first, static_cast<int64_t>(kChunk)));
  const auto down = down_of(partial + it.unit[kChunks] + matrix * per, per, st.eps, slots);
  const TA mu = static_cast<TA>(st.mu);
  for (int i = threadIdx.x; i < count; i += kThreads) {
    const int64_t e = matrix * size + first + i;
    TA u = gradient<TA>(it, e);
    if (it.momentum) u = direction(u, static_cast<const TA*>(it.momentum)[e], mu, st.nesterov);
    if constexpr (sizeof(TA) == 8) u = u * down.first * down.second;
    else u = static_cast<TA>(static_cast<double>(u) * down);
    if (last) finish(it, st, e, u); else X[it.x + e] = u;
  }
}

__device__ __forceinline__ void barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }   // (requests to memory stay under way)

// Element (i, k) of a matrix at p[i * ld + k * step].
template <typename TA>
struct View {
  const TA* p;
  int64_t ld, step;
  int rows, depth;
};

// A tile of kTile x kTile, kDepth reduced indices at a time.  Four waves of 16 rows x 64 columns, or of 16 x 16.
template <typename TA, int kTile>
struct Square {
  static constexpr int kDepth = 1024 / kTile, kPitch = kTile + 4;
  static constexpr int kAcross = kTile == 64 ? 1 : 2;          // waves side by side
  static constexpr int kColumns = kTile / 16 / kAcross;        // 16 x 16 of a wave
  typedef TA Space[kDepth][kPitch];
  typedef typename Mma<TA>::acc_t Sums[kColumns];
};

// Sums over k of P(i, k) Q(j, k) of the tile (i0, j0).
template <typename TA, int kTile>
__device__ __forceinline__ void product(const View<TA>& p, const View<TA>& q, int i0, int j0, typename Square<TA, kTile>::Space& ps,
                                        typename Square<TA, kTile>::Space& qs, typename Square<TA, kTile>::Sums& acc) {
  using S = Square<TA, kTile>;
  constexpr int kDepth = S::kDepth;
  const int lane = threadIdx.x & (kLanes - 1), wave = threadIdx.x / kLanes, thread = threadIdx.x;
  const int row0 = 16 * (wave / S::kAcross), col0 = 16 * (wave % S::kAcross);
  const int depth = p.depth;
  // (neighbouring threads along what is contiguous)
  auto load = [&](const View<TA>& v, int r0, int k, TA (&x)[4]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int kk = v.step == 1 ? k + thread % kDepth : k + thread / kTile + e * (kThreads / kTile);
      const int r = r0 + (v.step == 1 ? thread / kDepth + e * (kThreads / kDepth) : thread % kTile);
      x[e] = kk < depth && r < v.rows ? v.p[r * v.ld + kk * v.step] : TA(0);
    }
  };
  auto put = [&](const View<TA>& v, typename S::Space& to, const TA (&x)[4]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (v.step == 1) to[thread % kDepth][thread / kDepth + e * (kThreads / kDepth)] = x[e];
      else to[thread / kTile + e * (kThreads / kTile)][thread % kTile] = x[e];
    }
  };
  // (an fp32 instruction cuts off what is below the last bit of the sum it adds to, so a sum goes no further than kFlush indices and then joins another)
  constexpr bool kJoin = sizeof(TA) == 4;
  constexpr int kFlush = 128;
  typename S::Sums joined;
#pragma unroll
  for (int t = 0; t < S::kColumns; ++t) acc[t] = joined[t] = typename Mma<TA>::acc_t{0, 0, 0, 0};
  TA x[4], y[4];   // a stage's indices, requested while those before are multiplied
  load(p, i0, 0, x);
  load(q, j0, 0, y);
  for (int k = 0; k < depth; k += kDepth) {
    barrier();
    put(p, ps, x);
    put(q, qs, y);
    if (k + kDepth < depth) {
      load(p, i0, k + kDepth, x);
      load(q, j0, k + kDepth, y);
    }
    barrier();
#pragma unroll
    for (int s = 0; s < kDepth / 4; ++s) {
      const TA a = ps[4 * s + lane / 16][row0 + (lane & 15)];
#pragma unroll
      for (int t = 0; t < S::kColumns; ++t) acc[t] = Mma<TA>::mma(a, qs[4 * s + lane / 16][col0 + 16 * t + (lane & 15)], acc[t]);
    }
    if (kJoin && (k + kDepth) % kFlush == 0) {
#pragma unroll
      for (int t = 0; t < S::kColumns; ++t) {
        joined[t] += acc[t];
        acc[t] = typename Mma<TA>::acc_t{0, 0, 0, 0};
      }
    }
  }
  if (kJoin) {
#pragma unroll
    for (int t = 0; t < S::kColumns; ++t) acc[t] += joined[t];
  }
}

enum Phase { kS, kP, kX };

// The three products of a step: S from X; P from S; the next X from P and X (last: into the results).
template <typename TA, int kPhase, int kTile>
__global__ __launch_bounds__(kThreads) void product_kernel(const Item* __restrict__ items, int n, const Step st, bool last, const TA* __restrict__ X,
                                                           TA* __restrict__ next, TA* __restrict__ S, TA* __restrict__ P) {
  using Tile = Square<TA, kTile>;
  __shared__ typename Tile::Space ps, qs;
  constexpr int kind = kTile == 64 ? (kPhase == kX ? kProduct : kGram) : kPhase == kX ? kProductSmall : kGramSmall;
  const int lane = threadIdx.x & (kLanes - 1), wave = threadIdx.x / kLanes;
  const Item& it = items[item_of(items, n, kind, blockIdx.x)];
  const bool turned = it.rows > it.cols;
  const int m = turned ? it.cols : it.rows, l = turned ? it.rows : it.cols;   // X as m x l: element (i, k) at i * si + k * sk
  const int64_t si = turned ? 1 : it.cols, sk = turned ? it.cols : 1;
  const int columns = kPhase == kX ? l : m;
  const int row_tiles = (m + kTile - 1) / kTile, col_tiles = (columns + kTile - 1) / kTile;
  const int64_t unit = blockIdx.x - it.unit[kind], per = static_cast<int64_t>(row_tiles) * col_tiles, matrix = unit / per;
  const int tile = static_cast<int>(unit % per), i0 = tile / col_tiles * kTile, j0 = tile % col_tiles * kTile;
  const int64_t x0 = it.x + matrix * m * l, s0 = it.s + matrix * m * m;
  typename Tile::Sums acc;
  if constexpr (kPhase == kS) {
    const View<TA> v{X + x0, si, sk, m, l};
    product<TA, kTile>(v, v, i0, j0, ps, qs, acc);
  } else if constexpr (kPhase == kP) {
    const View<TA> v{S + s0, m, 1, m, m};
    product<TA, kTile>(v, v, i0, j0, ps, qs, acc);
  } else {
    const View<TA> p{P + s0, m, 1, m, m}, x{X + x0, sk, si, l, m};
    product<TA, kTile>(p, x, i0, j0, ps, qs, acc);
  }
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int i = i0 + 16 * (wave / Tile::kAcross) + Mma<TA>::row(lane, r);
#pragma unroll
    for (int t = 0; t < Tile::kColumns; ++t) {
      const int j = j0 + 16 * (wave % Tile::kAcross) + 16 * t + (lane & 15);
      if (i >= m || j >= columns) continue;
      if constexpr (kPhase == kS) {
        S[s0 + static_cast<int64_t>(i) * m + j] = acc[t][r];
      } else if constexpr (kPhase == kP) {
        const int64_t at = s0 + static_cast<int64_t>(i) * m + j;
        P[at] = static_cast<TA>(st.b) * S[at] + static_cast<TA>(st.c) * acc[t][r];
      } else {
        const int64_t at = i * si + j * sk;
        const TA x = static_cast<TA>(st.a) * X[x0 + at] + acc[t][r];
        if (last) finish(it, st, matrix * m * l + at, x); else next[x0 + at] = x;
      }
    }
  }
}

// ---- host side

// The ways: fp64; fp32 on fp32 instructions; products in tiles of parts; and matrices whose shorter side is at most 64 or 128, in slices or whole.  The four from kPlain on have the
// first pass together.
enum Way { kDouble, kPlain, kParts, kSlices64, kSlices128, kWhole64, kWhole128, kWays };
bool whole(int way) { return way == kWhole64 || way == kWhole128; }
bool sliced(int way) { return way == kSlices64 || way == kSlices128; }
bool large(int way) { return way == kWhole128 || way == kSlices128; }

// The tensors by the way that their matrices take, and where everything lies in the workspace.
struct Layout {
  Part part[kWays];
  std::vector<Item> items;   // of all ways, in their order
  size_t bytes = 0;
};

// Whether parts hold the steps as fp32 does.  A part of S, or of P = b S + c S S, is off by up to 2^-38 of what the bound `top` of the singular values allows, |b| top^2 + |c| top^4, however
// small the matrix's own values have become; a X stands beside P X.  So relative to X a step is off by sqrt(m) 2^-38 (|b| top^2 + |c| top^4) / |a|, for m of up to 65536 and a ratio
// of 64 by 2^-24.  The usual coefficients have 3.2; with a = 0 the values are cubed and nothing holds the small ones (three steps of X S: 64 x 64 off by 100%).
constexpr double kMostBeside = 64;
bool parts_hold(const ou_config* c) {
  double top = 1;
  for (int i = 0; i < c->steps; ++i) {
    const double square = std::max(top * top, kLeastBound);
    if (std::fabs(c->b) * square + std::fabs(c->c) * std::max(square * square, kLeastBound) > kMostBeside * std::fabs(c->a)) return false;
    top = growth(c, top);
  }
  return true;
}

// One workgroup holds what it can: one launch, or one a step, instead of three a step.
Way way_of(const ou_tensor& t, bool parts) {
  const int m = std::min(t.rows, t.cols), l = std::max(t.rows, t.cols);
  return t.dtype == SC_F64 ? kDouble : !parts ? kPlain : l <= 64 ? kWhole64 : l <= 128 ? kWhole128 : m <= 64 ? kSlices64 : m <= 128 ? kSlices128 : kParts;
}

void square_place(Part& p, Item& it, int64_t count) {
  const int64_t m = std::min(it.rows, it.cols), l = std::max(it.rows, it.cols);
  it.x = p.x;
  it.s = p.s;
  for (const int tile : {64, 32}) {
    const int64_t tm = ceil_div(m, tile), tl = ceil_div(l, tile);
    p.units[tile == 64 ? kGram : kGramSmall] += count * tm * tm;
    p.units[tile == 64 ? kProduct : kProductSmall] += count * tm * tl;
  }
  p.x += count * m * l;
  p.s += count * m * m;
}

void square_layout(Part& p, Room& room, int steps, size_t size) {
  if (steps == 0) return;
  p.at_x = room(p.x * size);
  p.at[0] = room(p.x * size);
  p.at[1] = room(p.s * size);
  p.at[2] = room(p.s * size);
}

Layout layout_of(const ou_config* cfg, int64_t n, const ou_tensor* tensors) {
  Layout l;
  const int steps = cfg->steps;
  const bool parts = parts_hold(cfg);
  int64_t matrices[kWays] = {};
  for (int64_t i = 0; i < n; ++i) matrices[way_of(tensors[i], parts)] += tensors[i].count;
  for (int64_t i = 0; i < n; ++i) {
    const ou_tensor& t = tensors[i];
    if (t.count == 0) continue;
    const Way way = way_of(t, parts);
    Part& p = l.part[way];
    Item it{};
    it.grad = t.grad;
    it.momentum = t.momentum;
    it.weight = t.weight;
    it.update = t.update;
    it.scale = t.scale;
    std::copy_n(p.units, static_cast<int>(kKinds), it.unit);
    it.rows = t.rows;
    it.cols = t.cols;
    it.dtype = t.dtype;
    if (!whole(way)) p.units[kChunks] += t.count * ceil_div(static_cast<int64_t>(t.rows) * t.cols, kChunk);
    if (way <= kPlain) square_place(p, it, t.count);
    else if (way == kParts) parts_place(p, it, t.count);
    else if (sliced(way)) slice_place(p, it, t.count, matrices[way], large(way));
    else p.units[kBlocks] += t.count;
    p.items.push_back(it);
  }
  Room room;
  room(n * sizeof(Item));
  l.part[kDouble].at_partial = room(l.part[kDouble].units[kChunks] * sizeof(Squares));
  int64_t chunks = 0;
  for (int way = kPlain; way <= kSlices128; ++way) {
    for (Item& it : l.part[way].items) it.unit[kChunks] += chunks;
    chunks += l.part[way].units[kChunks];
  }
  const size_t at_partial = room(chunks * sizeof(double));
  for (int way = 0; way < kWays; ++way) {
    Part& p = l.part[way];
    p.at_items = l.items.size() * sizeof(Item);
    l.items.insert(l.items.end(), p.items.begin(), p.items.end());
    if (way != kDouble) p.at_partial = at_partial;
    if (p.items.empty()) continue;
    if (way <= kPlain) square_layout(p, room, steps, way == kDouble ? sizeof(double) : sizeof(float));
    else if (way == kParts) parts_layout(p, room, steps);
    else if (sliced(way)) slice_layout(p, room, steps, large(way));
  }
  l.bytes = std::max<size_t>(room.bytes, 256);
  return l;
}

bool representable(double v, int32_t dtype) { return std::fabs(v) <= (dtype == SC_F64 ? DBL_MAX : static_cast<double>(FLT_MAX)); }

sc_status check(const char* fn, const ou_config* cfg, int64_t n, const ou_tensor* tensors) {
  auto bad = [&](sc_status st, const std::string& what) { return set_error(st, std::string(fn) + ": " + what); };
  if (!cfg) return bad(SC_ERR_INVALID_ARG, "cfg is NULL");
  if (cfg->struct_size != static_cast<int32_t>(sizeof(ou_config)))
    return bad(SC_ERR_INVALID_ARG, "struct_size does not match this library's ou_config");
  if (cfg->steps < 0) return bad(SC_ERR_INVALID_ARG, "steps < 0");
  if (cfg->steps > OU_MAX_STEPS) return bad(SC_ERR_UNSUPPORTED, "steps above OU_MAX_STEPS");
  if (cfg->flags & ~static_cast<uint32_t>(OU_NESTEROV)) return bad(SC_ERR_INVALID_ARG, "unknown flags");
  for (double v : {cfg->a, cfg->b, cfg->c, cfg->momentum, cfg->rate, cfg->decay})
    if (!std::isfinite(v)) return bad(SC_ERR_INVALID_ARG, "a coefficient, momentum, rate or decay is not finite");
  if (!(cfg->eps > 0) || !std::isfinite(cfg->eps)) return bad(SC_ERR_INVALID_ARG, "eps not above 0 or not finite");
  double top = 1;
  for (int i = 0; i < cfg->steps; ++i) {
    top = growth(cfg, top);
    if (!(top <= OU_MAX_GROWTH)) return bad(SC_ERR_UNSUPPORTED, "with these coefficients the iteration grows beyond OU_MAX_GROWTH");
  }
  if (n < 0) return bad(SC_ERR_INVALID_ARG, "n_tensors < 0");
  if (n > OU_MAX_TENSORS) return bad(SC_ERR_UNSUPPORTED, "more than OU_MAX_TENSORS tensors");
  if (n > 0 && !tensors) return bad(SC_ERR_INVALID_ARG, "tensors is NULL");
  int64_t total = 0;
  for (int64_t i = 0; i < n; ++i) {
    const ou_tensor& t = tensors[i];
    const char* what = nullptr;
    if (t.dtype != SC_F32 && t.dtype != SC_F64 && t.dtype != SC_BF16) what = "bad dtype";
    else if (t.reserved != 0) what = "reserved is not 0";
    else if (t.rows < 1 || t.cols < 1) what = "rows or cols < 1";
    else if (t.count < 0) what = "count < 0";
    else if (!representable(t.scale, t.dtype) || !representable(cfg->rate * t.scale, t.dtype)) what = "scale, or rate * scale, is not finite in the tensor's arithmetic";
    else if (!representable(cfg->momentum, t.dtype) || !representable(1 - cfg->rate * cfg->decay, t.dtype)) what = "momentum or rate * decay is not finite in the tensor's arithmetic";
    else if (t.count > 0 && !t.grad) what = "grad is NULL";
    else if (t.count > 0 && !t.weight && !t.update) what = "weight and update are both NULL";
    const size_t narrow = t.dtype == SC_F64 ? 8 : t.dtype == SC_F32 ? 4 : 2, wide = t.dtype == SC_F64 ? 8 : 4;
    if (!what && (misaligned(t.grad, narrow) || misaligned(t.update, narrow) || misaligned(t.momentum, wide) || misaligned(t.weight, wide)))
      what = "pointer not aligned to its element";
    if (what) return bad(SC_ERR_INVALID_ARG, "tensor " + std::to_string(i) + ": " + what);
    if (t.rows > OU_MAX_SIDE || t.cols > OU_MAX_SIDE) return bad(SC_ERR_UNSUPPORTED, "tensor " + std::to_string(i) + ": rows or cols above OU_MAX_SIDE");
    const int64_t tiles = ceil_div(t.rows, 64) * ceil_div(t.cols, 64);
    if (t.count > (OU_MAX_TILES - total) / tiles) return bad(SC_ERR_UNSUPPORTED, "more than OU_MAX_TILES tiles");
    total += t.count * tiles;
  }
  return SC_OK;
}

hipError_t send(const std::vector<Item>& items, char* base, hipStream_t stream) {
  const int n = static_cast<int>(items.size());
  for (int first = 0; first < n; first += kSent) {
    Sent sent{};
    sent.first = first;
    sent.count = std::min(kSent, n - first);
    std::copy_n(items.begin() + first, sent.count, sent.item);
    hipLaunchKernelGGL(send_kernel, dim3(1), dim3(kLanes), 0, stream, sent, reinterpret_cast<Item*>(base));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// Momentum and sums of squares of the ways from `way` to `end`.
template <typename TA>
hipError_t first_pass(const Layout& l, int way, int end, const Step& st, char* base, hipStream_t stream) {
  int n = 0;
  int64_t chunks = 0;
  for (int w = way; w <= end; ++w) {
    n += static_cast<int>(l.part[w].items.size());
    chunks += l.part[w].units[kChunks];
  }
  if (n == 0) return hipSuccess;
  hipLaunchKernelGGL(momentum_kernel<TA>, dim3(static_cast<unsigned>(chunks)), dim3(kThreads), 0, stream,
                     reinterpret_cast<const Item*>(base + l.part[way].at_items), n, st, reinterpret_cast<double*>(base + l.part[way].at_partial));
  return hipGetLastError();
}

// Tiles of 64 that do not fill the compute units: smaller ones (fp64, five steps of one 512 x 700 299 us instead of 716, of 40 512 x 512 4.1 ms instead of 3.5).
template <typename TA, int kPhase>
hipError_t launch(const Part& p, const Item* items, const Step& st, bool last, const TA* X, TA* next, TA* S, TA* P, hipStream_t stream) {
  const int n = static_cast<int>(p.items.size());
  const int64_t tiles = p.units[kPhase == kX ? kProduct : kGram];
  if (tiles > 256)
    hipLaunchKernelGGL((product_kernel<TA, kPhase, 64>), dim3(static_cast<unsigned>(tiles)), dim3(kThreads), 0, stream, items, n, st, last, X, next, S, P);
  else
    hipLaunchKernelGGL((product_kernel<TA, kPhase, 32>), dim3(static_cast<unsigned>(p.units[kPhase == kX ? kProductSmall : kGramSmall])), dim3(kThreads), 0, stream,
                       items, n, st, last, X, next, S, P);
  return hipGetLastError();
}

template <typename TA>
hipError_t square_run(const Part& p, const ou_config* cfg, const Step& st, char* base, hipStream_t stream) {
  const int n = static_cast<int>(p.items.size());
  const Item* const items = reinterpret_cast<const Item*>(base + p.at_items);
  const Sum<TA>* const partial = reinterpret_cast<const Sum<TA>*>(base + p.at_partial);
  TA* const X[2] = {reinterpret_cast<TA*>(base + p.at_x), reinterpret_cast<TA*>(base + p.at[0])};
  TA* const S = reinterpret_cast<TA*>(base + p.at[1]);
  TA* const P = reinterpret_cast<TA*>(base + p.at[2]);
  hipLaunchKernelGGL(normalise_kernel<TA>, dim3(static_cast<unsigned>(p.units[kChunks])), dim3(kThreads), 0, stream, items, n, st, cfg->steps == 0, X[0], partial);
  hipError_t e = hipGetLastError();
  for (int i = 0; i < cfg->steps && e == hipSuccess; ++i) {
    const bool last = i + 1 == cfg->steps;
    const TA* const x = X[i & 1];
    TA* const next = X[(i + 1) & 1];
    e = launch<TA, kS>(p, items, st, last, x, next, S, P, stream);
    if (e == hipSuccess) e = launch<TA, kP>(p, items, st, last, x, next, S, P, stream);
    if (e == hipSuccess) e = launch<TA, kX>(p, items, st, last, x, next, S, P, stream);
  }
  return e;
}

}  // namespace

double growth(const ou_config* c, double top) {
  auto f = [&](double x) { return std::fabs(x * (c->a + x * x * (c->b + x * x * c->c))); };
  double most = f(top);
  // where the derivative a + 3 b y + 5 c y^2, y = x^2, is zero
  const double q = 5 * c->c, p = 3 * c->b, d = p * p - 4 * q * c->a;
  double roots[3] = {-1, -1, -1};
  if (q != 0 && d >= 0) {
    roots[0] = (-p + std::sqrt(d)) / (2 * q);
    roots[1] = (-p - std::sqrt(d)) / (2 * q);
  }
  if (p != 0) roots[2] = -c->a / p;   // (without c; with it an ordinary point inside, which does no harm)
  for (double y : roots)
    if (y > 0 && y < top * top) most = std::max(most, f(std::sqrt(y)));
  return most;
}

}  // namespace ou

extern "C" {

sc_status ou_workspace_bytes(const ou_config* cfg, int64_t n_tensors, const ou_tensor* tensors, size_t* bytes) {
  using namespace ou;
  const sc_status st = check("ou_workspace_bytes", cfg, n_tensors, tensors);
  if (st != SC_OK) return st;
  if (!bytes) return set_error(SC_ERR_INVALID_ARG, "ou_workspace_bytes: bytes is NULL");
  try {
    *bytes = layout_of(cfg, n_tensors, tensors).bytes;
  } catch (const std::bad_alloc&) {
    return set_error(SC_ERR_ALLOC, "ou_workspace_bytes: out of host memory");
  }
  return SC_OK;
}

sc_status ou_step(const ou_config* cfg, int64_t n_tensors, const ou_tensor* tensors, void* workspace, size_t workspace_bytes,
                  void* hip_stream) {
  using namespace ou;
  const sc_status st = check("ou_step", cfg, n_tensors, tensors);
  if (st != SC_OK) return st;
  try {
    const Layout l = layout_of(cfg, n_tensors, tensors);
    if (l.items.empty()) return SC_OK;
    if (!workspace || workspace_bytes < l.bytes)
      return set_error(SC_ERR_WORKSPACE, "ou_step: workspace missing or smaller than ou_workspace_bytes()");
    if (misaligned(workspace, 256)) return set_error(SC_ERR_WORKSPACE, "ou_step: workspace not 256-byte aligned");
    DeviceGuard guard(cfg->device);
    if (!guard.ok) return set_error(SC_ERR_HIP, "ou_step: cannot make cfg->device current");
    const Step step{cfg->a, cfg->b, cfg->c, cfg->momentum, cfg->rate, 1 - cfg->rate * cfg->decay, cfg->eps, (cfg->flags & OU_NESTEROV) != 0};
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    char* const base = static_cast<char*>(workspace);
    hipError_t e = send(l.items, base, stream);
    if (e == hipSuccess) e = first_pass<double>(l, kDouble, kDouble, step, base, stream);
    if (e == hipSuccess) e = first_pass<float>(l, kPlain, kSlices128, step, base, stream);
    if (e == hipSuccess) e = whole_run(l.part[kWhole64], l.part[kWhole128], cfg, step, base, stream);
    for (int way = kDouble; way <= kSlices128 && e == hipSuccess; ++way) {
      const Part& p = l.part[way];
      if (p.items.empty()) continue;
      e = way == kDouble  ? square_run<double>(p, cfg, step, base, stream)
          : way == kPlain ? square_run<float>(p, cfg, step, base, stream)
          : way == kParts ? parts_run(p, cfg, step, base, stream)
                          : slice_run(p, cfg, step, large(way), base, stream);
    }
    if (e != hipSuccess) return set_error(SC_ERR_HIP, std::string("ou_step: kernel launch: ") + hipGetErrorString(e));
  } catch (const std::bad_alloc&) {
    return set_error(SC_ERR_ALLOC, "ou_step: out of host memory");
  }
  return SC_OK;
}

}  // extern "C"
