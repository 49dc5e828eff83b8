// The products of the orthogonalised update on the fp16 matrix cores, for matrices of any size.
//
// No element of X, S = X X^T or P = b S + c S S is larger than the largest singular value can be, which the host knows for every step.
// So an fp32 value v, times a power of two that brings that bound to at most 2^14, is the sum of two fp16 values h + l (h rounded from it, l from what is
// left): 22 bits of it down to 2^-16 of the bound, and an error of 2^-39 of the bound below, where it is lost in the matrix's norm.  A product is
// h h' + h l' + l h' (l l' is below 2^-22 of it): three instructions where bfloat16 parts take six and fp32 instructions the time of 16.
// An instruction cuts off what is below the last bit of the sum it adds to, so a sum goes no further than kFlush indices and then joins an fp32 sum.
//
// Every product is one of rows with rows, sum over k of A[i][k] B[j][k], both operands contiguous in k: S from X and X, P from S and S (symmetric), the
// next X from P and X transposed.  So the epilogues leave X in both orientations, split once where it is made and not where it is used.  Of S and P the
// tiles on and below the diagonal are computed and mirrored.
//
// A workgroup: 128 x 128, four waves of 64 x 64; 32 reduced indices of both operands' parts (32 KB) go from memory to LDS without passing registers while
// the 32 before are multiplied, and a second workgroup of the compute unit fills the waits (4096 x 4096: 0.97 ms a step, 850 TFLOP/s of fp16 products, where
// a large library product of fp16 reaches 1068).  Where there are not tiles enough for that (few_tiles), 64 x 64 with four stages (three and a third workgroup: 512 x 512
// 39 us a step instead of 30; eight and one workgroup: 32).  A row's four pieces of 16 bytes stand at places that differ between rows
// (swizzle), against bank conflicts.
#include <algorithm>
#include <cmath>

#include "ou_internal.h"

namespace ou {
namespace {

typedef _Float16 H8 __attribute__((ext_vector_type(8)));
typedef _Float16 H4 __attribute__((ext_vector_type(4)));
typedef float F16 __attribute__((ext_vector_type(16)));
typedef unsigned U4 __attribute__((ext_vector_type(4)));
typedef float F4 __attribute__((ext_vector_type(4)));
typedef float F4Loose __attribute__((ext_vector_type(4), aligned(4)));

constexpr int kDepth = 32, kFlush = 128;
constexpr int kRow = 2 * kDepth;          // elements of a row in LDS: h and l
constexpr int kPad = 32;                  // rows of the parts in memory are multiples of this
constexpr int kPitch = 36;                // floats of a row of a wave's 32 x 32 in LDS
constexpr int kXcds = 8;
constexpr int kFewTiles = 256;

// Columns of a row of parts in memory: an odd multiple of 32, so that the rows of a tile spread over the channels of the caches.
__host__ __device__ constexpr int64_t padded(int64_t n) { return ((n + kPad - 1) / kPad | 1) * kPad; }


// Buffers.  Parts: [rows][padded columns / 32][h, l][32] of each matrix: what a stage reads of a row is one line of the caches (with h and l apart, and so half
// lines: 4096 x 4096 twice 10.2 ms instead of 9.3).
struct Buffers {
  float* X;             // [m][l]
  _Float16* x;          // X
  _Float16* t;          // X transposed
  _Float16* next;       // the next X transposed
  _Float16* s;
  _Float16* p;
};

// Powers of two of a step.
struct Scales {
  float up;      // values that the phase makes to parts
  float down;    // sums of parts to values
  float beside;  // parts of S to values (phase P)
};

// The parts of a 32 x 32 block in LDS to rows of parts that begin at `to`, `pitch` apart; the block's columns are c on, a multiple of 32.  kTurned: value (i, j) is at
// block[j * kStep + i], otherwise at block[i * kStep + j].  Rows from `rows` on are not there, columns from `inside` on are zeros.  Eight lanes write the line of a row,
// the first four its h, eight values each, the others its l in reverse: a lane splits four of the eight values, and its mirror image the other four.
template <bool kTurned, int kStep>
__device__ __forceinline__ void put_parts(const float* block, float up, int rows, int inside, _Float16* to, int64_t pitch, int c) {
  const int lane = threadIdx.x & (kLanes - 1);
  const bool second = lane & 4;
  const int piece = (second ? 7 - lane % 8 : lane % 8) * 8, mine = piece + (second ? 4 : 0);
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int row = lane / 8 + 8 * k;
    float v[4];
    if (!kTurned && kStep % 4 == 0) {
      const F4 x = *reinterpret_cast<const F4*>(block + row * kStep + mine);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = x[i];
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = kTurned ? block[(mine + i) * kStep + row] : block[row * kStep + mine + i];
    }
    if (inside < 32) {
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = mine + i < inside ? v[i] : 0.f;
    }
    unsigned h[2], l[2], other[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      split2(v[2 * i] * up, v[2 * i + 1] * up, h[i], l[i]);
      other[i] = __builtin_amdgcn_update_dpp(0u, second ? h[i] : l[i], 0x141, 0xf, 0xf, true);   // (row_half_mirror)
    }
    const U4 parts = second ? U4{other[0], other[1], l[0], l[1]} : U4{h[0], h[1], other[0], other[1]};
    if (row < rows) *reinterpret_cast<U4*>(to + row * pitch + 2 * c + (second ? 32 : 0) + piece) = parts;
  }
}

// A 64 x 64 block of X = U / (norm + eps): X, and its parts in both orientations.  last: no steps follow.  Memory bounds it: 2 x 4096 x 4096 131 us for 268 MB read and
// 403 written.
__global__ __launch_bounds__(kThreads) void normalise_kernel(const Item* __restrict__ items, int n, const Step st, bool last, const Buffers buf, float up,
                                                             const double* __restrict__ partial) {
  __shared__ double slots[kWaves];
  __shared__ float block[64][65];
  const Item& it = items[item_of(items, n, kBlocks, blockIdx.x)];
  const bool turned = it.rows > it.cols;
  const int m = turned ? it.cols : it.rows, l = turned ? it.rows : it.cols;
  const int64_t size = static_cast<int64_t>(m) * l, per = chunks_of(size);
  const int col_blocks = (it.cols + 63) / 64, row_blocks = (it.rows + 63) / 64;
  const int64_t unit = blockIdx.x - it.unit[kBlocks], blocks = static_cast<int64_t>(col_blocks) * row_blocks, matrix = unit / blocks;
  const int b = static_cast<int>(unit % blocks), r0 = b / col_blocks * 64, c0 = b % col_blocks * 64;
  const double down = down_of(partial + it.unit[kChunks] + matrix * per, per, st.eps, slots);
  const float mu = static_cast<float>(st.mu);
  // (a quarter of the block's rows after the other, each read whole before the next is asked for)
  const int c = threadIdx.x % 64;
  for (int r = threadIdx.x / 64; r < 64; r += 16) {
    float u[4], v[4];
    bool inside[4];
    int64_t at[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      inside[k] = r0 + r + 4 * k < it.rows && c0 + c < it.cols;
      at[k] = matrix * size + static_cast<int64_t>(r0 + r + 4 * k) * it.cols + c0 + c;
      u[k] = inside[k] ? gradient<float>(it, at[k]) : 0.f;
    }
    if (it.momentum) {
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = inside[k] ? static_cast<const float*>(it.momentum)[at[k]] : 0.f;
#pragma unroll
      for (int k = 0; k < 4; ++k) u[k] = direction(u[k], v[k], mu, st.nesterov);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float x = static_cast<float>(static_cast<double>(u[k]) * down);
      if (last && inside[k]) finish(it, st, at[k], x);
      if (turned) block[c][r + 4 * k] = x; else block[r + 4 * k][c] = x;
    }
  }
  if (last) return;
  __syncthreads();
  const int i0 = turned ? c0 : r0, j0 = turned ? r0 : c0;   // of the m x l matrix
  for (int i = threadIdx.x; i < 64 * 64; i += kThreads)
    if (i0 + i / 64 < m && j0 + i % 64 < l) buf.X[it.x + matrix * size + static_cast<int64_t>(i0 + i / 64) * l + j0 + i % 64] = block[i / 64][i % 64];
  // (a wave a quarter of the block)
  const int64_t lp = padded(l), mp = padded(m);
  const int wave = threadIdx.x / kLanes, qi = wave / 2 * 32, qj = wave % 2 * 32;
  const int ib = i0 + qi, jb = j0 + qj;
  if (ib >= m || jb >= l) return;
  put_parts<false, 65>(&block[qi][qj], up, m - ib, l - jb, buf.x + it.px + 2 * (matrix * m + ib) * lp, 2 * lp, jb);
  put_parts<true, 65>(&block[qi][qj], up, l - jb, m - ib, buf.t + it.pt + 2 * (matrix * l + jb) * mp, 2 * mp, ib);
}

// Tile t of those on and below the diagonal of rows x rows tiles.  Eight rows of tiles at a time, column after column, so that what runs at the same time on
// an XCD shares its operands.
constexpr int kGroup = 8;
__device__ __forceinline__ void lower_tile(int t, int rows, int& i, int& j) {
  int g = static_cast<int>((sqrtf(16.f + 128.f * t) - 4.f) / 64.f);
  while (32 * (g + 1) * (g + 1) + 4 * (g + 1) <= t) ++g;
  while (32 * g * g + 4 * g > t) --g;
  t -= 32 * g * g + 4 * g;
  const int first = kGroup * g, high = min(kGroup, rows - first);
  if (t < first * high) {
    j = t / high;
    i = first + t % high;
    return;
  }
  t -= first * high;
  int r = 0;
  while ((r + 1) * (r + 2) / 2 <= t) ++r;
  i = first + r;
  j = first + t - r * (r + 1) / 2;
}
__device__ __forceinline__ void any_tile(int t, int rows, int cols, int& i, int& j) {
  const int g = t / (kGroup * cols), first = kGroup * g, high = min(kGroup, rows - first);
  t -= kGroup * cols * g;
  j = t / high;
  i = first + t % high;
}

__device__ __forceinline__ int swizzle(int row) { return ((row >> 1) & 7) ^ ((row & 1) << 2); }   // rows 0..7, and the even and the odd ones of 16, all differ

// Half of a tile's rows (clamped to the last), 32 reduced indices, to LDS: eight rows with each request of a wave.
template <int kLoads>
__device__ __forceinline__ void load_rows(const _Float16* __restrict__ from, const unsigned (&offset)[kLoads], _Float16* to) {
#pragma unroll
  for (int q = 0; q < kLoads; ++q) {
    const auto* const g = reinterpret_cast<const __attribute__((address_space(1))) unsigned*>(
        reinterpret_cast<uintptr_t>(reinterpret_cast<const char*>(from) + offset[q]));
    __builtin_amdgcn_global_load_lds(g, reinterpret_cast<__attribute__((address_space(3))) unsigned*>(reinterpret_cast<uintptr_t>(to + q * 8 * kRow)), 16, 0, 0);
  }
}

__device__ __forceinline__ void wave_sync() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// Waits until at most N of the wave's requests are under way, then for the workgroup.  Behind the barrier a slot is filled again that the waves have read before it: each waits
// for its reads here (lgkmcnt), since the products that use them are not held before the barrier by anything else.
template <int N>
__device__ __forceinline__ void arrived() { asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory"); }
// The stage that is multiplied next has arrived, of the `left` (at most kAhead) after it none has to.
template <int kAhead, int kLoads>
__device__ __forceinline__ void stage_arrived(int left) {
  if constexpr (kAhead == 0) arrived<0>();
  else if (left >= kAhead) arrived<kAhead * kLoads>();
  else stage_arrived<kAhead - 1, kLoads>(left);
}

// Four finished elements of X of which `inside` are there.
__device__ __forceinline__ void finish4(const Item& it, const Step& st, int64_t at, int inside, const F4& x) {
  if (inside >= 4 && it.dtype == SC_F32) {
    if (it.update) *reinterpret_cast<F4Loose*>(static_cast<float*>(it.update) + at) = x;
    if (it.weight) {
      F4Loose* const w = reinterpret_cast<F4Loose*>(static_cast<float*>(it.weight) + at);
      F4 v = *w;
#pragma unroll
      for (int n = 0; n < 4; ++n) v[n] = new_weight(it, st, static_cast<float>(v[n]), static_cast<float>(x[n]));
      *w = v;
    }
    return;
  }
#pragma unroll
  for (int n = 0; n < 4; ++n)
    if (n < inside) finish(it, st, at + n, static_cast<float>(x[n]));
}

enum Phase { kS, kP, kX };

template <int kTile, int kStages>
struct Ring {
  static constexpr int kOperand = kTile * kRow;
  static constexpr int kStage = 2 * kOperand;
  static constexpr int kBytes = kStages * kStage * 2;
};

template <int kPhase, int kTile, int kStages>
__global__ __launch_bounds__(kThreads, 2) void product_kernel(const Item* __restrict__ items, int n, const Step st, bool last, const Buffers buf, const Scales sc,
                                                              int total) {
  using R = Ring<kTile, kStages>;
  constexpr int kOperand = R::kOperand, kStage = R::kStage, kLoads = kTile / 16, kSide = kTile / 64;   // kSide: 32 x 32 blocks along a wave's side
  extern __shared__ __attribute__((aligned(16))) _Float16 lds[];
  constexpr int kind = kTile == 128 ? (kPhase == kX ? kProduct : kGram) : kPhase == kX ? kProductSmall : kGramSmall;
  const int per_xcd = (total + kXcds - 1) / kXcds;
  const int u = static_cast<int>(blockIdx.x) % kXcds * per_xcd + blockIdx.x / kXcds;
  if (u >= total) return;
  const Item& it = items[item_of(items, n, kind, u)];
  const bool turned = it.rows > it.cols;
  const int m = turned ? it.cols : it.rows, l = turned ? it.rows : it.cols;
  const int64_t mp = padded(m), lp = padded(l);
  const int tiles_m = (m + kTile - 1) / kTile, tiles_l = (l + kTile - 1) / kTile;
  const int per = kPhase == kX ? tiles_m * tiles_l : tiles_m * (tiles_m + 1) / 2;
  const int unit = static_cast<int>(u - it.unit[kind]), matrix = unit / per;
  int ti, tj;
  if constexpr (kPhase == kX) any_tile(unit % per, tiles_m, tiles_l, ti, tj);
  else lower_tile(unit % per, tiles_m, ti, tj);
  const int i0 = ti * kTile, j0 = tj * kTile;
  const int lane = threadIdx.x & (kLanes - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kLanes);

  // operands: rows of A and of B, both from the same matrix but for the last phase.  Two waves bring A, two B.
  const int64_t ld = 2 * (kPhase == kS ? lp : mp);
  const bool of_b = wave & 2;
  const _Float16* from = kPhase == kS   ? buf.x + it.px + matrix * m * ld
                         : kPhase == kP ? buf.s + it.ps + matrix * m * ld
                         : of_b         ? buf.t + it.pt + matrix * l * ld
                                        : buf.p + it.ps + matrix * m * ld;
  const int row0 = (of_b ? j0 : i0), left = (of_b && kPhase == kX ? l : m) - row0, half = wave % 2 * (kTile / 2);
  from += row0 * ld;
  unsigned offset[kLoads];
#pragma unroll
  for (int q = 0; q < kLoads; ++q) {
    const int r = half + 8 * q + lane / 8;
    offset[q] = 2u * (static_cast<unsigned>(min(r, left - 1)) * static_cast<unsigned>(ld) + 8u * ((lane % 8) ^ swizzle(r)));
  }
  const int stages = ((kPhase == kS ? l : m) + kDepth - 1) / kDepth;
  _Float16* const mine = lds + wave / 2 * kOperand + half * kRow;
  const int wi = wave / 2 * 32 * kSide, wj = wave % 2 * 32 * kSide;

  // (one block: each of the three products has a sum of its own, so that no instruction waits for the one before it)
  constexpr int kSums = kSide == 1 ? 3 : 1;
  F16 sum[kSide][kSide], part[kSums][kSide][kSide];
#pragma unroll
  for (int x = 0; x < kSide; ++x)
#pragma unroll
    for (int y = 0; y < kSide; ++y)
#pragma unroll
      for (int r = 0; r < 16; ++r) sum[x][y][r] = 0;

  struct Operands {
    H8 x[2][kSide][2], y[2][kSide][2];   // [16 indices][block][part]
  };
  auto read = [&](const _Float16* here, Operands& o) {
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int e = 0; e < kSide; ++e)
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          const int r = e * 32 + (lane & 31), piece = ((4 * q + 2 * s + lane / 32) ^ swizzle(r)) * 8;   // (wi and wj are multiples of 32)
          o.x[s][e][q] = *reinterpret_cast<const H8*>(here + (wi + r) * kRow + piece);
          o.y[s][e][q] = *reinterpret_cast<const H8*>(here + kOperand + (wj + r) * kRow + piece);
        }
  };
  auto multiply = [&](const Operands& o, int from_s, int to_s) {
#pragma unroll
    for (int s = from_s; s < to_s; ++s)
#pragma unroll
      for (int q = 0; q < 3; ++q)   // l h, h l, h h
#pragma unroll
        for (int e = 0; e < kSide; ++e)
#pragma unroll
          for (int f = 0; f < kSide; ++f) {
            F16& sums = part[kSums == 3 ? q : 0][e][f];
            sums = __builtin_amdgcn_mfma_f32_32x32x16_f16(o.x[s][e][q == 0], o.y[s][f][q == 1], sums, 0, 0, 0);
          }
  };
  // stage t stands in slot t % kStages
  int filled = 0, slot = 0, to = 0;
  auto fill = [&] {
    load_rows<kLoads>(from + static_cast<int64_t>(filled) * kRow, offset, mine + to * kStage);
    ++filled;
    to = to + 1 == kStages ? 0 : to + 1;
  };
  auto next_slot = [&] {
    const _Float16* const here = lds + slot * kStage;
    slot = slot + 1 == kStages ? 0 : slot + 1;
    return here;
  };
  while (filled < kStages - 1 && filled < stages) fill();
  // One block: a stage's operands are read while the one before it is multiplied, so that neither the reads nor the barrier are waited for alone.  A slot is filled again
  // after the barrier that follows the products of its stage.
  constexpr bool kAhead = kSide == 1;
  Operands operands[kAhead ? 2 : 1];
  if constexpr (kAhead) {
    stage_arrived<kStages - 2, kLoads>(stages - 1);
    read(next_slot(), operands[0]);
  }
  for (int first = 0; first < stages; first += kFlush / kDepth) {
#pragma unroll
    for (int k = 0; k < kSums; ++k)
#pragma unroll
      for (int e = 0; e < kSide; ++e)
#pragma unroll
        for (int f = 0; f < kSide; ++f)
#pragma unroll
          for (int r = 0; r < 16; ++r) part[k][e][f][r] = 0;
    if constexpr (kAhead) {
#pragma unroll
      for (int u = 0; u < kFlush / kDepth; ++u) {
        const int t = first + u;
        if (t >= stages) break;
        if (t + 1 < stages) stage_arrived<kStages - 3, kLoads>(stages - 2 - t);
        read(next_slot(), operands[(u + 1) & 1]);   // (after the last stage: whatever stands in the slot, not used)
        // (the requests go out while the matrix core works)
        multiply(operands[u & 1], 0, 1);
        __builtin_amdgcn_sched_barrier(0);
        if (filled < stages && t + 1 < stages) fill();
        multiply(operands[u & 1], 1, 2);
      }
    } else {
      const int until = min(first + kFlush / kDepth, stages);
      for (int t = first; t < until; ++t) {
        stage_arrived<kStages - 2, kLoads>(stages - 1 - t);
        if (filled < stages) fill();
        read(next_slot(), operands[0]);
        multiply(operands[0], 0, 2);
      }
    }
#pragma unroll
    for (int e = 0; e < kSide; ++e)
#pragma unroll
      for (int f = 0; f < kSide; ++f) {
        if constexpr (kSums == 3) sum[e][f] += part[2][e][f] + (part[0][e][f] + part[1][e][f]);
        else sum[e][f] += part[0][e][f];
      }
  }

  // results, 32 x 32 at a time through the wave's corner of LDS: row by row, then column by column
  const int row = lane / 8, column = lane % 8 * 4;   // fp32 values: eight lanes have a line
  const bool mirrored = kPhase != kX && ti != tj;
  const int columns = kPhase == kX ? l : m;
  const float ca = static_cast<float>(st.a), cb = static_cast<float>(st.b), cc = static_cast<float>(st.c);
  // what stands beside a block's sums, S (its parts) or X, requested a block ahead (rows beyond the last: the last one)
  constexpr int kBlocks = kSide * kSide;
  F4 beside[2][4];
  auto request = [&](int block) {
    if constexpr (kPhase == kS) return;
    const int ib = i0 + wi + 32 * (block / kSide), jb = j0 + wj + 32 * (block % kSide);
    if (ib >= m || jb >= columns) return;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int i = min(ib + row + 8 * k, m - 1), j = jb + column;
      F4 x{0, 0, 0, 0};
      if constexpr (kPhase == kP) {
        const _Float16* const parts = buf.s + it.ps + 2 * ((matrix * m + i) * mp + jb) + column;   // (22 bits of S; b S has no need of more beside S S of the same parts)
        const H4 h = *reinterpret_cast<const H4*>(parts), low = *reinterpret_cast<const H4*>(parts + 32);
        x = (__builtin_convertvector(h, F4) + __builtin_convertvector(low, F4)) * sc.beside;
      } else {
        const float* const X = buf.X + it.x + (static_cast<int64_t>(matrix) * m + i) * l;
        if (jb + 32 <= l) {
          x = *reinterpret_cast<const F4Loose*>(X + j);
        } else {
#pragma unroll
          for (int n = 0; n < 4; ++n) x[n] = X[min(j + n, l - 1)];
        }
      }
      beside[block & 1][k] = x;
    }
  };
  request(0);
  __syncthreads();
  float* const corner = reinterpret_cast<float*>(lds) + wave * 32 * kPitch;
#pragma unroll
  for (int e = 0; e < kSide; ++e)
#pragma unroll
    for (int f = 0; f < kSide; ++f) {
      const int block = e * kSide + f, ib = i0 + wi + 32 * e, jb = j0 + wj + 32 * f;
      if (block + 1 < kBlocks) request(block + 1);
      if (ib >= m || jb >= columns) continue;
#pragma unroll
      for (int r = 0; r < 16; ++r) corner[(8 * (r / 4) + 4 * (lane / 32) + r % 4) * kPitch + (lane & 31)] = sum[e][f][r] * sc.down;
      wave_sync();
      // what the phase makes of the sums, in fp32
#pragma unroll
      for (int k = 0; k < (kPhase == kS ? 0 : 4); ++k) {
        const int i = ib + row + 8 * k, j = jb + column;
        float* const here = corner + (row + 8 * k) * kPitch + column;
        F4 v = *reinterpret_cast<const F4*>(here);
        if constexpr (kPhase == kP) v = cb * beside[block & 1][k] + cc * v;
        if constexpr (kPhase == kX) v = ca * beside[block & 1][k] + v;
        if constexpr (kPhase == kX) {
          if (i < m) {
            const int64_t at = (static_cast<int64_t>(matrix) * m + i) * l + j;
            float* const X = buf.X + it.x + at;
            if (last) {
              if (!turned) finish4(it, st, at, l - j, v);
            } else if (j + 4 <= l) {
              *reinterpret_cast<F4Loose*>(X) = v;
            } else {
#pragma unroll
              for (int n = 0; n < 4; ++n)
                if (j + n < l) X[n] = v[n];
            }
          }
        }
        *reinterpret_cast<F4*>(here) = v;
      }
      if constexpr (kPhase != kS) wave_sync();
      if constexpr (kPhase == kX) {
        if (last) {
          if (turned) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const int j = jb + row + 8 * k, i = ib + column;
              F4 v;
#pragma unroll
              for (int n = 0; n < 4; ++n) v[n] = corner[(column + n) * kPitch + row + 8 * k];
              if (j < l && i < m) finish4(it, st, (static_cast<int64_t>(matrix) * l + j) * m + i, m - i, v);
            }
          }
        } else {
          put_parts<false, kPitch>(corner, sc.up, m - ib, l - jb, buf.x + it.px + 2 * (matrix * m + ib) * lp, 2 * lp, jb);
          put_parts<true, kPitch>(corner, sc.up, l - jb, m - ib, buf.next + it.pt + 2 * (matrix * l + jb) * mp, 2 * mp, ib);
        }
      } else {
        _Float16* const parts = (kPhase == kS ? buf.s : buf.p) + it.ps;
        put_parts<false, kPitch>(corner, sc.up, m - ib, m - jb, parts + 2 * (matrix * m + ib) * mp, 2 * mp, jb);
        if (mirrored) put_parts<true, kPitch>(corner, sc.up, m - jb, m - ib, parts + 2 * (matrix * m + jb) * mp, 2 * mp, ib);
      }
      wave_sync();
    }
}

}  // namespace

int exponent_of(double top) { return 14 - static_cast<int>(std::ceil(std::log2(std::max(top, kLeastBound)))); }

void parts_place(Part& p, Item& it, int64_t count) {
  const int64_t m = std::min(it.rows, it.cols), l = std::max(it.rows, it.cols);
  it.x = p.x;
  it.px = p.px;
  it.pt = p.pt;
  it.ps = p.ps;
  p.units[kBlocks] += count * ceil_div(m, 64) * ceil_div(l, 64);
  for (const int tile : {128, 64}) {
    const int64_t tm = ceil_div(m, tile), tl = ceil_div(l, tile);
    p.units[tile == 128 ? kGram : kGramSmall] += count * tm * (tm + 1) / 2;
    p.units[tile == 128 ? kProduct : kProductSmall] += count * tm * tl;
  }
  p.x += count * m * l;
  p.x = (p.x + 3) / 4 * 4;
  p.px += 2 * count * m * padded(l);
  p.pt += 2 * count * l * padded(m);
  p.ps += 2 * count * m * padded(m);
}

void parts_layout(Part& p, Room& room, int steps) {
  if (steps == 0) return;
  p.at_x = room(p.x * sizeof(float));
  p.at[0] = room(p.px * sizeof(_Float16));
  p.at[1] = room(p.pt * sizeof(_Float16));
  p.at[2] = room(p.pt * sizeof(_Float16));
  p.at[3] = room(p.ps * sizeof(_Float16));
  p.at[4] = room(p.ps * sizeof(_Float16));
}

namespace {

// Tiles of 128 that leave half of the chip's places for workgroups empty: smaller ones.  A step of one 512 x 512 takes 30 us with the smaller, 66 with the
// larger, 16 of them 64 and 74, 32 of them 116 and 107; one 2048 x 2048 170 and 176, one 4096 x 4096 1136 and 967.
bool few_tiles(int64_t tiles) { return tiles <= kFewTiles; }

template <int kPhase, int kTile, int kStages>
hipError_t launch(const Part& p, const Item* items, const Step& st, bool last, const Buffers& buf, const Scales& sc, hipStream_t stream) {
  constexpr int bytes = Ring<kTile, kStages>::kBytes;
  constexpr Kind kind = kTile == 128 ? (kPhase == kX ? kProduct : kGram) : kPhase == kX ? kProductSmall : kGramSmall;
  const void* const kernel = reinterpret_cast<const void*>(&product_kernel<kPhase, kTile, kStages>);
  if (bytes > 64 * 1024) {
    const hipError_t e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL((product_kernel<kPhase, kTile, kStages>), dim3(static_cast<unsigned>(ceil_div(p.units[kind], kXcds) * kXcds)), dim3(kThreads), bytes, stream,
                     items, static_cast<int>(p.items.size()), st, last, buf, sc, static_cast<int>(p.units[kind]));
  return hipGetLastError();
}

template <int kPhase>
hipError_t launch(const Part& p, const Item* items, const Step& st, bool last, const Buffers& buf, const Scales& sc, hipStream_t stream) {
  return few_tiles(p.units[kPhase == kX ? kProduct : kGram]) ? launch<kPhase, 64, 4>(p, items, st, last, buf, sc, stream)
                                                             : launch<kPhase, 128, 2>(p, items, st, last, buf, sc, stream);
}

}  // namespace

hipError_t parts_run(const Part& p, const ou_config* cfg, const Step& st, char* base, hipStream_t stream) {
  const int n = static_cast<int>(p.items.size());
  const Item* const items = reinterpret_cast<const Item*>(base + p.at_items);
  const double* const partial = reinterpret_cast<const double*>(base + p.at_partial);
  auto halfs = [&](int i) { return reinterpret_cast<_Float16*>(base + p.at[i]); };
  Buffers buf{reinterpret_cast<float*>(base + p.at_x), halfs(0), halfs(1), halfs(2), halfs(3), halfs(4)};
  double top = 1;
  int ex = exponent_of(top);
  hipLaunchKernelGGL(normalise_kernel, dim3(static_cast<unsigned>(p.units[kBlocks])), dim3(kThreads), 0, stream, items, n, st, cfg->steps == 0, buf,
                     std::ldexp(1.f, ex), partial);
  hipError_t e = hipGetLastError();
  for (int i = 0; i < cfg->steps && e == hipSuccess; ++i) {
    const bool last = i + 1 == cfg->steps;
    const double square = top * top;
    const int es = exponent_of(square), ep = exponent_of(std::fabs(cfg->b) * square + std::fabs(cfg->c) * square * square);
    top = growth(cfg, top);
    const int next = exponent_of(top);
    e = launch<kS>(p, items, st, last, buf, Scales{std::ldexp(1.f, es), std::ldexp(1.f, -2 * ex), 0}, stream);
    if (e == hipSuccess) e = launch<kP>(p, items, st, last, buf, Scales{std::ldexp(1.f, ep), std::ldexp(1.f, -2 * es), std::ldexp(1.f, -es)}, stream);
    if (e == hipSuccess) e = launch<kX>(p, items, st, last, buf, Scales{std::ldexp(1.f, next), std::ldexp(1.f, -ep - ex), 0}, stream);
    ex = next;
    std::swap(buf.t, buf.next);
  }
  return e;
}

}  // namespace ou
