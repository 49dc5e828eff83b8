// The products of dl_product.h on the bfloat16 matrix cores, every fp32 value as the sum of bfloat16 parts (el::split_pair: h + m + l, exact from
// 2^-110 on).  A 16x16x32 instruction occupies the matrix core for 16 cycles, eight 16x16x4 ones for 256, so even six products of parts
// take three eighths of the time.
//
//   fp32 rows       h h + (h m + m h + m m + h l + l h): what is left out is below 2^-24 of |x w|.  An instruction cuts its smaller products off at
//                   the last bit of the largest and of the sum it adds to, so the five small products are summed by themselves and join
//                   the sum of h h once per 32 reduced indices.
//   bfloat16 rows   an element of them is one part; W, G = dY act' and S = V dY act'' are fp32 values and keep their three.  Results that are rounded to
//                   bfloat16 and nothing else, of rows that are one part, take the three products into one sum, smallest first: two more
//                   cuts at its last bit per 32 reduced indices (990 001 rows, 64 -> 1280, forward 815 us with two sums, 685 with one).
//
// G and S hold derivatives of the activations, which fall to nothing far out: a GELU layer whose pre-activations have a deviation of 2 has some below
// 2^-110 in every tile.  Their parts are those of 2^16 times the value, which stand for every fp32 number below 2^111, and the sums are divided by 2^16
// at the end.
//
// A lane holds 8 consecutive reduced indices k = 8 q .. 8 q + 7 of index j.  Values that the parts do not stand for (not finite, beyond the largest
// bfloat16, not zero and below 2^-110) are noted by the wave that meets them, which then computes its tile with the products of
// dl_product.h.
#pragma once
#include "dl_product.h"

namespace dl {

using el::Bf8;
using el::pack_bf16;
using el::split_pair;
using el::SplitPair;
typedef unsigned U4 __attribute__((ext_vector_type(4)));
typedef unsigned U2 __attribute__((ext_vector_type(2)));
typedef Mma<float>::acc_t Acc;

constexpr int kRound = 32;   // reduced indices per round

// What an operand's values are multiplied by.
template <Source kSource>
constexpr float kScale = kSource == kPlain ? 1.f : 65536.f;
// Sums of such an operand's parts to sums of its values.  done: false for those that were made without parts.
template <Source kSource, int kR, int kC>
__device__ __forceinline__ void unscale(Acc (&acc)[kR][kC], bool done) {
  if constexpr (kScale<kSource> != 1.f) {
    const float down = done ? 1 / kScale<kSource> : 1.f;
#pragma unroll
    for (int i = 0; i < kR; ++i)
#pragma unroll
      for (int t = 0; t < kC; ++t) acc[i][t] *= down;
  }
}

__device__ __forceinline__ Acc mma_parts(const U4& a, const U4& b, const Acc& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(Bf8, a), __builtin_bit_cast(Bf8, b), c, 0, 0, 0);
}

// Adds a(i) b(i) to sum[i], i = 0..3: the products of the first parts to sum, the others to small (kOneSum: all to sum, the smallest first).
// Product by product over the four, as each instruction waits for the one before it on the same sum.
template <int NA, int NB, bool kOneSum, typename A, typename B>
__device__ __forceinline__ void multiply4(A&& a, B&& b, Acc (&sum)[4], Acc (&small)[4]) {
#pragma unroll
  for (int order = NA + NB - 2; order > 0; --order)
#pragma unroll
    for (int p = NA - 1; p >= 0; --p)
      if (order - p >= 0 && order - p < NB && order < (NA > NB ? NA : NB)) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          Acc& to = kOneSum ? sum[i] : small[i];
          to = mma_parts(a(i)[p], b(i)[order - p], to);
        }
      }
#pragma unroll
  for (int i = 0; i < 4; ++i) sum[i] = mma_parts(a(i)[0], b(i)[0], sum[i]);
}
template <bool kOneSum>
__device__ __forceinline__ void join4(Acc (&sum)[4], const Acc (&small)[4]) {
  if constexpr (!kOneSum) {
#pragma unroll
    for (int i = 0; i < 4; ++i) sum[i] += small[i];
  }
}

// dY act'(z), rounded to fp32 as a value of its own: contracted with the subtraction of its first part it would be one with more bits than three
// parts hold.
__device__ __forceinline__ float gated(const Gate<float>& gate, float x, float z) {
#pragma clang fp contract(off)
  const float g = x * gate.first(z);
  return g;
}

// Pairs of values into three parts, in the halves of a register each.  low: collects what the last part is rounded from (el::split_pair).
template <Source kSource>
__device__ __forceinline__ void split(float x, float y, unsigned (&part)[3], unsigned& low) {
  const SplitPair s = split_pair(x * kScale<kSource>, y * kScale<kSource>, low);
  part[0] = s.h, part[1] = s.m, part[2] = s.l;
}

// Rows as an operand: 16 rows x 32 reduced indices in kParts planes of the wave's corner of LDS (16 rows of 64 bytes each, the four pieces of a
// row at places that differ between groups of four rows).
template <typename T, Source kSource, int kParts>
struct PartsRows;

constexpr int kPlane = 256;   // 32-bit words of a plane
__device__ __forceinline__ int piece_at(int row, int piece) { return 16 * row + 4 * (piece ^ (row / 4)); }

// Four or eight elements at (row0 + r) of a tensor, columns k + c .. of k_end: row0 and k are the same for the wave.  Beyond the end of the row the
// address is that of its last elements.
template <typename V, typename T>
__device__ __forceinline__ V load_piece(const Matrix<T>& m, int64_t row0, int r, int k, int c, int k_end) {
  constexpr int kN = sizeof(V) / sizeof(T);
  typedef V Loose __attribute__((aligned(sizeof(T))));
  unsigned lane = static_cast<unsigned>(r) * static_cast<unsigned>(m.ld) + c;
  int64_t base = row0 * m.ld + k;
  if (k + kRound > k_end) {   // the last round: what is left may end inside it
    lane += min(k + c, k_end - kN) - c;
    base = row0 * m.ld;
  }
  return *reinterpret_cast<const Loose*>(at(m.p, Spot{base, lane}));
}

template <Source kSource, int kParts>
struct PartsRows<float, kSource, kParts> {
  static constexpr Source source = kSource;
  Operand<float, float, kSource> from;
  typedef float F4 __attribute__((ext_vector_type(4)));
  struct Raw {
    F4 v[2], z[kSource == kGated ? 2 : 1];   // rows 0..7 and 8..15: lane 8 row + piece of four elements
  };
  static __device__ __forceinline__ int column() { return 4 * (threadIdx.x % 8); }
  __device__ __forceinline__ void request(int64_t start, int left, int k, int k_end, Raw& raw, int first) const {   // rows start + first on, of those that are left from start on
    const int lane = threadIdx.x & (kLanes - 1);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int r = min(first + 8 * h + lane / 8, left - 1);
      raw.v[h] = load_piece<F4>(from.x, start, r, k, column(), k_end);
      if constexpr (kSource == kGated) raw.z[h] = load_piece<F4>(from.z, start, r, k, column(), k_end);
    }
  }
  __device__ __forceinline__ void put(Raw& raw, int k, int k_end, unsigned* planes, unsigned& low) const {
    const int lane = threadIdx.x & (kLanes - 1);
    if (k + kRound > k_end) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
        if (k + column() >= k_end) raw.v[h] = F4{0, 0, 0, 0};
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      F4 v = raw.v[h];
      if constexpr (kSource == kGated) {
        const bool inside = k + column() < k_end;   // (0 times what stands beyond the end may be a NaN)
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = inside ? gated(from.gate, v[i], raw.z[h][i]) : 0.f;
      }
      unsigned a[kParts], b[kParts];
      split<kSource>(v[0], v[1], a, low);
      split<kSource>(v[2], v[3], b, low);
      const int to = piece_at(8 * h + lane / 8, lane % 8 / 2) + 2 * (lane & 1);
#pragma unroll
      for (int p = 0; p < kParts; ++p) *reinterpret_cast<U2*>(planes + p * kPlane + to) = U2{a[p], b[p]};
    }
  }
};

template <Source kSource, int kParts>
struct PartsRows<__bf16, kSource, kParts> {
  static_assert(kSource != kPlain || kParts == 1, "an element is one part");
  static constexpr Source source = kSource;
  Operand<float, __bf16, kSource> from;
  struct Raw {
    U4 v, z;   // lane 4 row + piece of eight elements
  };
  static __device__ __forceinline__ int column() { return 8 * (threadIdx.x % 4); }
  __device__ __forceinline__ void request(int64_t start, int left, int k, int k_end, Raw& raw, int first) const {
    const int r = min(first + static_cast<int>(threadIdx.x & (kLanes - 1)) / 4, left - 1);
    raw.v = load_piece<U4>(from.x, start, r, k, column(), k_end);
    if constexpr (kSource == kGated) raw.z = load_piece<U4>(from.z, start, r, k, column(), k_end);
  }
  __device__ __forceinline__ void put(Raw& raw, int k, int k_end, unsigned* planes, unsigned& low) const {
    const int lane = threadIdx.x & (kLanes - 1);
    const bool inside = k + column() < k_end;
    U4 part[kParts];
    if constexpr (kSource == kPlain) {
      if (k + kRound > k_end && !inside) raw.v = U4{0, 0, 0, 0};
      part[0] = raw.v;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float x = gated(from.gate, el::low_half(raw.v[i]), el::low_half(raw.z[i]));
        const float y = gated(from.gate, el::high_half(raw.v[i]), el::high_half(raw.z[i]));
        unsigned s[kParts];
        split<kSource>(inside ? x : 0.f, inside ? y : 0.f, s, low);
#pragma unroll
        for (int p = 0; p < kParts; ++p) part[p][i] = s[p];
      }
    }
#pragma unroll
    for (int p = 0; p < kParts; ++p) *reinterpret_cast<U4*>(planes + p * kPlane + piece_at(lane / 4, lane % 4)) = part[p];
  }
};

// A round's operand of 16 rows from the planes.
template <int kParts>
__device__ __forceinline__ void get_parts(const unsigned* planes, U4 (&x)[kParts]) {
  const int lane = threadIdx.x & (kLanes - 1);
#pragma unroll
  for (int p = 0; p < kParts; ++p) x[p] = *reinterpret_cast<const U4*>(planes + p * kPlane + piece_at(lane & 15, lane / 16));
}

// 32 rows x 64 columns of a matrix whose columns are not reduced (W [k][n], and both operands of dW) as an operand: tile u holds columns
// c0 + 4 j + u.  Of the rows k + 8 q + i a lane requests kCount from kFirst on.
template <typename T, Source kSource, int kCount>
struct ColumnsRaw {
  typename Vec4<T>::type v[kCount], z[kSource == kGated ? kCount : 1];

  __device__ __forceinline__ void request(const Operand<float, T, kSource>& from, int first, int64_t k, int64_t k_end, int c0, int c_end) {
    const int lane = threadIdx.x & (kLanes - 1), q8 = 8 * (lane / 16);
    const int c = min(c0 + 4 * (lane & 15), c_end - 4);
    const unsigned ld = static_cast<unsigned>(from.x.ld);
    if (k + kRound <= k_end) {
#pragma unroll
      for (int i = 0; i < kCount; ++i) get(from, i, Spot{(k + first + i) * from.x.ld, q8 * ld + c});
    } else {   // rows beyond the last: the last one again
      const int left = static_cast<int>(k_end - k);
#pragma unroll
      for (int i = 0; i < kCount; ++i) get(from, i, Spot{k * from.x.ld, static_cast<unsigned>(min(q8 + first + i, left - 1)) * ld + c});
    }
  }
  __device__ __forceinline__ void get(const Operand<float, T, kSource>& from, int i, const Spot& spot) {
    v[i] = *reinterpret_cast<const typename Vec4<T>::type*>(at(from.x.p, spot));
    if constexpr (kSource == kGated) z[i] = *reinterpret_cast<const typename Vec4<T>::type*>(at(from.z.p, spot));
  }
  // what lies beyond the ends: zero (and act'(0) beside it)
  __device__ __forceinline__ void clear_outside(int first, int64_t k, int64_t k_end, int c0, int c_end) {
    if (k + kRound <= k_end && c0 + kCols <= c_end) return;
    const int lane = threadIdx.x & (kLanes - 1);
#pragma unroll
    for (int i = 0; i < kCount; ++i)
      if (c0 + 4 * (lane & 15) >= c_end || k + 8 * (lane / 16) + first + i >= k_end) {
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          v[i][u] = T(0.f);
          if constexpr (kSource == kGated) z[i][u] = T(0.f);
        }
      }
  }
  // the parts of rows first + i and first + i + 1 of tile u
  template <int kParts, bool kSum>
  __device__ __forceinline__ void pair(const Operand<float, T, kSource>& from, int i, int u, unsigned (&s)[kParts], float& sum, unsigned& low) const {
    if constexpr (sizeof(T) == 2 && kSource == kPlain) {
      static_assert(kParts == 1, "an element is one part");
      const U2 a = __builtin_bit_cast(U2, v[i]), b = __builtin_bit_cast(U2, v[i + 1]);
      s[0] = __builtin_amdgcn_perm(b[u / 2], a[u / 2], u & 1 ? 0x07060302 : 0x05040100);
      if constexpr (kSum) sum += static_cast<float>(v[i][u]) + static_cast<float>(v[i + 1][u]);
    } else {
      float a = static_cast<float>(v[i][u]), b = static_cast<float>(v[i + 1][u]);
      if constexpr (kSource == kGated) {
        a = gated(from.gate, a, static_cast<float>(z[i][u]));
        b = gated(from.gate, b, static_cast<float>(z[i + 1][u]));
      }
      if constexpr (kSum) sum += a + b;
      split<kSource>(a, b, s, low);
    }
  }
};

template <typename T, Source kSource, int kParts>
struct PartsColumns {
  Operand<float, T, kSource> from;
  typedef ColumnsRaw<T, kSource, 8> Raw;
  __device__ __forceinline__ void request(int64_t k, int64_t k_end, int c0, int c_end, Raw& raw) const { raw.request(from, 0, k, k_end, c0, c_end); }
  __device__ __forceinline__ void clear_outside(int64_t k, int64_t k_end, int c0, int c_end, Raw& raw) const {
    raw.clear_outside(0, k, k_end, c0, c_end);
  }
  // tile u's operand; sum: adds the column's values
  template <bool kSum>
  __device__ __forceinline__ void operand(const Raw& raw, int u, U4 (&part)[kParts], float& sum, unsigned& low) const {
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      unsigned s[kParts];
      raw.template pair<kParts, kSum>(from, i, u, s, sum, low);
#pragma unroll
      for (int p = 0; p < kParts; ++p) part[p][i / 2] = s[p];
    }
  }
};

// Did the wave meet a value that the parts do not stand for?  One that is not finite leaves a NaN in the sums.
template <int kR, int kC>
__device__ __forceinline__ bool unserved(const Acc (&acc)[kR][kC], unsigned low) {
  float mark = 0;
#pragma unroll
  for (int i = 0; i < kR; ++i)
#pragma unroll
    for (int t = 0; t < kC; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) mark = fmaf(acc[i][t][r], 0.f, mark);
  return __builtin_amdgcn_ballot_w64((low & 0xffffu) != 0 || mark != 0.f) != 0;   // mark is 0 or NaN
}

// 32 x 64 of an operand that all four waves of a workgroup use, as the instruction takes it: [part][tile u][lane][8 values] in LDS, two slots.  Wave
// w makes the pairs of rows 2 w, 2 w + 1 of each eight.
constexpr int kSharedPart = 4 * kLanes * 4;   // 32-bit words of a part
template <int kParts>
__host__ __device__ constexpr int shared_words() { return 2 * kParts * kSharedPart; }

template <typename T, Source kSource, int kParts>
struct SharedColumns {
  Operand<float, T, kSource> from;
  typedef ColumnsRaw<T, kSource, 2> Raw;
  __device__ __forceinline__ void request(int wave, int64_t k, int64_t k_end, int c0, int c_end, Raw& raw) const {
    raw.request(from, 2 * wave, k, k_end, c0, c_end);
  }
  // sum: adds the columns' values
  template <bool kSum>
  __device__ __forceinline__ void put(int wave, Raw& raw, int64_t k, int64_t k_end, int c0, int c_end, unsigned* slot, float (&sum)[4],
                                      unsigned& low) const {
    const int lane = threadIdx.x & (kLanes - 1);
    raw.clear_outside(2 * wave, k, k_end, c0, c_end);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      unsigned s[kParts];
      raw.template pair<kParts, kSum>(from, 0, u, s, sum[u], low);
#pragma unroll
      for (int p = 0; p < kParts; ++p) slot[((p * 4 + u) * kLanes + lane) * 4 + wave] = s[p];
    }
  }
};

template <int kParts>
__device__ __forceinline__ void get_shared(const unsigned* slot, int u, U4 (&part)[kParts]) {
  const int lane = threadIdx.x & (kLanes - 1);
#pragma unroll
  for (int p = 0; p < kParts; ++p) part[p] = *reinterpret_cast<const U4*>(slot + ((p * 4 + u) * kLanes + lane) * 4);
}

// Is there a wave of the workgroup that met a value the parts do not stand for?  flag: a word of LDS per wave.
__device__ __forceinline__ bool any_wave(bool mine, unsigned* flag) {
  const int wave = threadIdx.x / kLanes;
  __syncthreads();
  flag[wave] = mine;
  __syncthreads();
  bool any = false;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) any = any || flag[w] != 0;
  __syncthreads();
  return any;
}

// rows_product on parts: acc[rt][u] of 16 kRT rows from row0 and the 64 columns from n0 that the workgroup's four waves share, over all reduced
// indices.  planes: kRT * kX planes of this wave; shared: shared_words<kW>() of the workgroup.  All waves come here, the rows of some may lie
// beyond the last.  false for all waves: a value that the parts do not stand for.
template <int kRT, int kX, int kW, bool kOneSum, typename Rows, typename Weights>
__device__ __forceinline__ bool rows_parts(const Rows& a, const Weights& w, int64_t row0, int64_t rows, int n0, int n_end, int k_end,
                                           unsigned* planes, unsigned* shared, Acc (&acc)[kRT][4]) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kLanes);
#pragma unroll
  for (int i = 0; i < kRT; ++i)
#pragma unroll
    for (int t = 0; t < 4; ++t) acc[i][t] = Acc{0, 0, 0, 0};
  typename Rows::Raw raw[kRT];
  typename Weights::Raw next;
  unsigned low = 0;
  float none[4];
  const int64_t start = min(row0, rows - 1);   // (all rows beyond the last: the last one again)
  const int left = static_cast<int>(min(rows - start, static_cast<int64_t>(16 * kRT)));
  auto request_rows = [&](int k) {
#pragma unroll
    for (int i = 0; i < kRT; ++i) a.request(start, left, k, k_end, raw[i], 16 * i);
  };
  w.request(wave, 0, k_end, n0, n_end, next);
  request_rows(0);
  int at = 0;
  for (int k = 0; k < k_end; k += kRound, at ^= kW * kSharedPart) {
    w.template put<false>(wave, next, k, k_end, n0, n_end, shared + at, none, low);
    if (k + kRound < k_end) w.request(wave, k + kRound, k_end, n0, n_end, next);
#pragma unroll
    for (int i = 0; i < kRT; ++i) a.put(raw[i], k, k_end, planes + i * kX * kPlane, low);
    if (k + kRound < k_end) request_rows(k + kRound);
    // (one barrier a round: a wave that runs ahead writes the other slot)
    __syncthreads();
    U4 x[kRT][kX];
#pragma unroll
    for (int i = 0; i < kRT; ++i) get_parts<kX>(planes + i * kX * kPlane, x[i]);
    static_assert(kRT == 4 || kRT == 1, "four sums at a time");
    if constexpr (kRT == 4) {
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        U4 c[kW];
        get_shared<kW>(shared + at, u, c);
        Acc sum[4] = {acc[0][u], acc[1][u], acc[2][u], acc[3][u]}, small[4] = {};
        multiply4<kX, kW, kOneSum>([&](int i) -> const U4(&)[kX] { return x[i]; }, [&](int) -> const U4(&)[kW] { return c; }, sum, small);
        join4<kOneSum>(sum, small);
#pragma unroll
        for (int i = 0; i < kRT; ++i) acc[i][u] = sum[i];
      }
    } else {
      U4 c[4][kW];
#pragma unroll
      for (int u = 0; u < 4; ++u) get_shared<kW>(shared + at, u, c[u]);
      Acc small[4] = {};
      multiply4<kX, kW, kOneSum>([&](int) -> const U4(&)[kX] { return x[0]; }, [&](int u) -> const U4(&)[kW] { return c[u]; }, acc[0], small);
      join4<kOneSum>(acc[0], small);
    }
    Corner<float>::sync();
  }
  return !any_wave(unserved<kRT, 4>(acc, low), shared);
}

// outer_product on parts: acc[t][u] of the wave's 64 columns from n0 and the 64 rows from m0 of dW that the four waves share.
template <int kA, int kB, bool kSum, typename A, typename B>
__device__ __forceinline__ bool outer_parts(const A& a, const B& b, int m0, int m_end, int n0, int n_end, int64_t from, int64_t to,
                                            unsigned* shared, Acc (&acc)[4][4], float (&sum)[4]) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kLanes);
  typename A::Raw ra;
  typename B::Raw rb;
  unsigned low = 0;
  float none[4];
  if (from < to) {
    a.request(wave, from, to, m0, m_end, ra);
    b.request(from, to, n0, n_end, rb);
  }
  int at = 0;
  for (int64_t row = from; row < to; row += kRound, at ^= kA * kSharedPart) {
    a.template put<false>(wave, ra, row, to, m0, m_end, shared + at, none, low);
    if (row + kRound < to) a.request(wave, row + kRound, to, m0, m_end, ra);
    U4 g[4][kB];
    b.clear_outside(row, to, n0, n_end, rb);
#pragma unroll
    for (int u = 0; u < 4; ++u) b.template operand<kSum>(rb, u, g[u], sum[u], low);
    if (row + kRound < to) b.request(row + kRound, to, n0, n_end, rb);
    __syncthreads();
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      U4 x[kA];
      get_shared<kA>(shared + at, t, x);
      Acc small[4] = {};
      multiply4<kA, kB, kA == 1 && kB == 1>([&](int) -> const U4(&)[kA] { return x; }, [&](int u) -> const U4(&)[kB] { return g[u]; }, acc[t], small);
      join4<kA == 1 && kB == 1>(acc[t], small);
    }
  }
  return !any_wave(unserved<4, 4>(acc, low), shared);
}

// The same of one 64 x 64 block by the whole workgroup, both operands shared: wave w computes the rows m0 + 4 j + w, acc[u].  For blocks that the memory
// bounds: a quarter of the registers, so there are twice as many waves to wait for it.  sum: the shares of the wave's pairs of rows.
template <int kA, int kB, typename A, typename B>
__device__ __forceinline__ bool block_parts(const A& a, const B& b, int m0, int m_end, int n0, int n_end, int64_t from, int64_t to,
                                            unsigned* shared_a, unsigned* shared_b, Acc (&acc)[1][4], float (&sum)[4]) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kLanes);
  typename A::Raw ra;
  typename B::Raw rb;
  unsigned low = 0;
  float none[4];
  auto request = [&](int64_t row) {
    a.request(wave, row, to, m0, m_end, ra);
    b.request(wave, row, to, n0, n_end, rb);
  };
  if (from < to) request(from);
  int slot = 0;
  for (int64_t row = from; row < to; row += kRound, slot ^= 1) {
    unsigned* const sa = shared_a + slot * kA * kSharedPart;
    unsigned* const sb = shared_b + slot * kB * kSharedPart;
    a.template put<false>(wave, ra, row, to, m0, m_end, sa, none, low);
    b.template put<true>(wave, rb, row, to, n0, n_end, sb, sum, low);
    if (row + kRound < to) request(row + kRound);
    __syncthreads();
    U4 x[kA];
    get_shared<kA>(sa, wave, x);
    U4 g[4][kB];
#pragma unroll
    for (int u = 0; u < 4; ++u) get_shared<kB>(sb, u, g[u]);
    Acc small[4] = {};
    multiply4<kA, kB, kA == 1 && kB == 1>([&](int) -> const U4(&)[kA] { return x; }, [&](int u) -> const U4(&)[kB] { return g[u]; }, acc[0], small);
    join4<kA == 1 && kB == 1>(acc[0], small);
  }
  return !any_wave(unserved<1, 4>(acc, low), shared_a);
}

// The same operand of a matrix [n_end][k_end] whose second index is reduced (W in dX).
template <int kParts>
struct PartsTransposed {
  Matrix<float> from;
  struct Raw {
    float v[4][2][4];   // row c0 + 4 j + u, columns k + 8 q + 4 h + e
  };
  __device__ __forceinline__ void request(int64_t k, int64_t k_end, int c0, int c_end, Raw& raw) const {
    const int lane = threadIdx.x & (kLanes - 1);
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h)
        load4<true>(from.p + (min(c0 + 4 * (lane & 15), c_end - 4) + u) * from.ld, static_cast<int>(k) + 8 * (lane / 16) + 4 * h,
                    static_cast<int>(k_end), raw.v[u][h]);
  }
  __device__ __forceinline__ void clear_outside(int64_t k, int64_t k_end, int, int, Raw& raw) const {
    const int64_t k0 = k + 8 * ((threadIdx.x & (kLanes - 1)) / 16);
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h) zero_unless(k0 + 4 * h < k_end, raw.v[u][h]);
  }
  template <bool kSum>
  __device__ __forceinline__ void operand(const Raw& raw, int u, U4 (&part)[kParts], float&, unsigned& low) const {
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      unsigned s[kParts];
      split<kPlain>(raw.v[u][i / 4][i % 4], raw.v[u][i / 4][i % 4 + 1], s, low);
#pragma unroll
      for (int p = 0; p < kParts; ++p) part[p][i / 2] = s[p];
    }
  }
};

// ---- products with a matrix of at most 64 reduced indices: a wave keeps its 64 columns of it in registers and walks over the rows

template <int kRounds, int kW>
struct Kept {
  U4 c[kRounds][4][kW];
  bool served;   // the parts stand for every value of the wave's columns
};

template <int kRounds, int kW, typename Weights>
__device__ __forceinline__ void keep(const Weights& w, int n0, int n_end, int k_end, Kept<kRounds, kW>& kept) {
  unsigned low = 0;
  float none = 0, mark = 0;
#pragma unroll
  for (int r = 0; r < kRounds; ++r) {
    typename Weights::Raw raw;
    w.request(r * kRound, k_end, n0, n_end, raw);
    w.clear_outside(r * kRound, k_end, 0, kCols, raw);   // (of the reduced indices; lanes beyond the last column hold its four again)
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      w.template operand<false>(raw, u, kept.c[r][u], none, low);
#pragma unroll
      for (int i = 0; i < 4; ++i)   // not finite (or beyond the largest bfloat16): 0 times the first part is a NaN
        mark = fmaf(el::low_half(kept.c[r][u][0][i]), 0.f, fmaf(el::high_half(kept.c[r][u][0][i]), 0.f, mark));
    }
  }
  kept.served = __builtin_amdgcn_ballot_w64((low & 0xffffu) != 0 || mark != 0.f) == 0;
}

// The row tiles of a wave, kWc at a time: finish(row, column, results, beside) for the rows of each.  kWc waves stand side by side along the columns and
// share their rows: each puts the parts of one of the kWc tiles into LDS (two slots where they share: one barrier a turn, a wave that runs ahead
// writes the other slot).  The rows of the next turn, and what the epilogue reads of the next tile, are requested before the present ones are
// computed.  first: the group's first tile, step: from turn to turn, turns: the same for all waves of the workgroup; own: the wave's place among
// the kWc.  again: the product of a tile that the parts do not serve.
template <int kWc, int kRounds, int kX, int kW, bool kOneSum, typename Rows, typename T, int N, typename Again, typename F>
__device__ __forceinline__ void walk_rows(const Rows& a, const Kept<kRounds, kW>& kept, int64_t first, int64_t step, int64_t turns, int own, int64_t rows,
                                          int n0, int n_end, int k_end, unsigned* planes, unsigned* flags, const Beside<T, N>& beside, Again&& again,
                                          F&& finish) {
  constexpr int kTile = kRounds * kX * kPlane;   // words of a tile's planes
  constexpr int M = N > 0 ? N : 1;
  const int lane = threadIdx.x & (kLanes - 1), c = n0 + 4 * (lane & 15);
  typename Rows::Raw raw[kRounds];
  typename Vec4<T>::type next[M][4];
  auto request = [&](int64_t tile) {
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
      const int64_t row0 = min(16 * tile, rows - 1);
      a.request(row0, static_cast<int>(min(rows - row0, static_cast<int64_t>(16))), r * kRound, k_end, raw[r], 0);
    }
  };
  auto request_beside = [&](int64_t tile) {
#pragma unroll
    for (int e = 0; e < N; ++e)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int64_t row = min(16 * tile + r, rows - 1);
          const unsigned lr = static_cast<unsigned>(min(static_cast<int64_t>(lane_row<float>()), rows - 1 - row));
          next[e][r] = *reinterpret_cast<const typename Vec4<T>::type*>(
              at(beside.m[e].p, Spot{row * beside.m[e].ld, lr * static_cast<unsigned>(beside.m[e].ld) + min(c, n_end - 4)}));
        }
  };
  request(first + own);
  request_beside(first);
  int slot = 0;
  // The last turn alone can meet rows beyond the last.  In the others nothing is written conditionally: where a store may be left out, the next
  // request's arrival is only known once all stores are done.
  auto turn = [&](auto last, auto live) {   // live: the wave has columns
    constexpr bool kLast = decltype(last)::value;
    unsigned* const here = planes + slot * kWc * kTile;
    unsigned low = 0;
#pragma unroll
    for (int r = 0; r < kRounds; ++r) a.put(raw[r], r * kRound, k_end, here + own * kTile + r * kX * kPlane, low);
    if constexpr (kWc > 1) {
      const bool missed = __builtin_amdgcn_ballot_w64((low & 0xffffu) != 0) != 0;
      if (lane == 0) flags[slot * kWc + own] = missed;
    }
    if constexpr (!kLast) request(first + step + own);
    if constexpr (kWc > 1) __syncthreads();
    else Corner<float>::sync();
    if constexpr (!decltype(live)::value) return;
#pragma unroll
    for (int i = 0; i < kWc; ++i) {
      const int64_t tile = first + i;
      Acc acc[1][4], small[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) acc[0][u] = small[u] = Acc{0, 0, 0, 0};
#pragma unroll
      for (int r = 0; r < kRounds; ++r) {
        U4 x[kX];
        get_parts<kX>(here + i * kTile + r * kX * kPlane, x);
        multiply4<kX, kW, kOneSum>([&](int) -> const U4(&)[kX] { return x; }, [&](int u) -> const U4(&)[kW] { return kept.c[r][u]; }, acc[0], small);
      }
      join4<kOneSum>(acc[0], small);
      if constexpr (kWc > 1) low = flags[slot * kWc + i];
      // (all four tiles: a row that is not finite shows in each of them, a product beyond the largest number in its own only)
      const bool served = kept.served && !unserved<1, 4>(acc, low);
      float x[4][M][4];
#pragma unroll
      for (int e = 0; e < N; ++e)
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int k = 0; k < 4; ++k) x[r][e][k] = static_cast<float>(next[e][r][k]);
      if (!kLast || i + 1 < kWc) request_beside(i + 1 < kWc ? tile + 1 : first + step);
      if (!served && 16 * tile < rows) again(16 * tile, acc);
      unscale<Rows::source>(acc, served);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int64_t row = 16 * tile + r;
        const int lr = lane_row<float>();
        const float v[4] = {acc[0][0][r], acc[0][1][r], acc[0][2][r], acc[0][3][r]};
        if (!kLast || row + lr < rows) finish(row, lr, min(c, n_end - 4), v, x[r]);   // lanes beyond the last column repeat its four
      }
    }
    if constexpr (kWc == 1) Corner<float>::sync();
  };
  auto all = [&](auto live) {
    for (int64_t t = 1; t < turns; ++t, first += step, slot = kWc > 1 ? slot ^ 1 : 0) turn(std::false_type{}, live);
    turn(std::true_type{}, live);
  };
  if (kWc == 1 || n0 < n_end) all(std::true_type{});
  else if constexpr (kWc > 1) all(std::false_type{});
}

}  // namespace dl
