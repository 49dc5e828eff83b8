// Element embedding and the gradient of its table (include/ee.h).
//
// Forward: a row copy with a factor, bound by the rows that it writes.
//
// Gradient: dT[z] = scale * sum of the rows of dY with index z.  The rows are read once, which is what bounds it; everything else is there
// to keep the sums in a fixed order without atomics.
//   1. a stable counting sort of the indices, 10 bits a pass (one pass up to 1023 elements, two up to EE_MAX_ELEMENTS): workgroups count their
//      stretches of the batch, then each sums the counts before its own and scatters its stretch;
//   2. the sorted order is cut into pieces of kPiece rows; a wave sums the runs of equal indices of one piece, 64 lanes across the
//      channels.  A run inside one piece is a finished row of dT; one that goes on beyond it leaves its sum in a slot of the
//      piece (slot 0: the run came in from the piece before; slot 1: it starts here and goes on);
//   3. for each element the slots of its pieces are added in order, or its row is zeroed if it is absent.
// Small batches instead look through all indices for each element: one launch.  (Rules and times at search_few_kernel and searched.)
//
// Measured: 200 000 rows of 128 fp32 channels, 89 elements: forward 18.5 us (5.6 TB/s), count 3.5, scatter 9.2, pieces 30 (3.4 TB/s of dY), join 9.8; 32 768 rows of 512
// bfloat16 channels, 50 000 elements: forward 16 us, two sort passes 22, pieces 17, join (102 MB of dT, most of it zeros) 25.  61 rows: 2.5 and 2.7 us.
#include <algorithm>
#include <cmath>
#include <limits>
#include <type_traits>

#include "sc_internal.h"
#include "../../include/ee.h"

namespace ee {
namespace {

using sc::align_up;
using sc::DeviceGuard;
using sc::kLanes;
using sc::misaligned;
using sc::set_error;

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kLanes;
constexpr int kDigitBits = 10;
constexpr int kBins = 1 << kDigitBits;
constexpr int kSortBlocks = 256;     // most workgroups of a sort pass
constexpr int kSortChunk = 1024;     // rows of a workgroup below that
constexpr int kPiece = 32;           // sorted rows a wave sums
constexpr int kAhead = 8;            // rows (or slots) requested at a time

template <typename T, int N>
struct Vec {
  typedef T type __attribute__((ext_vector_type(N), aligned(sizeof(T))));   // wide accesses need element alignment only
};
template <typename T>
struct Vec<T, 1> {
  typedef T type __attribute__((ext_vector_type(1), aligned(sizeof(T))));
};

// ---- forward

// `rows` rows per workgroup, vectors of V channels; magic = 2^32 / per_row rounded up: i / per_row for i below 65536.
template <typename TS, typename TA, int V>
__global__ __launch_bounds__(kThreads) void forward_kernel(int64_t n, int channels, int elements, TA scale, int rows, int per_row,
                                                           unsigned magic, const int* __restrict__ z, const TA* __restrict__ T,
                                                           TS* __restrict__ Y) {
  typedef typename Vec<TA, V>::type VA;
  typedef typename Vec<TS, V>::type VS;
  const int64_t blocks = (n + rows - 1) / rows;
  for (int64_t block = blockIdx.x; block < blocks; block += gridDim.x) {
    const int64_t first = block * rows;
    const int count = static_cast<int>(min(static_cast<int64_t>(rows), n - first)) * per_row;
    constexpr int kEach = 4;   // vectors of a thread at a time
    for (int i0 = threadIdx.x; i0 < count; i0 += kEach * kThreads) {
      int r[kEach], c[kEach], element[kEach];
      VA t[kEach];
#pragma unroll
      for (int e = 0; e < kEach; ++e) {
        const int i = min(i0 + e * kThreads, count - 1);
        r[e] = per_row == 1 ? i : static_cast<int>(__umulhi(static_cast<unsigned>(i), magic));
        c[e] = (i - r[e] * per_row) * V;
        element[e] = z[first + r[e]];
      }
#pragma unroll
      for (int e = 0; e < kEach; ++e)   // an index outside the table reads row 0 and becomes zeros
        t[e] = *reinterpret_cast<const VA*>(T + static_cast<int64_t>(static_cast<unsigned>(element[e]) < static_cast<unsigned>(elements) ? element[e] : 0) *
                                                    channels + c[e]);
#pragma unroll
      for (int e = 0; e < kEach; ++e) {
        const bool inside = static_cast<unsigned>(element[e]) < static_cast<unsigned>(elements);
        VS y;
#pragma unroll
        for (int k = 0; k < V; ++k) y[k] = static_cast<TS>(inside ? scale * t[e][k] : TA(0));
        if (i0 + e * kThreads < count) *reinterpret_cast<VS*>(Y + (first + r[e]) * channels + c[e]) = y;
      }
    }
  }
}

// ---- sort

// The key of a row: its index, or `elements` for one outside the table.
__device__ __forceinline__ int key_of(int z, int elements) {
  return static_cast<unsigned>(z) < static_cast<unsigned>(elements) ? z : elements;
}

struct Sort {
  int64_t n, per_block;   // rows, rows of a workgroup (a multiple of kThreads)
  int elements, shift, bins;
  const int* z;
  const int* order;   // rows in the order of the previous pass, or NULL: 0, 1, 2, ...
};

__device__ __forceinline__ int row_at(const Sort& s, int64_t i) { return s.order ? s.order[i] : static_cast<int>(i); }
__device__ __forceinline__ int digit_of(const Sort& s, int row) { return (key_of(s.z[row], s.elements) >> s.shift) & (kBins - 1); }

// Adds the digits of rows i, i + step, .. below end to bin (whole numbers: any order); four requests at a time.
__device__ __forceinline__ void count_digits(const Sort& s, int64_t i, int64_t end, int step, int* bin) {
  for (; i < end; i += 4 * step) {
    int row[4], digit[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) row[k] = row_at(s, min(i + k * step, end - 1));
#pragma unroll
    for (int k = 0; k < 4; ++k) digit[k] = digit_of(s, row[k]);
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (i + k * step < end) atomicAdd(&bin[digit[k]], 1);
  }
}

// counts[block][bin]; on the way first[element] = -1 (no row yet).
__global__ __launch_bounds__(kThreads) void count_kernel(Sort s, int* __restrict__ counts, int* __restrict__ first) {
  __shared__ int bin[kBins];
  for (int i = threadIdx.x; i < s.bins; i += kThreads) bin[i] = 0;
  __syncthreads();
  const int64_t begin = blockIdx.x * s.per_block, end = min(s.n, begin + s.per_block);
  count_digits(s, begin + threadIdx.x, end, kThreads, bin);
  __syncthreads();
  for (int i = threadIdx.x; i < s.bins; i += kThreads) counts[blockIdx.x * static_cast<int64_t>(s.bins) + i] = bin[i];
  if (first)
    for (int i = blockIdx.x * kThreads + threadIdx.x; i < s.elements; i += gridDim.x * kThreads) first[i] = -1;
}

// Rows to their places: bins in order, inside a bin the order of the pass before.
// keys: of the sorted rows, written by the last pass (else NULL).
__global__ __launch_bounds__(kThreads) void scatter_kernel(Sort s, int blocks, const int* __restrict__ counts, int* __restrict__ out,
                                                           int* __restrict__ keys) {
  __shared__ int place[kWaves][kBins];   // next place of each bin for each wave
  __shared__ int4 all[kThreads], earlier[kThreads];   // of four bins, over a share of the workgroups
  __shared__ int wave_total[kWaves];
  const int lane = threadIdx.x & (kLanes - 1), wave = threadIdx.x / kLanes;
  const int64_t begin = blockIdx.x * s.per_block, end = min(s.n, begin + s.per_block);
  const int64_t per_wave = s.per_block / kWaves;
  const int64_t w0 = min(end, begin + wave * per_wave), w1 = min(end, w0 + per_wave);
  for (int i = threadIdx.x; i < kWaves * kBins; i += kThreads) (&place[0][0])[i] = 0;
  __syncthreads();
  count_digits(s, w0 + lane, w1, kLanes, place[wave]);
  // four bins a thread (the bins are a multiple of four), the workgroups shared by kThreads / width groups of threads
  const int quads = s.bins / 4;
  int width = 1;
  while (width < quads) width *= 2;
  const int group = threadIdx.x / width, quad = threadIdx.x % width, groups = kThreads / width;
  int4 sum = {0, 0, 0, 0}, part = {0, 0, 0, 0};
  if (quad < quads) {
    const int per = (blocks + groups - 1) / groups, b0 = group * per, b1 = min(blocks, b0 + per);
    for (int b = b0; b < b1; b += kAhead) {
      int4 v[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k)
        v[k] = reinterpret_cast<const int4*>(counts + min(b + k, b1 - 1) * static_cast<int64_t>(s.bins))[quad];
#pragma unroll
      for (int k = 0; k < kAhead; ++k)
        if (b + k < b1) {
          sum.x += v[k].x, sum.y += v[k].y, sum.z += v[k].z, sum.w += v[k].w;
          if (b + k < static_cast<int>(blockIdx.x)) part.x += v[k].x, part.y += v[k].y, part.z += v[k].z, part.w += v[k].w;
        }
    }
  }
  all[threadIdx.x] = sum;
  earlier[threadIdx.x] = part;
  __syncthreads();
  // thread t: bins 4 t .. 4 t + 3
  constexpr int kOwn = 4;
  int total[kOwn] = {}, before[kOwn] = {};
  const int b0 = threadIdx.x * kOwn;
  if (b0 < s.bins)
    for (int g = 0; g < groups; ++g) {
      const int4 a = all[g * width + threadIdx.x], e = earlier[g * width + threadIdx.x];
      total[0] += a.x, total[1] += a.y, total[2] += a.z, total[3] += a.w;
      before[0] += e.x, before[1] += e.y, before[2] += e.z, before[3] += e.w;
    }
  const int mine = total[0] + total[1] + total[2] + total[3];
  int up = mine;   // inclusive sum over the lanes
#pragma unroll
  for (int d = 1; d < kLanes; d *= 2) {
    const int v = __shfl_up(up, d);
    if (lane >= d) up += v;
  }
  if (lane == kLanes - 1) wave_total[wave] = up;
  __syncthreads();
  int at = up - mine;
  for (int w = 0; w < wave; ++w) at += wave_total[w];
  if (b0 < s.bins) {
#pragma unroll
    for (int k = 0; k < kOwn; ++k) {
      int next = at + before[k];
      for (int w = 0; w < kWaves; ++w) {
        const int c = place[w][b0 + k];
        place[w][b0 + k] = next;
        next += c;
      }
      at += total[k];
    }
  }
  __syncthreads();
  // 64 rows at a time: a row's rank among the earlier lanes with the same bin, then the first of them moves the bin on
  volatile int* const next = place[wave];
  int row = w0 < w1 ? row_at(s, min(w0 + lane, w1 - 1)) : 0, key = w0 < w1 ? key_of(s.z[row], s.elements) : 0;
  for (int64_t i = w0; i < w1; i += kLanes) {
    const bool live = i + lane < w1;
    const int d = (key >> s.shift) & (kBins - 1);
    int row_next = 0, key_next = 0;
    if (i + kLanes < w1) {
      row_next = row_at(s, min(i + kLanes + lane, w1 - 1));
      key_next = key_of(s.z[row_next], s.elements);
    }
    unsigned long long same = __ballot(live);
#pragma unroll
    for (int bit = 0; bit < kDigitBits; ++bit) {
      const unsigned long long set = __ballot((d >> bit) & 1);
      same &= (d >> bit) & 1 ? set : ~set;
    }
    const unsigned long long below = same & ((1ull << lane) - 1);
    int start = 0;
    if (live) {
      start = next[d];
      out[start + __popcll(below)] = row;
      if (keys) keys[start + __popcll(below)] = key;
    }
    __builtin_amdgcn_wave_barrier();   // every lane has read the place before it moves
    if (live && below == 0) next[d] = start + __popcll(same);
    __builtin_amdgcn_wave_barrier();
    row = row_next;
    key = key_next;
  }
}

// ---- sums

template <typename TS, typename TA, int V>
struct Row {
  typedef typename Vec<TS, V>::type VS;
  typedef typename Vec<TA, V>::type VA;
  static __device__ __forceinline__ void add(TA (&acc)[V], const VS& v) {
#pragma unroll
    for (int k = 0; k < V; ++k) acc[k] += static_cast<TA>(v[k]);
  }
  static __device__ __forceinline__ void store(TA* p, const TA (&acc)[V], TA scale) {
    VA v;
#pragma unroll
    for (int k = 0; k < V; ++k) v[k] = scale * acc[k];
    *reinterpret_cast<VA*>(p) = v;
  }
};

// One piece of the sorted order, 64 V channels, by a wave.  first / last: sorted positions of an element's first and last row.
template <typename TS, typename TA, int V>
__device__ __forceinline__ void sum_piece(int64_t piece, int col_block, int64_t n, int channels, int elements, TA scale, const int* __restrict__ keys,
                                          const int* __restrict__ order, const TS* __restrict__ dY, TA* __restrict__ dT, TA* __restrict__ slots,
                                          int* __restrict__ first, int* __restrict__ last) {
  typedef Row<TS, TA, V> R;
  const int lane = threadIdx.x & (kLanes - 1);
  const int c = (col_block * kLanes + lane) * V;
  const bool live = c < channels;
  const int64_t p0 = piece * kPiece;
  const int count = static_cast<int>(min(static_cast<int64_t>(kPiece), n - p0));
  static_assert(kPiece <= kLanes, "a lane holds the row and the key of one position");
  const int row = lane < count ? order[p0 + lane] : 0;
  const int key = lane < count ? keys[p0 + lane] : -1;
  const int before = p0 > 0 ? keys[p0 - 1] : -1;             // keys of the neighbouring positions
  const int after = p0 + count < n ? keys[p0 + count] : -1;
  const int up = __shfl_up(key, 1), down = __shfl_down(key, 1);   // with all lanes active
  const int left = lane == 0 ? before : up, right = lane == count - 1 ? after : down;
  if (c == lane * V && lane < count && key < elements) {      // the first column block writes the bounds
    if (left != key) first[key] = static_cast<int>(p0) + lane;
    if (right != key) last[key] = static_cast<int>(p0) + lane;
  }
  const unsigned long long ends = __ballot(lane < count && right != key || lane == count - 1);   // last positions of the runs of this piece
  TA acc[V] = {};
  typename R::VS next[kAhead];
  auto request = [&](int i) {
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int r = __builtin_amdgcn_readlane(row, min(i + k, count - 1));
      if (live) next[k] = *reinterpret_cast<const typename R::VS*>(dY + static_cast<int64_t>(r) * channels + c);
    }
  };
  int run_start = 0;
  request(0);
  for (int i = 0; i < count; i += kAhead) {
    typename R::VS v[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) v[k] = next[k];
    if (i + kAhead < count) request(i + kAhead);
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      if (i + k >= count) break;
      if (live) R::add(acc, v[k]);
      if ((ends >> (i + k)) & 1) {
        const int e = __builtin_amdgcn_readlane(key, i + k);
        if (e < elements && live) {
          const bool came_in = run_start == 0 && before == e, goes_on = i + k == count - 1 && after == e;
          if (came_in) R::store(slots + (piece * 2) * channels + c, acc, TA(1));
          else if (goes_on) R::store(slots + (piece * 2 + 1) * channels + c, acc, TA(1));
          else R::store(dT + static_cast<int64_t>(e) * channels + c, acc, scale);
        }
#pragma unroll
        for (int q = 0; q < V; ++q) acc[q] = TA(0);
        run_start = i + k + 1;
      }
    }
  }
}

template <typename TS, typename TA, int V>
__global__ __launch_bounds__(kThreads) void piece_kernel(int64_t n, int64_t pieces, int col_blocks, int channels, int elements, TA scale,
                                                         const int* __restrict__ keys, const int* __restrict__ order,
                                                         const TS* __restrict__ dY, TA* __restrict__ dT, TA* __restrict__ slots,
                                                         int* __restrict__ first, int* __restrict__ last) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kLanes);
  for (int64_t task = blockIdx.x * static_cast<int64_t>(kWaves) + wave; task < pieces * col_blocks; task += gridDim.x * static_cast<int64_t>(kWaves))
    sum_piece<TS, TA, V>(task / col_blocks, static_cast<int>(task % col_blocks), n, channels, elements, scale, keys, order, dY, dT, slots, first, last);
}

// Rows of dT whose rows span pieces, and those of absent elements.  A workgroup has `own` elements: kWaves of a long table, each a wave's, or
// one of a table with fewer elements than the chip has places for workgroups, which then have kJoinWaves.  Spans from kLongSpan pieces on are
// shared by all waves (625 pieces of an element with a tenth of 200 000 rows: 19 us by 4 waves, 10 by 16).
constexpr int kLongSpan = 16;
constexpr int kShortTable = 1024;
constexpr int kJoinWaves = 16;

template <typename TA, int V>
__device__ __forceinline__ void add_slots(const TA* __restrict__ slots, int64_t p0, int64_t from, int64_t to, int channels, int c, TA (&acc)[V]) {
  typedef typename Vec<TA, V>::type VA;
  for (int64_t p = from; p < to; p += kAhead) {
    VA v[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int64_t q = min(p + k, to - 1);
      v[k] = *reinterpret_cast<const VA*>(slots + (q * 2 + (q == p0)) * channels + c);
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
      if (p + k < to)
#pragma unroll
        for (int i = 0; i < V; ++i) acc[i] += v[k][i];
  }
}

template <typename TA, int V, int kW>
__global__ __launch_bounds__(kW * kLanes) void join_kernel(int own, int channels, int elements, TA scale, const TA* __restrict__ slots,
                                                        const int* __restrict__ first, const int* __restrict__ last, TA* __restrict__ dT) {
  typedef Row<TA, TA, V> R;
  __shared__ TA part[kW][kLanes * V];
  const int lane = threadIdx.x & (kLanes - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kLanes);
  for (int64_t e0 = static_cast<int64_t>(blockIdx.x) * own; e0 < elements; e0 += static_cast<int64_t>(gridDim.x) * own) {
    for (int w = 0; w < own; ++w) {
      const int64_t e = e0 + w;
      if (e >= elements) break;
      const int a = first[e];
      const int64_t p0 = a / kPiece, p1 = a < 0 ? 0 : last[e] / kPiece;
      if (a >= 0 && p0 == p1) continue;                       // summed inside one piece
      const bool is_long = a >= 0 && p1 - p0 >= kLongSpan;    // the same for all waves
      if (!is_long && w != wave) continue;
      for (int c0 = 0; c0 < channels; c0 += kLanes * V) {
        const int c = c0 + lane * V;
        TA acc[V] = {};
        if (!is_long) {
          if (c < channels) {
            if (a >= 0) add_slots<TA, V>(slots, p0, p0, p1 + 1, channels, c, acc);
            R::store(dT + e * channels + c, acc, a >= 0 ? scale : TA(0));
          }
        } else {
          const int64_t per = (p1 + 1 - p0 + kW - 1) / kW, from = min(p1 + 1, p0 + wave * per), to = min(p1 + 1, from + per);
          if (c < channels) add_slots<TA, V>(slots, p0, from, to, channels, c, acc);
          __syncthreads();
#pragma unroll
          for (int k = 0; k < V; ++k) part[wave][lane * V + k] = acc[k];
          __syncthreads();
          if (wave == 0 && c < channels) {
            for (int v = 1; v < kW; ++v)
#pragma unroll
              for (int k = 0; k < V; ++k) acc[k] += part[v][lane * V + k];
            R::store(dT + e * channels + c, acc, scale);
          }
        }
      }
    }
  }
}

// Adds the rows list[from], .. list[to - 1], not none, in order, a batch of kAhead requested while the one before is added.
template <typename TS, typename TA, int V>
__device__ __forceinline__ void add_rows(const unsigned short* list, int from, int to, const TS* __restrict__ dY, int channels, int c, TA (&acc)[V]) {
  typedef Row<TS, TA, V> R;
  typename R::VS next[kAhead];
  auto request = [&](int i) {
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
      next[k] = *reinterpret_cast<const typename R::VS*>(dY + static_cast<int64_t>(list[min(i + k, to - 1)]) * channels + c);
  };
  request(from);
  for (int i = from; i < to; i += kAhead) {
    typename R::VS v[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) v[k] = next[k];
    if (i + kAhead < to) request(i + kAhead);
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
      if (i + k < to) R::add(acc, v[k]);
  }
}

// Small batches, by search: a wave looks through all indices for the rows of its element.  A workgroup has kWaves elements.
//
// Up to kFewRows rows: the wave adds what it finds among 64 indices, kAhead at a time.  (One at a time 0.14 us a row, 19 us for 128 rows of one element; so 10.)
constexpr int kFewRows = 128;

template <typename TS, typename TA, int V>
__global__ __launch_bounds__(kThreads) void search_few_kernel(int n, int channels, int elements, TA scale, const int* __restrict__ z,
                                                              const TS* __restrict__ dY, TA* __restrict__ dT) {
  typedef Row<TS, TA, V> R;
  const int lane = threadIdx.x & (kLanes - 1), element = blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x / kLanes);
  if (element >= elements) return;
  const int c = (blockIdx.y * kLanes + lane) * V;
  TA acc[V] = {};
  for (int i = 0; i < n; i += kLanes) {
    unsigned long long hits = __ballot(i + lane < n && z[min(i + lane, n - 1)] == element);
    while (hits) {
      const int count = __popcll(hits);
      int row = 0;
      typename R::VS v[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {   // beyond the last one that one again
        if (hits) row = i + __builtin_ctzll(hits);
        hits &= hits - 1;
        if (c < channels) v[k] = *reinterpret_cast<const typename R::VS*>(dY + static_cast<int64_t>(row) * channels + c);
      }
#pragma unroll
      for (int k = 0; k < kAhead; ++k)
        if (k < count && c < channels) R::add(acc, v[k]);
    }
  }
  if (c < channels) R::store(dT + static_cast<int64_t>(element) * channels + c, acc, scale);
}

// Up to kSearchRows rows: the wave lists them first.  Up to kLongList of them it adds itself; of an element with more every wave of the workgroup adds a
// share, joined in order.  (1024 rows of one element by one wave, one after the other, 148 us; so 16, and sorted 24.)  x of the grid: elements; y: col_step blocks of
// 64 V channels.
constexpr int kSearchRows = 1024;
constexpr int kLongList = 32;
constexpr int kManyGroups = 4096;   // workgroups of elements

template <typename TS, typename TA, int V>
__global__ __launch_bounds__(kThreads) void search_kernel(int n, int col_blocks, int col_step, int channels, int elements, TA scale,
                                                          const int* __restrict__ z, const TS* __restrict__ dY, TA* __restrict__ dT) {
  typedef Row<TS, TA, V> R;
  __shared__ unsigned short list[kWaves][kSearchRows];
  __shared__ int4 found;
  __shared__ TA part[kWaves][kLanes * V];
  static_assert(kWaves == 4, "a component of `found` for each wave");
  const int lane = threadIdx.x & (kLanes - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kLanes);
  const int first = blockIdx.x * kWaves, element = first + wave;   // (beyond the table: no row has that index)
  const int cb0 = blockIdx.y * col_step, cb1 = min(col_blocks, cb0 + col_step);
  int count = 0;
  for (int i = 0; i < n; i += kLanes) {
    const bool hit = i + lane < n && element < elements && z[min(i + lane, n - 1)] == element;
    const unsigned long long hits = __ballot(hit);
    if (hit) list[wave][count + __popcll(hits & ((1ull << lane) - 1))] = static_cast<unsigned short>(i + lane);
    count += __popcll(hits);
  }
  if (lane == 0) reinterpret_cast<int*>(&found)[wave] = count;
  __syncthreads();
  if (element < elements && count <= kLongList)
    for (int cb = cb0; cb < cb1; ++cb) {
      const int c = (cb * kLanes + lane) * V;
      if (c >= channels) break;
      TA acc[V] = {};
      if (count > 0) add_rows<TS, TA, V>(list[wave], 0, count, dY, channels, c, acc);
      R::store(dT + static_cast<int64_t>(element) * channels + c, acc, scale);
    }
  const int4 all = found;
  if (max(max(all.x, all.y), max(all.z, all.w)) <= kLongList) return;   // the same for all waves
  for (int w = 0; w < kWaves; ++w) {
    const int rows = w == 0 ? all.x : w == 1 ? all.y : w == 2 ? all.z : all.w;
    if (rows <= kLongList) continue;
    const int per = (rows + kWaves - 1) / kWaves, from = min(rows, wave * per), to = min(rows, from + per);
    for (int cb = cb0; cb < cb1; ++cb) {
      const int c = (cb * kLanes + lane) * V;
      TA acc[V] = {};
      if (c < channels && from < to) add_rows<TS, TA, V>(list[w], from, to, dY, channels, c, acc);
#pragma unroll
      for (int k = 0; k < V; ++k) part[wave][lane * V + k] = acc[k];
      __syncthreads();
      if (wave == 0 && c < channels) {
        for (int v = 1; v < kWaves; ++v)
#pragma unroll
          for (int k = 0; k < V; ++k) acc[k] += part[v][lane * V + k];
        R::store(dT + static_cast<int64_t>(first + w) * channels + c, acc, scale);
      }
      __syncthreads();   // part is the next block's
    }
  }
}

// ---- host side

size_t row_size(const ee_config* c) { return c->dtype == SC_F64 ? 8 : c->dtype == SC_F32 ? 4 : 2; }
size_t table_size(const ee_config* c) { return c->dtype == SC_F64 ? 8 : 4; }

sc_status check_config(const char* fn, const ee_config* cfg, int64_t n) {
  auto bad = [&](sc_status st, const char* what) { return set_error(st, std::string(fn) + ": " + what); };
  if (!cfg) return bad(SC_ERR_INVALID_ARG, "cfg is NULL");
  if (cfg->struct_size != static_cast<int32_t>(sizeof(ee_config)))
    return bad(SC_ERR_INVALID_ARG, "struct_size does not match this library's ee_config");
  if (cfg->num_elements < 1 || cfg->num_channels < 1) return bad(SC_ERR_INVALID_ARG, "num_elements or num_channels < 1");
  if (cfg->num_elements > EE_MAX_ELEMENTS || cfg->num_channels > EE_MAX_CHANNELS)
    return bad(SC_ERR_UNSUPPORTED, "num_elements above EE_MAX_ELEMENTS or num_channels above EE_MAX_CHANNELS");
  if (cfg->dtype != SC_F32 && cfg->dtype != SC_F64 && cfg->dtype != SC_BF16) return bad(SC_ERR_INVALID_ARG, "bad dtype");
  if (!std::isfinite(cfg->scale)) return bad(SC_ERR_INVALID_ARG, "scale not finite");
  if (cfg->dtype != SC_F64 && std::fabs(cfg->scale) > std::numeric_limits<float>::max()) return bad(SC_ERR_INVALID_ARG, "scale beyond fp32");
  if (n < 0 || n > (int64_t(1) << 30)) return bad(SC_ERR_INVALID_ARG, "n_nodes outside 0..2^30");
  return SC_OK;
}

// Does the search take a batch?  It is one launch instead of four, for long tables six, and no slower than those however the rows are spread over the elements
// (search, sort; 128 and 512 channels): 64 rows of one element 6 and 6 us, 18 and 20; 1024 rows of one element 15 and 20, 24 and 28, of 10 elements 12 and 15, 18 and 22, of
// 10 000 elements 9 and 17, 34 and 39, of 65 536 39 and 49, 62 and 68, of one of those 39 and 50, 60 and 65; 67 rows of a million elements of 4 channels 84 and 517.
bool searched(const ee_config* c, int64_t n) { return n <= kSearchRows && n * c->num_elements <= 1 << 26; }

int64_t sort_rows_per_block(int64_t n) {
  const int64_t per = std::max<int64_t>(kSortChunk, (n + kSortBlocks - 1) / kSortBlocks);
  return (per + kThreads - 1) / kThreads * kThreads;
}
int sort_passes(const ee_config* c) { return c->num_elements < kBins ? 1 : 2; }
int sort_bins(const ee_config* c, int pass) {
  const int keys = c->num_elements + 1;
  const int bins = sort_passes(c) == 1 ? keys : pass == 0 ? kBins : (keys - 1) / kBins + 1;
  return (bins + 3) / 4 * 4;
}

struct Workspace {
  int *order, *order0, *keys, *counts, *first, *last;
  void* slots;
  size_t bytes;
};

Workspace carve(const ee_config* c, int64_t n, void* base) {
  Workspace w{};
  size_t at = 0;
  auto take = [&](size_t bytes) {
    void* p = static_cast<char*>(base) + at;
    at += align_up(bytes, 256);
    return p;
  };
  if (!searched(c, n)) {
    const int64_t blocks = (n + sort_rows_per_block(n) - 1) / sort_rows_per_block(n);
    w.order = static_cast<int*>(take(n * 4));
    w.order0 = sort_passes(c) == 2 ? static_cast<int*>(take(n * 4)) : nullptr;
    w.keys = static_cast<int*>(take(n * 4));
    w.counts = static_cast<int*>(take(blocks * kBins * 4));
    w.first = static_cast<int*>(take(static_cast<size_t>(c->num_elements) * 4));
    w.last = static_cast<int*>(take(static_cast<size_t>(c->num_elements) * 4));
    w.slots = take(static_cast<size_t>((n + kPiece - 1) / kPiece) * 2 * c->num_channels * table_size(c));
  }
  w.bytes = at + 256;
  return w;
}

// Workgroups for so many waves' tasks.  A launch has fewer than 2^32 threads: beyond 2^22 workgroups a wave takes several tasks.
unsigned blocks_of(int64_t waves) { return static_cast<unsigned>(std::min<int64_t>((waves + kWaves - 1) / kWaves, 1 << 22)); }

template <typename TS, typename TA>
struct Calls {
  const ee_config* c;
  int64_t n;
  hipStream_t stream;

  template <int V>
  hipError_t forward_v(const int32_t* z, const void* T, void* Y) const {
    const int per_row = c->num_channels / V;
    const int rows = std::min<int64_t>(std::max(1, 2048 / per_row), std::max<int64_t>(1, n));
    const unsigned magic = per_row == 1 ? 0 : static_cast<unsigned>(((uint64_t(1) << 32) + per_row - 1) / per_row);
    const int64_t blocks = std::min<int64_t>((n + rows - 1) / rows, 1 << 20);
    hipLaunchKernelGGL((forward_kernel<TS, TA, V>), dim3(static_cast<unsigned>(blocks)), dim3(kThreads), 0, stream, n, c->num_channels,
                       c->num_elements, static_cast<TA>(c->scale), rows, per_row, magic, z, static_cast<const TA*>(T),
                       static_cast<TS*>(Y));
    return hipGetLastError();
  }

  hipError_t forward(const int32_t* z, const void* T, void* Y) const {
    if (c->num_channels % 4 == 0) return forward_v<4>(z, T, Y);
    return c->num_channels % 2 == 0 ? forward_v<2>(z, T, Y) : forward_v<1>(z, T, Y);
  }

  hipError_t sort(const int32_t* z, const Workspace& w) const {
    Sort s{n, sort_rows_per_block(n), c->num_elements, 0, 0, z, nullptr};
    const int blocks = static_cast<int>((n + s.per_block - 1) / s.per_block);
    const int passes = sort_passes(c);
    for (int pass = 0; pass < passes; ++pass) {
      s.shift = pass * kDigitBits;
      s.bins = sort_bins(c, pass);
      s.order = pass == 0 ? nullptr : w.order0;
      hipLaunchKernelGGL(count_kernel, dim3(blocks), dim3(kThreads), 0, stream, s, w.counts, pass == 0 ? w.first : nullptr);
      hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
      hipLaunchKernelGGL(scatter_kernel, dim3(blocks), dim3(kThreads), 0, stream, s, blocks, w.counts, pass + 1 < passes ? w.order0 : w.order,
                         pass + 1 < passes ? nullptr : w.keys);
      e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    return hipSuccess;
  }

  template <int V>
  hipError_t backward_v(const int32_t* z, const void* dY, void* dT, void* ws) const {
    const int k = c->num_channels, elements = c->num_elements;
    const int col_blocks = (k + kLanes * V - 1) / (kLanes * V);
    const TA scale = static_cast<TA>(c->scale);
    if (searched(c, n)) {
      const int groups = (elements + kWaves - 1) / kWaves;
      if (n <= kFewRows) {
        hipLaunchKernelGGL((search_few_kernel<TS, TA, V>), dim3(groups, col_blocks), dim3(kThreads), 0, stream, static_cast<int>(n), k, elements, scale, z,
                           static_cast<const TS*>(dY), static_cast<TA*>(dT));
        return hipGetLastError();
      }
      // A workgroup does one block of channels, or all where the elements alone make more workgroups than the chip holds: the indices are looked through
      // once (1024 rows of 65 536 elements, 512 channels, 92 us and 49).
      const int col_step = groups >= kManyGroups ? col_blocks : 1;
      hipLaunchKernelGGL((search_kernel<TS, TA, V>), dim3(groups, (col_blocks + col_step - 1) / col_step), dim3(kThreads), 0, stream, static_cast<int>(n),
                         col_blocks, col_step, k, elements, scale, z, static_cast<const TS*>(dY), static_cast<TA*>(dT));
      return hipGetLastError();
    }
    const Workspace w = carve(c, n, ws);
    hipError_t e = sort(z, w);
    if (e != hipSuccess) return e;
    const int64_t pieces = (n + kPiece - 1) / kPiece;
    hipLaunchKernelGGL((piece_kernel<TS, TA, V>), dim3(blocks_of(pieces * col_blocks)), dim3(kThreads), 0, stream, n, pieces, col_blocks, k,
                       elements, scale, w.keys, w.order, static_cast<const TS*>(dY), static_cast<TA*>(dT), static_cast<TA*>(w.slots), w.first,
                       w.last);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    auto join = [&](auto waves, int own) {
      hipLaunchKernelGGL((join_kernel<TA, V, waves.value>), dim3((elements + own - 1) / own), dim3(waves.value * kLanes), 0, stream, own, k, elements,
                         scale, static_cast<const TA*>(w.slots), w.first, w.last, static_cast<TA*>(dT));
    };
    if (elements <= kShortTable) join(std::integral_constant<int, kJoinWaves>{}, 1);
    else join(std::integral_constant<int, kWaves>{}, kWaves);
    return hipGetLastError();
  }

  // channels of a lane: as many as leave no lane idle, four at most
  hipError_t backward(const int32_t* z, const void* dY, void* dT, void* ws) const {
    const int k = c->num_channels;
    if (k % 4 == 0 && k >= 4 * kLanes) return backward_v<4>(z, dY, dT, ws);
    if (k % 2 == 0 && k >= 2 * kLanes) return backward_v<2>(z, dY, dT, ws);
    return backward_v<1>(z, dY, dT, ws);
  }
};

__global__ void zero_kernel(unsigned* __restrict__ p, int64_t words) {
  for (int64_t i = blockIdx.x * static_cast<int64_t>(kThreads) + threadIdx.x; i < words; i += static_cast<int64_t>(gridDim.x) * kThreads) p[i] = 0;
}

template <typename F>
hipError_t by_type(const ee_config* c, int64_t n, hipStream_t stream, F&& f) {
  switch (c->dtype) {
    case SC_F64: return f(Calls<double, double>{c, n, stream});
    case SC_BF16: return f(Calls<__bf16, float>{c, n, stream});
    default: return f(Calls<float, float>{c, n, stream});
  }
}

}  // namespace
}  // namespace ee

extern "C" {

sc_status ee_forward(const ee_config* cfg, int64_t n_nodes, const int32_t* z, const void* T, void* Y, void* hip_stream) {
  using namespace ee;
  const sc_status st = check_config("ee_forward", cfg, n_nodes);
  if (st != SC_OK || n_nodes == 0) return st;
  if (!z || !T || !Y) return set_error(SC_ERR_INVALID_ARG, "ee_forward: NULL tensor argument");
  if (misaligned(z, 16) || misaligned(T, 16) || misaligned(Y, 16))
    return set_error(SC_ERR_INVALID_ARG, "ee_forward: tensor pointer not 16-byte aligned");
  DeviceGuard guard(cfg->device);
  if (!guard.ok) return set_error(SC_ERR_HIP, "ee_forward: cannot make cfg->device current");
  const hipError_t e = by_type(cfg, n_nodes, static_cast<hipStream_t>(hip_stream), [&](const auto& calls) { return calls.forward(z, T, Y); });
  if (e != hipSuccess) return set_error(SC_ERR_HIP, std::string("ee_forward: kernel launch: ") + hipGetErrorString(e));
  return SC_OK;
}

sc_status ee_workspace_bytes(const ee_config* cfg, int64_t n_nodes, size_t* bytes) {
  using namespace ee;
  const sc_status st = check_config("ee_workspace_bytes", cfg, n_nodes);
  if (st != SC_OK) return st;
  if (!bytes) return set_error(SC_ERR_INVALID_ARG, "ee_workspace_bytes: bytes is NULL");
  *bytes = n_nodes == 0 ? 256 : carve(cfg, n_nodes, nullptr).bytes;
  return SC_OK;
}

sc_status ee_backward(const ee_config* cfg, int64_t n_nodes, const int32_t* z, const void* dY, void* dT, void* workspace,
                      size_t workspace_bytes, void* hip_stream) {
  using namespace ee;
  const sc_status st = check_config("ee_backward", cfg, n_nodes);
  if (st != SC_OK) return st;
  if (!dT) return set_error(SC_ERR_INVALID_ARG, "ee_backward: dT is NULL");
  if (misaligned(z, 16) || misaligned(dY, 16) || misaligned(dT, 16))
    return set_error(SC_ERR_INVALID_ARG, "ee_backward: tensor pointer not 16-byte aligned");
  if (n_nodes > 0) {
    if (!z || !dY) return set_error(SC_ERR_INVALID_ARG, "ee_backward: NULL tensor argument");
    if (!workspace || workspace_bytes < carve(cfg, n_nodes, nullptr).bytes)
      return set_error(SC_ERR_WORKSPACE, "ee_backward: workspace missing or smaller than ee_workspace_bytes()");
    if (misaligned(workspace, 256)) return set_error(SC_ERR_WORKSPACE, "ee_backward: workspace not 256-byte aligned");
  }
  DeviceGuard guard(cfg->device);
  if (!guard.ok) return set_error(SC_ERR_HIP, "ee_backward: cannot make cfg->device current");
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  hipError_t e;
  if (n_nodes == 0) {
    const int64_t words = static_cast<int64_t>(cfg->num_elements) * cfg->num_channels * (table_size(cfg) / 4);
    hipLaunchKernelGGL(zero_kernel, dim3(static_cast<unsigned>(std::min<int64_t>((words + kThreads - 1) / kThreads, 2048))), dim3(kThreads), 0,
                       stream, static_cast<unsigned*>(dT), words);
    e = hipGetLastError();
  } else {
    e = by_type(cfg, n_nodes, stream, [&](const auto& calls) { return calls.backward(z, dY, dT, workspace); });
  }
  if (e != hipSuccess) return set_error(SC_ERR_HIP, std::string("ee_backward: kernel launch: ") + hipGetErrorString(e));
  return SC_OK;
}

}  // extern "C"
