// How the dense layer's work is cut: what launches, workspace and kernels agree on.
#pragma once
#include <algorithm>

#include "dl_parts.h"

namespace dl {

using sc::align_up;

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

// Workgroups that share rows, `shared` of them for each of `groups` groups of rows.  All of a group go to one XCD (workgroups are dealt out to the
// XCDs in turn), whose L2 then holds the rows - where the groups come out even to a quarter.  Where they are few the XCDs take them as they come
// (250 rows, 1024 -> 1024: all of one group on one XCD 104 us for dX, 16 on all).
struct Deal {
  int64_t groups, shared;
  __host__ __device__ int64_t rounded() const { return (groups + kXcds - 1) / kXcds * kXcds; }
  __host__ __device__ bool by_xcd() const { return 4 * rounded() <= 5 * groups; }
  __host__ __device__ int64_t count() const { return (by_xcd() ? rounded() : groups) * shared; }
  __device__ bool at(int64_t t, int64_t* group, int64_t* i) const {
    const bool even = by_xcd();
    const int64_t local = even ? t / kXcds : t;
    *group = even ? local / shared * kXcds + t % kXcds : local / shared;
    *i = local % shared;
    return *group < groups;
  }
};

// Row groups x column groups of workgroups.
struct Walk {
  int64_t row_groups;
  int col_groups;
  __host__ __device__ Deal deal() const { return {row_groups, col_groups}; }
  __host__ __device__ int64_t count() const { return deal().count(); }
  __device__ bool at(int64_t t, int64_t* row, int* col) const {
    int64_t i;
    const bool inside = deal().at(t, row, &i);
    *col = static_cast<int>(i);
    return inside;
  }
};

constexpr int kPartsTiles = 4;   // row tiles of a wave, where there are rows enough (parts_tiles)

// Which results a call wants.
struct Wanted {
  bool dx, dw, db;
};

// What a launch of the backward does: the rows in chunks, of each chunk first dx_groups workgroups of dX, then dw_groups of the chunk's partial dW and
// db.  A chunk stays on one XCD and its two halves run at about the same time: the second reading of dY (and Z) comes from the caches.
struct Plan {
  int64_t rows, per;    // per: rows of a chunk, a multiple of 64
  int64_t chunks;
  int64_t dx_groups, dw_groups;   // workgroups of a chunk
  int dx_col_groups, dw_col_groups;
  Shape dx, dw;
  int64_t n_dw, n_db;   // elements of dW and of db that a chunk's partial results hold, dW first: 0 for one that is not wanted
  __host__ __device__ int64_t stride() const { return n_dw + n_db; }
  __host__ __device__ Deal deal() const { return {chunks, dx_groups + dw_groups}; }
};

// ---- host side

inline size_t row_size(const dl_config* c) { return c->dtype == SC_F64 ? 8 : c->dtype == SC_F32 ? 4 : 2; }
inline size_t weight_size(const dl_config* c) { return c->dtype == SC_F64 ? 8 : 4; }
inline int64_t ld_in(const dl_config* c) { return c->ld_in ? c->ld_in : c->k_in; }
inline int64_t ld_out(const dl_config* c) { return c->ld_out ? c->ld_out : c->k_out; }

inline int64_t blocks_of(int64_t n, int64_t size) { return (n + size - 1) / size; }

// Waves side by side along the columns: as many as there are column blocks, up to four.
inline Shape shape_of(int cols) {
  const int64_t blocks = blocks_of(cols, kCols);
  return blocks >= 3 ? Shape{4, 1} : blocks == 2 ? Shape{2, 2} : Shape{1, 4};
}

// Row tiles of a wave: the fewer the rows the fewer, so that there are two waves for every SIMD of 256 CUs as long as possible.
inline int row_tiles(int64_t rows, int cols, int most) {
  const int64_t waves = blocks_of(rows, 16) * blocks_of(cols, kCols);
  int rt = 1;
  while (rt < most && waves / (2 * rt) >= 2048) rt *= 2;
  return rt;
}

// Do all waves of a workgroup share one tile?  Where there is at most one row tile for every SIMD and the sum is long (a wave a tile -> shared: forward of
// 200 rows, 256 -> 64 fp32 15.2 -> 7.7 us, 100 rows, 1024 -> 1024 44 -> 13.5; 10 000 rows, 128 -> 16 fp64 16.7 -> 14.6).
inline bool split_sum(int64_t rows, int cols, int k) { return k >= 128 && blocks_of(rows, 16) * blocks_of(cols, kCols) <= 1024; }

inline void set_partials(const dl_config* c, const Wanted& want, Plan* p) {
  p->n_dw = want.dw ? static_cast<int64_t>(c->k_in) * c->k_out : 0;
  p->n_db = want.db ? c->k_out : 0;
}
// db without dW takes the blocks of the first 64 rows of dW only, in more chunks: as many as find room where the partial dW of this plan would be.
inline int64_t room_for_db(const dl_config* c, const Plan& with_dw) { return with_dw.chunks > 1 ? with_dw.chunks * (c->k_in + 1) : 1; }

inline Plan plan_of(const dl_config* c, int64_t n, const Wanted& want, bool split, int rt) {
  const int split_waves = c->dtype == SC_F64 ? dl::split_waves<double>() : dl::split_waves<float>();
  Plan p{};
  p.rows = n;
  p.dw = shape_of(c->k_out);
  if (split) p.dw = {1, split_waves};
  const bool only_db = want.db && !want.dw;
  const int64_t dw_rows = only_db ? 1 : blocks_of(c->k_in, kCols), blocks = dw_rows * blocks_of(c->k_out, kCols);
  constexpr int kMinShare = 16;
  // about 2048 waves of dW, none with less than 16 rows (1000 rows, 256 -> 256 in fp32: dW 21 us so, 28 with 32; 10 000, 128 -> 16 in fp64: 22, 25)
  int64_t chunks = std::max<int64_t>(1, std::min(2048 / (blocks * p.dw.wr), n / (kMinShare * p.dw.wr)));
  if (only_db) chunks = std::min(chunks, room_for_db(c, plan_of(c, n, {want.dx, true, true}, split, rt)));
  p.per = blocks_of(n, chunks);
  p.per = blocks_of(p.per, p.per < 256 ? 64 : 256) * (p.per < 256 ? 64 : 256);
  p.chunks = blocks_of(n, p.per);
  p.dx = split ? Shape{1, 1} : shape_of(c->k_in);
  p.dx_col_groups = static_cast<int>(blocks_of(c->k_in, kCols * p.dx.wc));
  p.dx_groups = want.dx ? blocks_of(p.per, split ? 16 : 16 * rt * p.dx.wr) * p.dx_col_groups : 0;
  p.dw_col_groups = static_cast<int>(blocks_of(c->k_out, kCols * p.dw.wc));
  p.dw_groups = want.dw || want.db ? dw_rows * p.dw_col_groups : 0;
  set_partials(c, want, &p);
  return p;
}

inline bool curved(const dl_config* c) { return c->activation == DL_SILU || c->activation == DL_GELU; }

// Do the bfloat16 matrix cores serve a product of rows (dl_parts.h)?  From 1024 blocks of 64 x 64 results on, and where the sum is long and there is a
// block for every second CU; of the forward, whose launch does nothing else, on fp32 rows a block for every CU.  (dX, dW and db together, GELU, fp32
// instruction -> parts, us.  bfloat16 rows: 512 rows, 1024 -> 1024 59 -> 66, 640 rows 75 -> 65, 1000 rows 102 -> 78, 2100 rows 245 -> 103, 8000 rows, 128 -> 128
// 40 -> 23, 6000 rows, 128 -> 1240 127 -> 75; fp32 rows: 512 rows, 1024 -> 1024 57 -> 65, 640 rows 69 -> 66, 1280 rows 142 -> 81, 2000 rows, 512 -> 512 72 -> 45,
// 8000 rows, 128 -> 128 41 -> 26.  Shorter sums: 25 000 rows, 64 -> 64, second order 41 -> 56.)
constexpr int64_t kFewBlocks = 128;
constexpr int kLongSum = 128;
inline bool in_parts(const dl_config* c, int64_t n, int cols, int k, int64_t few = kFewBlocks) {
  // (the lanes' places in 64 rows are 32-bit byte offsets)
  if (ld_in(c) > (1 << 22) || ld_out(c) > (1 << 22)) return false;
  if (c->dtype == SC_F64 || c->k_in % 4 != 0 || c->k_out % 4 != 0 || k <= 16 || (c->dtype == SC_BF16 && k % 8 != 0)) return false;
  const int64_t blocks = blocks_of(n, 64) * blocks_of(cols, kCols);
  return blocks >= 1024 || (blocks >= few && k >= kLongSum);
}

// Row tiles of a wave: one where four would leave CUs without a workgroup (2100 rows, 1024 -> 1024, dX 90 us with four, 83 with one; forward 86, 59).
inline int parts_tiles(int64_t n, int cols) { return blocks_of(n, 64) * blocks_of(cols, kCols) >= 1024 ? kPartsTiles : 1; }

// Do the waves keep W (walk_rows)?  Its parts of up to 64 reduced indices fit the registers.
inline bool kept_ok(const dl_config* c, int64_t n, int cols, int k) { return k <= 2 * kRound && in_parts(c, n, cols, k); }

// Is a wave's share of dW 64 x 64 (parts_dw_role)?
inline bool wide_parts(const dl_config* c) { return c->k_out > 2 * kCols; }

inline Plan parts_plan(const dl_config* c, int64_t n, const Wanted& want) {
  Plan p{};
  p.rows = n;
  const bool wide = wide_parts(c);
  p.dw = {wide ? kWaves : 1, 1};
  p.dw_col_groups = static_cast<int>(blocks_of(c->k_out, kCols * p.dw.wc));
  const bool only_db = want.db && !want.dw;
  const int64_t groups = (only_db ? 1 : blocks_of(c->k_in, kCols)) * p.dw_col_groups;
  // Of dW alone as many workgroups as the chip has places for, two a CU (64 x 64 blocks: three) and the same for every XCD: one more would run when
  // the others are done.  None with less than 256 rows.  (990 001 rows, 64 -> 1280: 65 workgroups on an XCD with 64 places 1640 us, 60 1190.)  Wider layers
  // a chunk for every XCD; where one chunk has workgroups for all places, the fewest chunks that leave a quarter of the places idle at most, as every chunk writes a
  // dW that is read again (2048 rows, 4096 -> 4096 bfloat16, dW 464 us with eight, 135 with one; 8192 rows, 4096 -> 2560, 513 and 404 with two).
  const int64_t places = wide ? 64 : 96, all = places * kXcds;
  int64_t chunks = kXcds;
  if (groups <= places) {
    chunks = places / groups * kXcds;
  } else if (groups >= all) {
    chunks = 1;
    while (chunks < kXcds && 4 * chunks * groups < 3 * all * blocks_of(chunks * groups, all)) ++chunks;
  }
  const int rt = parts_tiles(n, c->k_in);
  chunks = std::max<int64_t>(1, std::min<int64_t>(chunks, n / (rt == 1 ? 128 : 256)));
  // With dX beside it no more than 4 MB of dY, so that what the workgroups of the chip read twice at a time stays in the caches: 990 001 rows of
  // bfloat16, 64 -> 1280, 1325 us with 26 MB, 1120 with 10, 1017 with 4.  But no chunk of less than four times as many rows as dW has, or the partial results
  // would outweigh dY (dX and dW of 16 384 rows, 4096 -> 4096 bfloat16, 3560 us and 2.2 GB of workspace with 32 chunks, 2685 and 0.13 with one; 60 000 rows,
  // 1280 -> 1280, 1211 with 37, 1109 with 11).
  if (want.dx && want.dw)
    chunks = std::max(chunks, std::min(blocks_of(n * c->k_out * static_cast<int64_t>(row_size(c)), 4 << 20), n / (4 * static_cast<int64_t>(c->k_in))));
  if (only_db) chunks = std::min(chunks, room_for_db(c, parts_plan(c, n, {want.dx, true, true})));
  const int64_t unit = want.dx ? 16 * rt * kWaves : 32;
  p.per = blocks_of(blocks_of(n, chunks), unit) * unit;
  p.chunks = blocks_of(n, p.per);
  p.dx = {1, kWaves};
  p.dx_col_groups = static_cast<int>(blocks_of(c->k_in, kCols));
  p.dx_groups = want.dx ? blocks_of(p.per, 16 * rt * kWaves) * p.dx_col_groups : 0;
  p.dw_groups = want.dw || want.db ? groups : 0;
  set_partials(c, want, &p);
  return p;
}

// Is G made first?  It would be made again for every column block of dX, which then takes longer than its writing and reading; in fp64, whose
// exponential is some sixty instructions of half the rate, always but for the smallest batches (10 000 rows, 128 -> 16, dX, dW and db together 33 us so and 39
// without, second order 46 and 56; dX alone 3 us more).
inline bool g_first(const dl_config* c, int64_t n) {
  if (c->activation == DL_NONE) return false;
  return c->dtype == SC_F64 ? n >= 1024 : c->k_in > kCols && in_parts(c, n, c->k_in, c->k_out);
}

// Workspace: [ S of the second-order pass, or G of the backward ][ G of the second-order pass ][ W transposed ][ partial dW and db per chunk ].
inline size_t s_bytes(const dl_config* c, int64_t n) {
  return curved(c) || g_first(c, n) ? align_up(static_cast<size_t>(n) * c->k_out * weight_size(c), 256) : 0;
}

// Does dX take W transposed (a launch of its own, 2 us)?  Where the reading of W as it is, four times the accesses, would take longer:
// beyond the batches of a single round (3000 rows, 64 -> 64 fp32: dX 9.4 us without, 12.5 with).
inline bool transposed(int64_t n, const dl_config* c) { return n >= 4096 || in_parts(c, n, c->k_in, c->k_out); }

inline size_t wt_bytes(int64_t n, const dl_config* c) {
  return transposed(n, c) ? align_up(static_cast<size_t>(c->k_in) * c->k_out * weight_size(c), 256) : 0;
}

// Partial results: none where a single chunk writes the outputs themselves.
inline size_t partial_bytes(const dl_config* c, int64_t n) {
  int64_t most = 0;
  for (bool dx : {false, true}) {
    const Wanted want{dx, true, true};
    const Plan p = in_parts(c, n, c->k_in, c->k_out) ? parts_plan(c, n, want) : plan_of(c, n, want, split_sum(n, c->k_in, c->k_out), 1);
    if (p.chunks > 1) most = std::max(most, p.chunks * p.stride());
  }
  return static_cast<size_t>(most) * weight_size(c);
}

inline size_t workspace_bytes(const dl_config* c, int64_t n) {
  if (n == 0) return 256;
  return (curved(c) && g_first(c, n) ? 2 : 1) * s_bytes(c, n) + wt_bytes(n, c) + align_up(partial_bytes(c, n), 256) + 256;
}


// The calls of one type (dl_calls.h).  c and the tensors have been checked.
struct Entries {
  hipError_t (*forward)(const dl_config* c, int64_t n, hipStream_t stream, const void* X, const void* W, const void* b, const void* residual, void* Y,
                        void* Z);
  hipError_t (*backward)(const dl_config* c, int64_t n, hipStream_t stream, const void* X, const void* W, const void* Z, const void* dY, void* dX,
                         void* dW, void* db, void* ws);
  hipError_t (*double_backward)(const dl_config* c, int64_t n, hipStream_t stream, const void* X, const void* W, const void* Z, const void* dY,
                                const void* HX, void* ddY, void* X2, void* W2, void* b2, void* ws);
  hipError_t (*zero)(const dl_config* c, hipStream_t stream, void* dW, void* db);
};
Entries entries_f32();
Entries entries_f64();
Entries entries_bf16();

}  // namespace dl
