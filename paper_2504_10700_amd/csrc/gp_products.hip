// The products by element of include/gp.h: arguments, entry points, and the kernels that serve every width and type (gp_parts.hip: fp32 and
// bfloat16 on the bfloat16 matrix cores; gp_few.hip: the rows of batches without a grouping).
//
// Rows (Y, dX): a workgroup computes 64 rows of one bucket x 64 columns; the rows are gathered by the grouping's order, the reduced index goes
// through LDS 16 at a time.  dW: a workgroup computes 64 x 64 of one element's matrix over a chunk of the element's rows; elements with several chunks leave
// partial matrices that a second launch adds in order.  fp64, 60 000 rows, 10 elements, 128 x 128: Y 64 us, dX 61, dW 81 with the chunks' sums, where the products at the
// rate of a large one are 31 and the memory 26: a stage is 16 reduced indices in loads of an element each, and one stage is requested ahead.
#include <algorithm>
#include <cmath>
#include <initializer_list>
#include <string>

#include "gp_blocks.h"

namespace gp {
namespace {

using sc::DeviceGuard;
using sc::misaligned;
using sc::set_error;

template <typename T, typename TA, bool kBack>
__global__ __launch_bounds__(kThreads) void rows_kernel(const Rows a) {
  __shared__ BlockSpace<TA> space;
  const int columns = (a.columns + kBlock - 1) / kBlock;
  for (int64_t block = blockIdx.x;; block += gridDim.x) {
    int which;
    const Place p = place_of(a.group.offsets, a.elements + 1, a.n, block, columns, [&](int atoms) { return (atoms * a.components + kBlock - 1) / kBlock; }, &which);
    if (p.bucket < 0) return;
    rows_block<T, TA, kBack>(a, p.bucket, p.begin, p.atoms * a.components, p.local * kBlock, which * kBlock, space);
  }
}

template <typename T, typename TA>
__global__ __launch_bounds__(kThreads) void outer_kernel(const Outer a) {
  __shared__ BlockSpace<TA> space;
  __shared__ int32_t list[GP_UNGROUPED];
  const int lane = threadIdx.x & (kLanes - 1), wave = threadIdx.x / kLanes;
  const int32_t* order = a.group.order;
  const int64_t size = static_cast<int64_t>(a.k_in) * a.k_out;
  const int col_tiles = (a.k_out + kBlock - 1) / kBlock, tiles = (a.k_in + kBlock - 1) / kBlock * col_tiles;
  Chunk c;
  if (a.group.offsets) {
    int which;
    if (!chunk_of(a, blockIdx.x, 1, &c, &which)) return;
  } else {   // the atoms of the element, found here
    static_assert(GP_UNGROUPED <= kLanes, "a lane an atom");
    const int element = blockIdx.x;
    const unsigned long long mine = __builtin_amdgcn_ballot_w64(lane < a.n && a.z[min(static_cast<int64_t>(lane), a.n - 1)] == element);
    if (wave == 0 && (mine >> lane) & 1) list[__popcll(mine & ((1ull << lane) - 1))] = lane;
    __syncthreads();
    order = list;
    c = {0, 0, static_cast<int>(__popcll(mine)) * a.components, element, false};
  }
  TA* const out = static_cast<TA*>(c.partial ? a.partial : a.dW) + c.matrix * size;
  for (int tile = blockIdx.y; tile < tiles; tile += gridDim.y)
    outer_block<T, TA>(a, order, c.begin, c.first, c.last, tile / col_tiles * kBlock, tile % col_tiles * kBlock, out, space);
}

__device__ __forceinline__ int atoms_of(const Outer& a, int element) {
  auto at = [&](int e) { return min(max(a.group.offsets[e], 0), static_cast<int>(a.n)); };
  return max(at(element + 1) - at(element), 0);
}

// Slots of the elements before this one: the lanes of a wave add up theirs.
__device__ __forceinline__ int slots_before(const Outer& a, int element) {
  int sum = 0;
  for (int e = threadIdx.x & (kLanes - 1); e < element; e += kLanes) {
    const int atoms = atoms_of(a, e);
    const int k = chunks_of(atoms * a.components, a.per);
    sum += k > 1 ? k : 0;
  }
#pragma unroll
  for (int d = 32; d > 0; d /= 2) sum += __shfl_xor(sum, d);
  return __builtin_amdgcn_readfirstlane(sum);
}

// The matrices of elements with several chunks: their partial ones in order.
template <typename TA>
__global__ __launch_bounds__(kThreads) void join_kernel(const Outer a) {
  const int64_t size = static_cast<int64_t>(a.k_in) * a.k_out;
  const int element = blockIdx.x;
  const int n_slots = slots_before(a, element);
  const int n = chunks_of(atoms_of(a, element) * a.components, a.per);
  if (n < 2 || n_slots > a.slots - n) return;
  const TA* const from = static_cast<const TA*>(a.partial) + n_slots * size;
  TA* const to = static_cast<TA*>(a.dW) + element * size;
  for (int64_t i = static_cast<int64_t>(blockIdx.y) * kThreads + threadIdx.x; i < size; i += static_cast<int64_t>(gridDim.y) * kThreads) {
    TA sum = 0;
#pragma unroll 8
    for (int c = 0; c < n; ++c) sum += from[c * size + i];
    to[i] = sum;
  }
}

template <typename TA>
__global__ __launch_bounds__(kThreads) void zero_kernel(TA* p, int64_t n) {
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; i < n; i += static_cast<int64_t>(gridDim.x) * kThreads) p[i] = 0;
}

// ---- host side

// Rows of a chunk of dW: enough chunks for the chip where the matrices alone do not fill it (200 000 rows, 128 x 128: 79 us, with two thirds of the chunks 100, with
// twice as many 91), none so short that adding them up costs more (6000 rows, 256 x 256: 26 us, with 256 rows at least 33; 10 000 rows, 128 x 128: 23, with 64 30).
constexpr int64_t kLeastRows = 128;
int64_t chunks_wanted(const gp_config* c) {
  const int64_t side = parts_serve(c) ? 128 : kBlock;
  return std::max<int64_t>(1, 384 / (ceil_div(c->k_in, side) * ceil_div(c->k_out, side)));
}
int chunk_rows(const gp_config* c, int64_t n) {
  return static_cast<int>(std::min<int64_t>(std::max<int64_t>(kLeastRows, ceil_div(ceil_div(n * c->components, chunks_wanted(c)), kBlock) * kBlock), int64_t(1) << 30));
}

// Batches without a grouping.  Their own kernels read an element's weights once for every four rows of it (dW: take its rows one after the other), which is best for few rows; for more the call
// makes a grouping itself, a launch of 5 us, and takes the tiles.  What decides is an estimate of both sides' time in us, from both measured at 600 sizes (1 to 64 atoms, 1 to 64 components, 1 to
// 89 elements, 33 x 65 to 2048 x 1024).  E.g. own kernels and tiles, 64 atoms: fp32, 89 elements, 128 x 128: Y 4.7 and 14, dX 5.3 and 14; bfloat16, 8 elements, 1024 x 1024: Y 63 and 40, dX 39 and 33;
// fp32, 64 components, one element, 128 x 128: Y 200 and 15, dW 218 and 24.
struct FewCosts {
  struct Side {
    double weight;   // own kernel: an element of the matrices that are there
    double again;    // the same for each row that makes it be read again
    double group;    // a workgroup
    double stage;    // tiles: a reduced index
    double crowd;    // the same for each tile a compute unit
  } side[2];         // Y, dX
  struct {
    double row, work;                                // own kernel: a row of an element; a product
    double first, tile_row, partial, tile_work;      // tiles: the launches, a row of a chunk, an element of a partial matrix, a product,
    double write;                                    // what an element of dW takes more
  } outer;
};
constexpr FewCosts kFewF32{{{6.5e-7, 3.3e-7, 0.0069, 0.036, 0.020}, {3.0e-7, 2.0e-7, 0.0041, 0.030, 0.022}}, {0.041, 2.1e-8, 12, 0.071, 7.3e-6, 0.9e-8, 3.1e-7}};
constexpr FewCosts kFewBf16{{{7.8e-7, 6.5e-7, 0.0061, 0.027, 0.008}, {5.7e-7, 4.6e-7, 0.0042, 0.020, 0.011}}, {0.068, 2.4e-8, 11, 0.038, 7.3e-6, 0.2e-8, 1.9e-7}};
constexpr FewCosts kFewF64{{{11e-7, 5.3e-7, 0.0048, 0.064, 0.033}, {9.4e-7, 3.3e-7, 0.0140, 0.055, 0.040}}, {0.062, 3.1e-8, 9, 0.084, 0, 10.8e-8, 2.0e-7}};
const FewCosts& few_costs(const gp_config* c) { return c->dtype == SC_F32 ? kFewF32 : c->dtype == SC_F64 ? kFewF64 : kFewBf16; }

bool rows_of_few(const gp_config* c, int64_t n, bool back) {
  if (n > GP_UNGROUPED) return false;
  const FewCosts::Side& f = few_costs(c).side[back];
  const int reduced = back ? c->k_out : c->k_in, columns = back ? c->k_in : c->k_out;
  const double rows = static_cast<double>(n) * c->components, present = static_cast<double>(std::min<int64_t>(c->num_elements, n));   // (at most)
  const double size = static_cast<double>(reduced) * columns, tiles = (rows / kBlock + present) * ceil_div(columns, 128);
  const double own = 4.5 + f.weight * present * size + f.again * std::max(0.0, rows - 4 * present) * size + f.group * rows * ceil_div(columns, 32);
  return own <= 9.3 + (f.stage + f.crowd * tiles / 256) * reduced;
}

bool outer_of_few(const gp_config* c, int64_t n) {
  if (n > GP_UNGROUPED) return false;
  const auto& f = few_costs(c).outer;
  const double rows = static_cast<double>(n) * c->components, present = static_cast<double>(std::min<int64_t>(c->num_elements, n)), size = static_cast<double>(c->k_in) * c->k_out;
  const double each = rows / present, per = chunk_rows(c, n), partial = each > per ? std::ceil(each / per) * present : 0;
  return 5 + f.row * each + f.work * rows * size <=
         f.first + f.tile_row * std::min(per, each) + f.partial * partial * size + f.tile_work * rows * size + f.write * c->num_elements * size;
}

// Chunks of the elements that have several, at most.
int64_t slots_of(const gp_config* c, int64_t n) {
  const int64_t rows = n * c->components, per = chunk_rows(c, n);
  return outer_of_few(c, n) || rows <= per ? 0 : 2 * ceil_div(rows, per);
}
size_t element_size(const gp_config* c) { return c->dtype == SC_F64 ? 8 : c->dtype == SC_F32 ? 4 : 2; }
size_t weight_size(const gp_config* c) { return c->dtype == SC_F64 ? 8 : 4; }
// The workspace: a grouping for batches that come without one, partial matrices.  A workspace for a large batch serves smaller ones: it has room for the grouping too, and for the most slots that a
// batch of so many rows can have (with the chunks' length in whole blocks, more rows may have fewer).
size_t own_grouping_bytes(const gp_config* c) { return offsets_bytes(c->num_elements) + order_bytes(GP_UNGROUPED); }
size_t workspace_bytes(const gp_config* c, int64_t n) {
  const int64_t rows = n * c->components, most = outer_of_few(c, n) || rows <= kLeastRows ? 0 : 2 * std::min(ceil_div(rows, kLeastRows), chunks_wanted(c));
  return own_grouping_bytes(c) + align_up(static_cast<size_t>(most) * c->k_in * c->k_out * weight_size(c), 256);
}

sc_status check_config(const char* fn, const gp_config* cfg, int64_t n) {
  auto bad = [&](sc_status st, const char* what) { return set_error(st, std::string(fn) + ": " + what); };
  if (!cfg) return bad(SC_ERR_INVALID_ARG, "cfg is NULL");
  if (cfg->struct_size != static_cast<int32_t>(sizeof(gp_config)))
    return bad(SC_ERR_INVALID_ARG, "struct_size does not match this library's gp_config");
  if (cfg->num_elements < 1 || cfg->k_in < 1 || cfg->k_out < 1 || cfg->components < 1)
    return bad(SC_ERR_INVALID_ARG, "num_elements, k_in, k_out or components < 1");
  if (cfg->num_elements > GP_MAX_ELEMENTS) return bad(SC_ERR_UNSUPPORTED, "num_elements above GP_MAX_ELEMENTS");
  if (cfg->k_in > GP_MAX_WIDTH || cfg->k_out > GP_MAX_WIDTH) return bad(SC_ERR_UNSUPPORTED, "k_in or k_out above GP_MAX_WIDTH");
  if (cfg->components > GP_MAX_COMPONENTS) return bad(SC_ERR_UNSUPPORTED, "components above GP_MAX_COMPONENTS");
  if (cfg->dtype != SC_F32 && cfg->dtype != SC_F64 && cfg->dtype != SC_BF16) return bad(SC_ERR_INVALID_ARG, "bad dtype");
  if (cfg->reserved != 0) return bad(SC_ERR_INVALID_ARG, "reserved is not 0");
  if (cfg->ld_in != 0 && cfg->ld_in < static_cast<int64_t>(cfg->components) * cfg->k_in)
    return bad(SC_ERR_INVALID_ARG, "ld_in below components * k_in");
  if (cfg->ld_out != 0 && cfg->ld_out < static_cast<int64_t>(cfg->components) * cfg->k_out)
    return bad(SC_ERR_INVALID_ARG, "ld_out below components * k_out");
  if (cfg->ld_in > GP_MAX_STRIDE || cfg->ld_out > GP_MAX_STRIDE) return bad(SC_ERR_UNSUPPORTED, "ld_in or ld_out above GP_MAX_STRIDE");
  if (n < 0) return bad(SC_ERR_INVALID_ARG, "n_nodes < 0");
  if (n > GP_MAX_ROWS / cfg->components) return bad(SC_ERR_UNSUPPORTED, "n_nodes * components above GP_MAX_ROWS");
  return SC_OK;
}

sc_status check_tensors(const char* fn, size_t align, std::initializer_list<const void*> needed, std::initializer_list<const void*> optional) {
  for (const void* p : needed)
    if (!p) return set_error(SC_ERR_INVALID_ARG, std::string(fn) + ": NULL tensor argument");
  for (auto list : {needed, optional})
    for (const void* p : list)
      if (misaligned(p, align)) return set_error(SC_ERR_INVALID_ARG, std::string(fn) + ": tensor pointer not aligned to its element");
  return SC_OK;
}

sc_status check_grouping(const char* fn, const gp_config* cfg, int64_t n, const void* grouping) {
  if (n > GP_UNGROUPED && !grouping) return set_error(SC_ERR_INVALID_ARG, std::string(fn) + ": grouping is NULL");
  if (misaligned(grouping, 256)) return set_error(SC_ERR_INVALID_ARG, std::string(fn) + ": grouping not 256-byte aligned");
  return SC_OK;
}

sc_status check_workspace(const char* fn, const gp_config* cfg, int64_t n, const void* workspace, size_t given) {
  if (!workspace || given < workspace_bytes(cfg, n))
    return set_error(SC_ERR_WORKSPACE, std::string(fn) + ": workspace missing or smaller than gp_workspace_bytes()");
  if (misaligned(workspace, 256)) return set_error(SC_ERR_WORKSPACE, std::string(fn) + ": workspace not 256-byte aligned");
  return SC_OK;
}

sc_status launched(const char* fn, hipError_t e) {
  return e == hipSuccess ? SC_OK : set_error(SC_ERR_HIP, std::string(fn) + ": kernel launch: " + hipGetErrorString(e));
}

int64_t ld_in_of(const gp_config* c) { return c->ld_in ? c->ld_in : static_cast<int64_t>(c->components) * c->k_in; }
int64_t ld_out_of(const gp_config* c) { return c->ld_out ? c->ld_out : static_cast<int64_t>(c->components) * c->k_out; }
// The grouping that a call reads: the caller's, one that it makes itself, none.
hipError_t grouping_for(const gp_config* c, int64_t n, const int32_t* z, const void* grouping, bool few, void* workspace, hipStream_t stream, Grouping* group) {
  *group = Grouping{nullptr, nullptr};
  if (n > GP_UNGROUPED) {
    *group = grouping_of(grouping, c->num_elements);
  } else if (!few) {
    *group = grouping_of(workspace, c->num_elements);
    return launch_group(c, n, z, workspace, stream);
  }
  return hipSuccess;
}

template <bool kBack>
hipError_t launch_rows(const gp_config* c, const Rows& a, hipStream_t stream) {
  if (!a.group.offsets) return launch_rows_few(c, a, kBack, stream);
  if (parts_serve(c)) return launch_rows_parts(c, a, kBack, stream);
  const int64_t tiles = ceil_div(a.n * c->components, kBlock) + std::min<int64_t>(c->num_elements + 1, a.n);
  const dim3 grid(static_cast<unsigned>(std::min(kMaxGrid, ceil_div(tiles * ceil_div(a.columns, kBlock), kXcds) * kXcds)));
  if (c->dtype == SC_F64) hipLaunchKernelGGL((rows_kernel<double, double, kBack>), grid, dim3(kThreads), 0, stream, a);
  else if (c->dtype == SC_F32) hipLaunchKernelGGL((rows_kernel<float, float, kBack>), grid, dim3(kThreads), 0, stream, a);
  else hipLaunchKernelGGL((rows_kernel<__bf16, float, kBack>), grid, dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_outer(const gp_config* c, const Outer& a, hipStream_t stream) {
  const int64_t rows = a.n * c->components;
  hipError_t e;
  if (a.group.offsets && parts_serve(c)) {
    e = launch_outer_parts(c, a, stream);
  } else {
    const int64_t tiles = ceil_div(c->k_in, kBlock) * ceil_div(c->k_out, kBlock);
    const int64_t chunks = a.group.offsets ? ceil_div(c->num_elements + rows / a.per, kXcds) * kXcds : c->num_elements;
    const dim3 grid(static_cast<unsigned>(chunks), static_cast<unsigned>(std::min<int64_t>(tiles, 32768)));
    if (c->dtype == SC_F64) hipLaunchKernelGGL((outer_kernel<double, double>), grid, dim3(kThreads), 0, stream, a);
    else if (c->dtype == SC_F32) hipLaunchKernelGGL((outer_kernel<float, float>), grid, dim3(kThreads), 0, stream, a);
    else hipLaunchKernelGGL((outer_kernel<__bf16, float>), grid, dim3(kThreads), 0, stream, a);
    e = hipGetLastError();
  }
  if (e != hipSuccess || slots_of(c, a.n) == 0) return e;
  const int64_t size = static_cast<int64_t>(c->k_in) * c->k_out;
  const dim3 join(static_cast<unsigned>(c->num_elements), static_cast<unsigned>(std::min<int64_t>(ceil_div(size, kThreads), 64)));
  if (c->dtype == SC_F64) hipLaunchKernelGGL(join_kernel<double>, join, dim3(kThreads), 0, stream, a);
  else hipLaunchKernelGGL(join_kernel<float>, join, dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace
}  // namespace gp

extern "C" {

sc_status gp_grouping_bytes(const gp_config* cfg, int64_t n_nodes, size_t* bytes) {
  const sc_status st = gp::check_config("gp_grouping_bytes", cfg, n_nodes);
  if (st != SC_OK) return st;
  if (!bytes) return sc::set_error(SC_ERR_INVALID_ARG, "gp_grouping_bytes: bytes is NULL");
  *bytes = gp::grouping_bytes(cfg->num_elements, n_nodes);
  return SC_OK;
}

sc_status gp_group(const gp_config* cfg, int64_t n_nodes, const int32_t* z, void* grouping, size_t grouping_bytes_given, void* hip_stream) {
  using namespace gp;
  sc_status st = check_config("gp_group", cfg, n_nodes);
  if (st != SC_OK || n_nodes <= GP_UNGROUPED) return st;
  st = check_tensors("gp_group", 4, {z}, {});
  if (st == SC_OK) st = check_grouping("gp_group", cfg, n_nodes, grouping);
  if (st != SC_OK) return st;
  if (grouping_bytes_given < grouping_bytes(cfg->num_elements, n_nodes))
    return set_error(SC_ERR_WORKSPACE, "gp_group: grouping smaller than gp_grouping_bytes()");
  DeviceGuard guard(cfg->device);
  if (!guard.ok) return set_error(SC_ERR_HIP, "gp_group: cannot make cfg->device current");
  return launched("gp_group", launch_group(cfg, n_nodes, z, grouping, static_cast<hipStream_t>(hip_stream)));
}

sc_status gp_workspace_bytes(const gp_config* cfg, int64_t n_nodes, size_t* bytes) {
  const sc_status st = gp::check_config("gp_workspace_bytes", cfg, n_nodes);
  if (st != SC_OK) return st;
  if (!bytes) return sc::set_error(SC_ERR_INVALID_ARG, "gp_workspace_bytes: bytes is NULL");
  *bytes = gp::workspace_bytes(cfg, n_nodes);
  return SC_OK;
}

sc_status gp_forward(const gp_config* cfg, int64_t n_nodes, const int32_t* z, const void* grouping, const void* X, const void* W,
                     const void* residual, void* Y, void* workspace, size_t workspace_bytes_given, void* hip_stream) {
  using namespace gp;
  sc_status st = check_config("gp_forward", cfg, n_nodes);
  if (st != SC_OK || n_nodes == 0) return st;
  st = check_tensors("gp_forward", 4, {z}, {});
  if (st == SC_OK) st = check_tensors("gp_forward", element_size(cfg), {X, Y}, {residual});
  if (st == SC_OK) st = check_tensors("gp_forward", weight_size(cfg), {W}, {});
  if (st == SC_OK) st = check_grouping("gp_forward", cfg, n_nodes, grouping);
  if (st == SC_OK) st = check_workspace("gp_forward", cfg, n_nodes, workspace, workspace_bytes_given);
  if (st != SC_OK) return st;
  DeviceGuard guard(cfg->device);
  if (!guard.ok) return set_error(SC_ERR_HIP, "gp_forward: cannot make cfg->device current");
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  Grouping group;
  const hipError_t e = grouping_for(cfg, n_nodes, z, grouping, rows_of_few(cfg, n_nodes, false), workspace, stream, &group);
  if (e != hipSuccess) return launched("gp_forward", e);
  const Rows a{n_nodes, ld_in_of(cfg), ld_out_of(cfg), z, group, cfg->num_elements, cfg->components, cfg->k_in, cfg->k_out, X, W, residual, Y};
  return launched("gp_forward", launch_rows<false>(cfg, a, stream));
}

sc_status gp_backward(const gp_config* cfg, int64_t n_nodes, const int32_t* z, const void* grouping, const void* X, const void* W,
                      const void* dY, void* dX, void* dW, void* workspace, size_t workspace_bytes_given, void* hip_stream) {
  using namespace gp;
  sc_status st = check_config("gp_backward", cfg, n_nodes);
  if (st != SC_OK) return st;
  if (!dX && !dW) return set_error(SC_ERR_INVALID_ARG, "gp_backward: dX and dW are both NULL");
  st = check_tensors("gp_backward", element_size(cfg), {}, {X, dY, dX});
  if (st == SC_OK) st = check_tensors("gp_backward", weight_size(cfg), {}, {W, dW});
  if (st != SC_OK) return st;
  if (n_nodes > 0) {
    st = check_tensors("gp_backward", 4, {z}, {});
    if (st == SC_OK) st = check_tensors("gp_backward", 1, {dY}, {});
    if (st == SC_OK && dX) st = check_tensors("gp_backward", 1, {W}, {});
    if (st == SC_OK && dW) st = check_tensors("gp_backward", 1, {X}, {});
    if (st == SC_OK) st = check_grouping("gp_backward", cfg, n_nodes, grouping);
    if (st == SC_OK) st = check_workspace("gp_backward", cfg, n_nodes, workspace, workspace_bytes_given);
    if (st != SC_OK) return st;
  } else if (!dW) {
    return SC_OK;
  }
  DeviceGuard guard(cfg->device);
  if (!guard.ok) return set_error(SC_ERR_HIP, "gp_backward: cannot make cfg->device current");
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  if (n_nodes == 0) {
    const int64_t size = static_cast<int64_t>(cfg->num_elements) * cfg->k_in * cfg->k_out;
    const dim3 grid(static_cast<unsigned>(std::min<int64_t>(ceil_div(size, kThreads), 4096)));
    if (cfg->dtype == SC_F64) hipLaunchKernelGGL(zero_kernel<double>, grid, dim3(kThreads), 0, stream, static_cast<double*>(dW), size);
    else hipLaunchKernelGGL(zero_kernel<float>, grid, dim3(kThreads), 0, stream, static_cast<float*>(dW), size);
    return launched("gp_backward", hipGetLastError());
  }
  const bool rows_few = !dX || rows_of_few(cfg, n_nodes, true), outer_few = !dW || outer_of_few(cfg, n_nodes);
  Grouping group;
  hipError_t e = grouping_for(cfg, n_nodes, z, grouping, rows_few && outer_few, workspace, stream, &group);
  const bool ungrouped = n_nodes <= GP_UNGROUPED;
  const Grouping none{nullptr, nullptr};
  if (dX && e == hipSuccess) {
    const Rows a{n_nodes, ld_out_of(cfg), ld_in_of(cfg), z, ungrouped && rows_few ? none : group, cfg->num_elements, cfg->components, cfg->k_out, cfg->k_in, dY, W, nullptr, dX};
    e = launch_rows<true>(cfg, a, stream);
  }
  if (dW && e == hipSuccess) {
    const Outer a{n_nodes, ld_in_of(cfg), ld_out_of(cfg), z, ungrouped && outer_few ? none : group, cfg->num_elements, cfg->components, cfg->k_in, cfg->k_out,
                  chunk_rows(cfg, n_nodes), static_cast<int>(slots_of(cfg, n_nodes)), X, dY, dW, static_cast<char*>(workspace) + own_grouping_bytes(cfg)};
    e = launch_outer(cfg, a, stream);
  }
  return launched("gp_backward", e);
}

}  // extern "C"
