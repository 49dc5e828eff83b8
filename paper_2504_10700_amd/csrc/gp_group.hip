// The grouping of include/gp.h: a stable counting sort of the atoms by element.
//
// A wave takes a stretch of the batch, 64 atoms at a time: ballots over the bits of the key tell every lane which others have its element,
// so an atom's rank among them is a count of bits and no atomics are needed.  Up to kSortAtoms atoms one workgroup does it all; larger
// batches are counted by kSortGroups workgroups, and a second launch of the same workgroups places the atoms, each adding up what stands before its
// own counts by itself (a few thousand words from the caches: cheaper than a launch between the two).  Latency bounds it: 1000 atoms 5.4 us, 10 000 9.2, 200 000 11.4 (two launches of 5.0 and 7.6).
#include <algorithm>

#include "gp_internal.h"

namespace gp {
namespace {

__device__ __forceinline__ int bucket_of(int z, int elements) { return static_cast<unsigned>(z) < static_cast<unsigned>(elements) ? z : elements; }

// The lanes with this lane's key (all lanes call; keys of lanes that take no part: -1, which no other lane has).
__device__ __forceinline__ unsigned long long same_key(int key, int bits) {
  unsigned long long same = ~0ull;
  for (int b = 0; b < bits; ++b) {
    const bool on = (key >> b) & 1;
    const unsigned long long m = __builtin_amdgcn_ballot_w64(on);
    same &= on ? m : ~m;
  }
  const unsigned long long out = __builtin_amdgcn_ballot_w64(key < 0);
  return key < 0 ? out : same & ~out;
}

// Counts of a workgroup's atoms by wave and bucket: count[wave][buckets].
__device__ __forceinline__ void count_stretch(const int32_t* __restrict__ z, int64_t from, int64_t to, int elements, int bits, int* count) {
  const int lane = threadIdx.x & (kLanes - 1);
  for (int64_t i = from; i < to; i += kLanes) {
    const int key = i + lane < to ? bucket_of(z[i + lane], elements) : -1;
    const unsigned long long same = same_key(key, bits);
    if (key >= 0 && (same & ((1ull << lane) - 1)) == 0) count[key] += __popcll(same);   // the first of each key
    __builtin_amdgcn_wave_barrier();
  }
}
__device__ __forceinline__ void place_stretch(const int32_t* __restrict__ z, int64_t from, int64_t to, int elements, int bits, int* next, int32_t* order,
                                              int64_t n) {
  const int lane = threadIdx.x & (kLanes - 1);
  for (int64_t i = from; i < to; i += kLanes) {
    const int key = i + lane < to ? bucket_of(z[i + lane], elements) : -1;
    const unsigned long long same = same_key(key, bits), before = same & ((1ull << lane) - 1);
    int base = 0;
    if (key >= 0) base = next[key];
    if (key >= 0) {
      const int at = base + __popcll(before);
      if (at < n) order[at] = static_cast<int32_t>(i + lane);   // (z that changes between the two launches stays inside)
    }
    __builtin_amdgcn_wave_barrier();
    if (key >= 0 && before == 0) next[key] = base + __popcll(same);
    __builtin_amdgcn_wave_barrier();
  }
}

// A wave's stretch of the workgroup's atoms, whole groups of 64.
struct Stretch {
  int64_t from, to;
};
__device__ __forceinline__ Stretch stretch_of(int64_t n, int groups, int group) {
  const int wave = threadIdx.x / kLanes;
  const int64_t per = (n + static_cast<int64_t>(groups) * kSortWaves * kLanes - 1) / (static_cast<int64_t>(groups) * kSortWaves * kLanes) * kLanes;
  const int64_t from = (static_cast<int64_t>(group) * kSortWaves + wave) * per;
  return {min(from, n), min(from + per, n)};
}

__device__ __forceinline__ void clear(int* p, int n) {
  for (int i = threadIdx.x; i < n; i += kSortThreads) p[i] = 0;
}

// Exclusive prefix sums of v[0..n), in place, by the workgroup.  total: of all.
__device__ __forceinline__ void exclusive_scan(int* v, int n, int* wave_sums) {
  const int lane = threadIdx.x & (kLanes - 1), wave = threadIdx.x / kLanes;
  const int x = threadIdx.x < n ? v[threadIdx.x] : 0;   // (n <= kSortThreads)
  int s = x;
#pragma unroll
  for (int d = 1; d < kLanes; d *= 2) {
    const int a = __shfl_up(s, d);
    if (lane >= d) s += a;
  }
  if (lane == kLanes - 1) wave_sums[wave] = s;
  __syncthreads();
  int before = 0;
  for (int w = 0; w < wave; ++w) before += wave_sums[w];
  if (threadIdx.x < n) v[threadIdx.x] = before + s - x;
  __syncthreads();
}

// LDS: count[kSortWaves][elements + 1], start[elements + 2].
// kPlace: 0: counts alone, to counts[group][bucket]; 1: places the atoms after such a launch; 2: both (one workgroup).
template <int kPlace>
__global__ __launch_bounds__(kSortThreads) void sort_kernel(int64_t n, int elements, int bits, const int32_t* __restrict__ z, int32_t* __restrict__ counts,
                                                            int32_t* __restrict__ offsets, int32_t* __restrict__ order) {
  extern __shared__ int lds[];
  __shared__ int wave_sums[kSortWaves];
  const int buckets = elements + 1;
  int* const count = lds;
  int* const start = lds + kSortWaves * buckets;
  const int wave = threadIdx.x / kLanes, groups = gridDim.x, group = blockIdx.x;
  clear(count, kSortWaves * buckets);
  clear(start, buckets);
  __syncthreads();
  const Stretch s = stretch_of(n, groups, group);
  count_stretch(z, s.from, s.to, elements, bits, count + wave * buckets);
  __syncthreads();
  if (kPlace == 0) {
    for (int b = threadIdx.x; b < buckets; b += kSortThreads) {
      int sum = 0;
      for (int w = 0; w < kSortWaves; ++w) sum += count[w * buckets + b];
      counts[static_cast<int64_t>(group) * buckets + b] = sum;
    }
    return;
  }
  // atoms of each bucket in all workgroups, and in those before this one
  int* const before = lds + kSortWaves * buckets + buckets;
  clear(before, buckets);
  __syncthreads();
  if (kPlace == 1) {
    const int parts = max(1, kSortThreads / buckets);   // integer additions: their order does not matter
    for (int i = threadIdx.x; i < parts * buckets; i += kSortThreads) {
      const int b = i % buckets;
      int all = 0, mine = 0;
#pragma unroll 8
      for (int g = i / buckets; g < groups; g += parts) {
        const int c = counts[static_cast<int64_t>(g) * buckets + b];
        all += c;
        mine += g < group ? c : 0;
      }
      atomicAdd(start + b, all);
      atomicAdd(before + b, mine);
    }
  } else {
    for (int b = threadIdx.x; b < buckets; b += kSortThreads) {
      int sum = 0;
      for (int w = 0; w < kSortWaves; ++w) sum += count[w * buckets + b];
      start[b] = sum;
    }
  }
  __syncthreads();
  // (buckets can be one more than the threads: the last bucket's start is what the others leave)
  exclusive_scan(start, min(buckets, kSortThreads), wave_sums);
  if (buckets > kSortThreads) {
    if (threadIdx.x == 0) {
      int last = start[kSortThreads - 1];
      int in_last = 0;
      if (kPlace == 1) for (int g = 0; g < groups; ++g) in_last += counts[static_cast<int64_t>(g) * buckets + kSortThreads - 1];
      else for (int w = 0; w < kSortWaves; ++w) in_last += count[w * buckets + kSortThreads - 1];
      start[kSortThreads] = last + in_last;
    }
    __syncthreads();
  }
  if (group == 0) {
    for (int b = threadIdx.x; b < buckets; b += kSortThreads) offsets[b] = start[b];
    if (threadIdx.x == 0) offsets[buckets] = static_cast<int32_t>(n);
  }
  for (int b = threadIdx.x; b < buckets; b += kSortThreads) {
    int at = start[b] + before[b];
    for (int w = 0; w < kSortWaves; ++w) {
      const int c = count[w * buckets + b];
      count[w * buckets + b] = at;
      at += c;
    }
  }
  __syncthreads();
  place_stretch(z, s.from, s.to, elements, bits, count + wave * buckets, order, n);
}

}  // namespace

hipError_t launch_group(const gp_config* cfg, int64_t n, const int32_t* z, void* grouping, hipStream_t stream) {
  const int elements = cfg->num_elements;
  int32_t* const offsets = static_cast<int32_t*>(grouping);
  int32_t* const order = reinterpret_cast<int32_t*>(static_cast<char*>(grouping) + offsets_bytes(elements));
  int32_t* const counts = reinterpret_cast<int32_t*>(reinterpret_cast<char*>(order) + order_bytes(n));
  int bits = 1;
  while ((1 << bits) < elements + 1) ++bits;
  const size_t lds = static_cast<size_t>(elements + 1) * (kSortWaves + 2) * 4;   // at most 73.8 KB
  auto set = [&](const void* kernel) {
    return lds > 64 * 1024 ? hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(lds)) : hipSuccess;
  };
  if (n <= kSortAtoms) {
    const hipError_t e = set(reinterpret_cast<const void*>(&sort_kernel<2>));
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((sort_kernel<2>), dim3(1), dim3(kSortThreads), lds, stream, n, elements, bits, z, counts, offsets, order);
    return hipGetLastError();
  }
  hipError_t e = set(reinterpret_cast<const void*>(&sort_kernel<0>));
  if (e == hipSuccess) e = set(reinterpret_cast<const void*>(&sort_kernel<1>));
  if (e != hipSuccess) return e;
  const int groups = static_cast<int>(std::min<int64_t>(kSortGroups, (n + kSortAtoms - 1) / kSortAtoms * 4));
  hipLaunchKernelGGL((sort_kernel<0>), dim3(groups), dim3(kSortThreads), lds, stream, n, elements, bits, z, counts, offsets, order);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((sort_kernel<1>), dim3(groups), dim3(kSortThreads), lds, stream, n, elements, bits, z, counts, offsets, order);
  return hipGetLastError();
}

}  // namespace gp
