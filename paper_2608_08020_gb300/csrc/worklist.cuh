// Sorted work lists built by one CTA: the units of many sources (sequences, shared segments, beams)
// in descending order of cost, so that taken in turn they make even shares, the longest begun first.
#pragma once
#include "internal.cuh"

namespace gb {

constexpr int kListThreads = 1024;    // threads of a planner CTA: sources per chunk, and cost buckets
struct ListSmem {
  int pre[kListThreads + 1];          // units of the chunk's earlier sources
  int hist[kListThreads];             // units per cost, then the next place of each cost
  int tmp[33];
};

// Adds x over the CTA; cell: a word of shared memory that was 0 and that nobody uses again.
__device__ __forceinline__ int block_sum(int x, int* cell) {
  x = __reduce_add_sync(0xffffffffu, x);
  if ((threadIdx.x & 31) == 0 && x != 0) atomicAdd(cell, x);
  __syncthreads();
  return *cell;
}

// units(s): units of source s; cost(s, i): cost of its i-th unit (clamped to the last bucket);
// emit(s, i, place): writes it.  Every thread of the CTA calls it.  Returns the number of units.
// Units of one cost come in the order of their sources, so the list is the same each time.
// The planner's time is latency (one CTA, cold code): lists of up to kListThreads units keep what the count found.
template <class Units, class Cost, class Emit>
__device__ int emit_sorted(ListSmem& sm, int nsrc, Units units, Cost cost, Emit emit) {
  const int tid = threadIdx.x, lane = tid & 31;
  sm.hist[tid] = 0;
  int all = 0, s = 0, i = 0, c = -1;  // the thread's unit and its bucket
#pragma unroll 1
  for (int pass = 0; pass < 2; ++pass) {
    const bool kept = pass == 1 && nsrc <= kListThreads && all <= kListThreads;
#pragma unroll 1
    for (int base = 0; base < nsrc; base += kListThreads) {
      int total;
      if (pass == 0 || nsrc > kListThreads) {
        const int src = base + tid;
        const int n = src < nsrc ? units(src) : 0;
        sm.pre[tid] = block_exclusive_scan(n, sm.tmp, &total);
        if (tid == 0) sm.pre[kListThreads] = total;
        __syncthreads();
      }
      total = sm.pre[kListThreads];
#pragma unroll 1
      for (int f0 = 0; f0 < total; f0 += kListThreads) {
        const int f = f0 + tid;
        if (!kept) {
          c = -1;
          if (f < total) {
            int lo = 0, hi = min(kListThreads, nsrc - base);  // the last source whose first unit is <= f
            while (hi - lo > 1) {
              const int mid = (lo + hi) >> 1;
              if (sm.pre[mid] <= f) lo = mid;
              else hi = mid;
            }
            s = base + lo;
            i = f - sm.pre[lo];
            c = kListThreads - 1 - min(max(cost(s, i), 0), kListThreads - 1);
          }
        }
        if (pass == 0) {
          if (c >= 0) atomicAdd(&sm.hist[c], 1);
          continue;
        }
        // Places: a warp's units of one cost by lane, the warps one after another.
        unsigned same = 0;
        int first = 0, at = 0;
        if (f0 + (tid & ~31) < total) {
          same = __match_any_sync(0xffffffffu, c);
          first = __ffs(same) - 1;
        }
        for (int w = 0; w < kListThreads / 32 && f0 + 32 * w < total; ++w) {
          if (tid >> 5 == w && c >= 0 && lane == first) {
            at = sm.hist[c];
            sm.hist[c] = at + __popc(same);
          }
          __syncthreads();
        }
        at = __shfl_sync(0xffffffffu, at, first) + __popc(same & ((1u << lane) - 1));
        if (c >= 0) emit(s, i, at);
      }
      if (pass == 0) all += total;
      __syncthreads();
    }
    if (pass == 0) {
      int total;
      const int first = block_exclusive_scan(sm.hist[tid], sm.tmp, &total);
      sm.hist[tid] = first;
      __syncthreads();
    }
  }
  return all;
}

}  // namespace gb
