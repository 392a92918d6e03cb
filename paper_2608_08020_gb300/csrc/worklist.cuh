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

// units(s): units of source s; cost(s, i): cost of its i-th unit (clamped to the last bucket);
// emit(s, i, place): writes it.  Every thread of the CTA calls it.  Returns the number of units.
// Units of one cost come in the order of their sources, so the list is the same each time.
template <class Units, class Cost, class Emit>
__device__ int emit_sorted(ListSmem& sm, int nsrc, Units units, Cost cost, Emit emit) {
  const int tid = threadIdx.x;
  sm.hist[tid] = 0;
  int all = 0;
  for (int pass = 0; pass < 2; ++pass) {
    for (int base = 0; base < nsrc; base += kListThreads) {
      int total;
      if (pass == 0 || nsrc > kListThreads) {
        const int s = base + tid;
        const int n = s < nsrc ? units(s) : 0;
        sm.pre[tid] = block_exclusive_scan(n, sm.tmp, &total);
        if (tid == 0) sm.pre[kListThreads] = total;
        __syncthreads();
      }
      total = sm.pre[kListThreads];
      for (int f0 = 0; f0 < total; f0 += kListThreads) {
        const int f = f0 + tid, lane = tid & 31;
        int lo = 0, hi = kListThreads;  // the last source whose first unit is <= f
        while (hi - lo > 1) {
          const int mid = (lo + hi) >> 1;
          if (sm.pre[mid] <= f) lo = mid;
          else hi = mid;
        }
        const int s = base + lo, i = f - sm.pre[lo];
        const int c = f < total ? kListThreads - 1 - min(max(cost(s, i), 0), kListThreads - 1) : -1;
        if (pass == 0) {
          if (c >= 0) atomicAdd(&sm.hist[c], 1);
          continue;
        }
        // Places: a warp's units of one cost by lane, the warps one after another.
        const unsigned same = __match_any_sync(0xffffffffu, c);
        const int first = __ffs(same) - 1;
        int at = 0;
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
