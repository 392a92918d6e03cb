// Trees of drafted tokens over a beam pool: their attention (gb_draft_attention), the append of an accepted
// path (gb_accept_draft) and cutting a beam short (gb_truncate).
//
//   out[b][i][h] = sum_j p_j v_j,  p = softmax_j(scale q[b][i][h] . k_j)
// where j runs over beam b's context (through its block table) and over i and its ancestors in the beam's
// tree, whose keys and values are the caller's.
//
// A round's plan, made with layer 0: every shared-prefix segment's pages, down to the depth that pays, are read once for
// all drafted tokens of the beams that share them (rows (beam, token, query head), up to 256 to a unit), every beam's remainder
// and its drafts by units of its own; long runs of keys are split.  A beam whose rows one unit answers gets
// its result from it; the others' units leave records (sum, maximum, row sum) that k_draft_merge joins.
// bf16: flash.cuh; fp32: tile.cuh, without segments.
//
// Bound by the reads of the cache while rows x 2 flops a byte stay below the machine's ~280, i.e. up to some
// 100 rows a shared token, and by the tensor cores beyond.  Measured (bf16): a layer of 64 traces at 4000 tokens, trees of up to
// 16, 114 us with its plan and join (387 MB in 95 us inside the attention, 4.1 TB/s); 198 traces at 8000 tokens 255 us; a
// layer of 128 traces of 190 tokens 44 us.
#include <algorithm>
#include <atomic>
#include <type_traits>

#include "flash.cuh"
#include "tile.cuh"
#include "worklist.cuh"

namespace gb {
namespace {

constexpr int kMaxDraft = 64;   // tokens of a tree: a row's ancestors are one 64-bit word
constexpr int kTailRec = kMaxSegDepth;  // rec_off column of a beam's own units
constexpr int kRecOffs = kMaxSegDepth + 1;

// Workspace words of control.
enum DraftCtl : int { kDrUnits = 0, kDrFew = 1, kDrChanges = 2, kDrToken = 4, kDrWords = 64 };

struct DraftUnit {
  int seg;         // -1: a beam's own unit
  int beam;        // whose table lists the pages
  int e0, ntok;    // rows: entries [e0, e0 + ntok) of the token list, or the beam's tokens
  int tok0, tok1;  // context positions
  int drafts;      // the beam's drafted tokens, which follow; 0: none
  int rec;         // a segment's: which of its pieces; a beam's own: the record, -1: the output itself
};

// Byte offsets of the workspace.
struct DraftLayout {
  size_t units, anc, cnt, nrec, rec_base, rec_off, depth, seg_cnt, seg_list, off, list, acc, ml, rec, total;
  int rec_cap, max_units;
};

int ws_rows(const gb_pool_config& c, int T) { return T * (c.num_q_heads / c.num_kv_heads); }

DraftLayout draft_layout(const gb_pool_config& c, int num_sms, int T) {
  DraftLayout d{};
  const size_t B = (size_t)c.max_beams;
  size_t o = 0;
  auto take = [&](size_t bytes) { const size_t at = o; o = (o + bytes + 255) & ~(size_t)255; return at; };
  // Records: six a beam (shared segments and its own units; the plan stops splitting, then
  // leaves the deepest segments to the beams, when there would be more), and what splits a few long
  // beams over all SMs.
  d.rec_cap = (int)(6 * B) + 2 * num_sms;
  d.max_units = d.rec_cap * ((ws_rows(c, T) + kTileRows - 1) / kTileRows + 1);
  take(kDrWords * sizeof(int));
  d.units = take((size_t)d.max_units * sizeof(DraftUnit));
  d.anc = take(B * T * sizeof(unsigned long long));
  d.cnt = take(B * sizeof(int));
  d.nrec = take(B * sizeof(int));
  d.rec_base = take(B * sizeof(int));
  d.rec_off = take(B * kRecOffs * sizeof(int));
  d.depth = take(B * sizeof(int));
  d.seg_cnt = take(B * kMaxSegDepth * sizeof(int));
  d.seg_list = take(B * kMaxSegDepth * sizeof(int));
  d.off = take(B * kMaxSegDepth * sizeof(int));
  d.list = take(B * kMaxSegDepth * T * sizeof(int2));
  d.acc = take(B * 4 * sizeof(int) + B * sizeof(unsigned long long));
  const size_t rows = (size_t)d.rec_cap * c.num_kv_heads * ws_rows(c, T);
  d.ml = take(rows * sizeof(float2));
  d.rec = take(rows * c.head_dim * sizeof(float));
  d.total = o;
  return d;
}

// The workspace's parts, by value to the kernels.
struct DraftView {
  int T, rows;              // tokens of a tree, rows of a beam and KV head (T x G)
  int rec_cap, max_units;
  unsigned long long token; // the plan's name
  int* ctl;
  DraftUnit* units;
  unsigned long long* anc;  // [max_beams][T] ancestors and self
  int* cnt;                 // [max_beams] drafted tokens, 0 for an inactive slot
  int* nrec;                // [max_beams] records
  int* rec_base;            // [max_beams] the first of them
  int* rec_off;             // [max_beams][kRecOffs] those of the k-th segment, and of the beam's own units
  int* depth;               // [max_beams] segments used
  int* seg_cnt;             // [segments] drafted tokens of its beams
  int* seg_list;            // [segments] where its token list begins
  int* off;                 // [max_beams][kMaxSegDepth] the beam's place in that list
  int2* list;               // (beam | token << 10, record of the beam's first piece of the segment)
  int* acc_n;               // [max_beams] accept: tokens appended,
  int* acc_pos;             //   the position of the first,
  int* acc_old;             //   the shared tail page they moved away from, or -1
  unsigned long long* acc_path;  // the path's tokens
  float2* ml;               // [rec_cap][Hkv][rows] (maximum, sum)
  float* rec;               // [rec_cap][Hkv][rows][D]
};

DraftView draft_view(const gb_pool* p, const DraftLayout& d, int T, void* ws, unsigned long long token) {
  char* m = static_cast<char*>(ws);
  const size_t B = (size_t)p->cfg.max_beams;
  DraftView v{};
  v.T = T;
  v.token = token;
  v.rows = ws_rows(p->cfg, T);
  v.rec_cap = d.rec_cap;
  v.max_units = d.max_units;
  v.ctl = reinterpret_cast<int*>(m);
  v.units = reinterpret_cast<DraftUnit*>(m + d.units);
  v.anc = reinterpret_cast<unsigned long long*>(m + d.anc);
  v.cnt = reinterpret_cast<int*>(m + d.cnt);
  v.nrec = reinterpret_cast<int*>(m + d.nrec);
  v.rec_base = reinterpret_cast<int*>(m + d.rec_base);
  v.rec_off = reinterpret_cast<int*>(m + d.rec_off);
  v.depth = reinterpret_cast<int*>(m + d.depth);
  v.seg_cnt = reinterpret_cast<int*>(m + d.seg_cnt);
  v.seg_list = reinterpret_cast<int*>(m + d.seg_list);
  v.off = reinterpret_cast<int*>(m + d.off);
  v.list = reinterpret_cast<int2*>(m + d.list);
  v.acc_path = reinterpret_cast<unsigned long long*>(m + d.acc);
  v.acc_n = reinterpret_cast<int*>(v.acc_path + B);
  v.acc_pos = v.acc_n + B;
  v.acc_old = v.acc_pos + B;
  v.ml = reinterpret_cast<float2*>(m + d.ml);
  v.rec = reinterpret_cast<float*>(m + d.rec);
  return v;
}

// Whether the workspace still holds the launch's own plan, of the pool as it is.  The host knows the calls, not the replays of
// graphs, which change the pool or plan a round of their own in this workspace.
__device__ __forceinline__ bool plan_holds(const PoolView& v, const DraftView& w) {
  return *reinterpret_cast<const unsigned long long*>(w.ctl + kDrToken) == w.token && w.ctl[kDrChanges] == v.ctl[kCtlChanges];
}

// One warp, where the plan does not hold: says so, and leaves in its place one by which the join has nothing to write.  (A check
// of its own would cost each of the join's many CTAs a load more: 36 layers 1657 -> 1690 us.)
__device__ __forceinline__ void spoil_plan(const PoolView& v, const DraftView& w) {
  const int lane = threadIdx.x & 31;
  if (lane == 0) {
    set_status(v.ctl, GB_ERR_STATE);
    *reinterpret_cast<unsigned long long*>(w.ctl + kDrToken) = 0;
  }
  for (int b = lane; b < v.max_beams; b += 32) {
    w.cnt[b] = w.T;
    w.nrec[b] = 1;
  }
}

// A warp's slot b: lane l's masks of tokens l and l + 32 (ancestors and self; 0 from `count` on), by
// doubling the paths.  A parent that is no earlier token counts as none and makes *bad true.
__device__ __forceinline__ void ancestors(const int* parent, int T, int count, unsigned long long* lo,
                                          unsigned long long* hi, bool* bad) {
  const int lane = threadIdx.x & 31;
  unsigned long long a[2];
  int up[2];
  bool wrong = false;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int i = lane + 32 * k;
    const bool on = i < count;
    int p = on ? parent[i] : -1;
    if (p < -1 || p >= i) {
      wrong |= on;
      p = -1;
    }
    up[k] = p;
    a[k] = on ? 1ull << i : 0ull;
  }
#pragma unroll
  for (int s = 0; s < 6; ++s) {  // paths of up to 2^6 tokens
    unsigned long long na[2];
    int nu[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int from = up[k] & 31;
      const unsigned long long a0 = __shfl_sync(0xffffffffu, a[0], from), a1 = __shfl_sync(0xffffffffu, a[1], from);
      const int u0 = __shfl_sync(0xffffffffu, up[0], from), u1 = __shfl_sync(0xffffffffu, up[1], from);
      na[k] = up[k] < 0 ? a[k] : a[k] | (up[k] < 32 ? a0 : a1);
      nu[k] = up[k] < 0 ? -1 : (up[k] < 32 ? u0 : u1);
    }
    a[0] = na[0];
    a[1] = na[1];
    up[0] = nu[0];
    up[1] = nu[1];
  }
  *lo = a[0];
  *hi = a[1];
  *bad = __any_sync(0xffffffffu, wrong);
}

// Tiles of 128 keys of n context tokens and the drafts: the drafted tokens lie in the second half of the
// last tile, beside at most 64 context tokens.
__device__ __forceinline__ int tail_tiles(int n) { return n / flash::kTok + (n % flash::kTok <= 64 ? 1 : 2); }

__device__ __forceinline__ int drafted(const int* count, int b, int T, bool act, bool* bad) {
  const int n = !act ? 0 : count ? count[b] : T;
  if (n < 0 || n > T) {
    *bad = true;
    return n < 0 ? 0 : T;
  }
  return n;
}

// What the plan counts a unit as, in eighths of the time of a 128-key tile of up to 128 rows: a tile of more rows is
// twice that, a unit's start and end (queries, pipeline, result) kUnitCost more per 128 rows, and a record that has to be written
// and joined kRecCost per 128 rows.
constexpr int kTileCost = 8, kUnitCost = 10, kRecCost = 14;

// Slots up to which the planner's CTA also writes the rows (a slot to a warp), without a launch of its own: 8 slots 28 us, with
// the launch 32; 64 slots in this way 262.5 us, with the launch 260.
constexpr int kOneLaunch = 16;

// A warp per slot of [first, first + step, ...): the ancestor masks of its tokens, and their entries in the lists of the
// slot's segments.
__device__ __forceinline__ void draft_rows(const PoolView& v, const DraftView& w, const int* parent, const int* count,
                                           int first, int step) {
  const int lane = threadIdx.x & 31;
  for (int b = first; b < v.max_beams; b += step) {
    bool bad = false;
    const int n = drafted(count, b, w.T, v.active[b] != 0, &bad), nd = w.depth[b], base = w.rec_base[b];
    int at = 0, rec = 0;
    if (lane < nd && n > 0) {  // lane k: the slot's k-th segment
      at = w.seg_list[v.seg_bid[b * kMaxSegDepth + lane]] + w.off[b * kMaxSegDepth + lane];
      rec = base + w.rec_off[b * kRecOffs + lane];
    }
    unsigned long long lo, hi;
    bool wrong;
    ancestors(parent + (size_t)b * w.T, w.T, n, &lo, &hi, &wrong);
    if (lane < w.T) w.anc[(size_t)b * w.T + lane] = lo;
    if (lane + 32 < w.T) w.anc[(size_t)b * w.T + lane + 32] = hi;
    if ((bad || wrong) && lane == 0) set_status(v.ctl, GB_ERR_INVALID);
    for (int k = 0; k < nd; ++k) {
      int2* to = w.list + __shfl_sync(0xffffffffu, at, k);
      const int r = __shfl_sync(0xffffffffu, rec, k);
      for (int i = lane; i < n; i += 32) to[i] = make_int2(b | i << 10, r);
    }
  }
}
// The work list (one CTA).  2^`shift` tokens to a unit, 2^`small` where there are few units; `least`: tiles below which a
// run of keys is not split; `coarse`: bits dropped from the costs, so that their sums stay in range.
//
// Down to which depth the shared segments are used is chosen by the cost above: a segment's unit reads
// its pages once for up to 256 rows, but every piece of a beam's context beyond the first costs a record.  64 beams of 50 rows
// over 64 shared and 130 own tokens run without segments; 64 beams of 50 rows at 4000 tokens use them all.
//
// The time is latency, nothing else runs meanwhile: loads are issued together, counts and sums stay in shared memory (10 us for
// 64 to 200 slots, from 18 with counts in memory and the list's places searched twice).
__global__ void __launch_bounds__(kListThreads) k_draft_plan(PoolView v, DraftView w, const int* parent, const int* count,
                                                             int shift, int small, int least, int coarse, bool segs) {
  pdl_wait();
  pdl_launch_dependents();
  constexpr int kCached = 4096;         // segments whose rows, tiles and depth fit in shared memory
  __shared__ ListSmem sm;
  __shared__ short s_cnt[kMaxBeams];
  __shared__ unsigned s_src[kCached];   // rows, then rows | tiles << 16, each clamped (a source with more is read from memory)
  constexpr int kStaged = 512;          // slots whose segments' lengths do
  __shared__ unsigned short s_seg[kStaged * kMaxSegDepth];
  __shared__ int s_cost[kMaxSegDepth + 1];
  __shared__ int s_start[kMaxBeams], s_len[kMaxBeams];
  constexpr int kFewTries = 24;
  enum { kSumFew, kSumWork, kSumWorkFew, kSumList, kSumTry, kSums = kSumTry + kFewTries };
  __shared__ int s_sum[kSums];
  const int tid = threadIdx.x;
  const int b = tid, cap = v.max_beams;
  bool act = false;
  int L = 0, nd = 0;
  if (b < cap) {
    const int on = v.active[b], len = v.seq_len[b], deep = segs ? v.seg_nseg[b] : 0;
    act = on != 0;
    L = act ? len : 0;
    nd = deep;
  }
  bool bad = false;
  const int cnt = b < cap ? drafted(count, b, w.T, act, &bad) : 0;
  const int nseg = segs ? v.ctl[kCtlSegCount] : 0;
  if (cnt <= 0) nd = 0;
  s_cnt[b] = (short)cnt;
  if (b < cap) w.cnt[b] = cnt;
  if (tid < kSums) s_sum[tid] = 0;
  if (tid <= kMaxSegDepth) s_cost[tid] = 0;
  for (int s = tid; s < nseg; s += kListThreads) {
    if (s < kCached) s_src[s] = 0;
    else w.seg_cnt[s] = 0;
  }
  // The depth and tiles of the thread's first segment.
  int depth0 = 0, tiles0 = 0;
  auto seg_tiles = [&](int s) { return (v.seg_len[s] * v.P + flash::kTok - 1) / flash::kTok; };
  if (tid < nseg) {
    tiles0 = seg_tiles(tid);
    depth0 = v.seg_members[v.seg_mem_off[tid]] % kMaxSegDepth;
  }
  auto seg_depth = [&](int s) { return s < kListThreads ? depth0 : v.seg_members[v.seg_mem_off[s]] % kMaxSegDepth; };
  auto own_tiles = [&](int s) { return s < kListThreads ? tiles0 : seg_tiles(s); };  // (s: of this thread)
  __syncthreads();
  // Segments: their drafted tokens, and each beam's place among them.
#pragma unroll 1
  for (int e = tid; e < (segs ? cap * kMaxSegDepth : 0); e += kListThreads) {
    const int c = s_cnt[e / kMaxSegDepth], k = e % kMaxSegDepth, deep = v.seg_nseg[e / kMaxSegDepth], s = v.seg_bid[e];
    if (c > 0 && k < deep) {
      if (cap <= kStaged) s_seg[e] = (unsigned short)v.seg_len[s];  // (a table has at most 65535 entries then)
      w.off[e] = s < kCached ? (int)atomicAdd(&s_src[s], (unsigned)c) : atomicAdd(&w.seg_cnt[s], c);
    }
  }
  const bool staged = cap <= kStaged && v.max_pages < 65536;
  __syncthreads();
  // Drafted tokens of segment s; until its tiles are noted beside them.
  auto seg_count = [&](int s) { return s < kCached ? (int)s_src[s] : w.seg_cnt[s]; };
  auto depth_pages = [&](int k) {  // pages of this slot's k-th segment
    return staged ? (int)s_seg[b * kMaxSegDepth + k] : v.seg_len[v.seg_bid[b * kMaxSegDepth + k]];
  };
  auto depth_tiles = [&](int k) { return (depth_pages(k) * v.P + flash::kTok - 1) / flash::kTok; };
  auto unit_cost = [&](int rows, int tiles, int rec) {  // of `rows` tokens over `tiles` tiles
    const int full = rows >> shift, rest = rows & ((1 << shift) - 1), halves = 2 * full + (rest > 0) + (rest > 1 << shift >> 1);
    return (int)((long long)halves * (tiles * kTileCost + kUnitCost + rec) >> coarse);
  };
  // Cost of the beams' own units by depth, for the beams that reach it; then the segments'.
  {
    int at = 0;
    if (cnt > 0) {
      int before = unit_cost(cnt, tail_tiles(L), 0);
      atomicAdd(&s_cost[0], before);
#pragma unroll 1
      for (int k = 0; k < nd; ++k) {
        // What using the k-th segment too changes: a shorter rest, and for the first one a record.
        at += depth_pages(k) * v.P;
        const int after = unit_cost(cnt, tail_tiles(L - at), kRecCost);
        atomicAdd(&s_cost[k + 1], after - before);
        before = after;
      }
    }
  }
#pragma unroll 1
  for (int s = tid; s < nseg; s += kListThreads) {
    const int c = seg_count(s);
    if (c > 0) atomicAdd(&s_cost[seg_depth(s) + 1], unit_cost(c, own_tiles(s), kRecCost));
  }
  int dmax = 0, all;
  __syncthreads();
  {
    int cost = s_cost[0], best = cost;
    for (int d = 1; d <= kMaxSegDepth; ++d) {
      cost += s_cost[d];
      if (cost < best) {
        best = cost;
        dmax = d;
      }
    }
  }
#pragma unroll 1
  for (; (dmax + 1) * cap > w.rec_cap && dmax > 0; --dmax) {  // a record each, and one for the rest, must fit
    block_exclusive_scan(cnt > 0 ? min(nd, dmax) + 1 : 0, sm.tmp, &all);
    if (all <= w.rec_cap) break;
  }
  nd = min(nd, dmax);
  int start = 0;
  for (int k = 0; k < nd; ++k) start += depth_pages(k) * v.P;
  const int tail = cnt > 0 ? tail_tiles(L - start) : 0;
  auto up = [&](int rows, int sh) { return (rows + (1 << sh) - 1) >> sh; };
  // Few units of 128 rows: that many rows to a unit, and one unit per SM (two shorter ones leave SMs idle in the second
  // wave: a 20000-token beam of 8 KV heads in 256 units of 5 tiles took as long as 144 of 9 would in two waves).
  int whole = up(cnt, small), work = tail * up(cnt, shift), work_few = tail * whole;
#pragma unroll 1
  for (int s = tid; s < nseg; s += kListThreads) {
    const int c = seg_depth(s) < dmax ? seg_count(s) : 0, t = own_tiles(s);
    if (s < kCached) s_src[s] = (unsigned)min(c, 65535) | (unsigned)min(t, 65535) << 16;
    if (s >= kCached || c >= 65535) w.seg_cnt[s] = c;
    whole += up(c, small);
    work += t * up(c, shift);
    work_few += t * up(c, small);
    if (c > 0) w.seg_list[s] = atomicAdd(&s_sum[kSumList], c);
  }
  work = __reduce_add_sync(0xffffffffu, work);
  work_few = __reduce_add_sync(0xffffffffu, work_few);
  if ((tid & 31) == 0) {
    atomicAdd(&s_sum[kSumWork], work);
    atomicAdd(&s_sum[kSumWorkFew], work_few);
  }
  const bool few = (long long)block_sum(whole, &s_sum[kSumFew]) * v.Hkv <= v.num_sms;
  if (few) shift = small;
  const int tokens = 1 << shift;
  struct Source {
    int rows, tiles;
  };
  auto segment = [&](int s) {  // rows 0: not used
    const unsigned x = s < kCached ? s_src[s] : ~0u;
    Source r;
    r.rows = (x & 0xffff) == 0xffff ? w.seg_cnt[s] : x & 0xffff;
    r.tiles = r.rows == 0 ? 0 : x >> 16 == 0xffff ? seg_tiles(s) : x >> 16;
    return r;
  };
  // Tiles per unit: half an SM's share at most, which the sorted list evens out, but not too short ones, and no more
  // records than there is room for.
  const int share = (few ? 1 : 2) * v.num_sms;
  all = s_sum[few ? kSumWorkFew : kSumWork];
  constexpr int kLongest = 1 << 20;  // no run of keys has more tiles
  int mine, base, per = min(kLongest, max(least, (int)(((long long)all * v.Hkv + share - 1) / share)));
  float inv;  // 1 / per, for quotients of counts of tiles: (x + 1/2) / per is at least 1 / (2 per) from a whole number, more than its error
  auto pieces = [&](int tiles) { return (int)(((float)(tiles + per - 1) + 0.5f) * inv); };
  inv = 1.f / (float)per;
#pragma unroll 1
  for (int k = 0; few; ++k) {  // until the pieces fit too
    if (k == kFewTries) {      // (a piece each does)
      per = kLongest;
      inv = 1.f / (float)per;
      break;
    }
    int n = up(cnt, shift) * pieces(tail);
    for (int s = tid; s < nseg; s += kListThreads) {
      const Source r = segment(s);
      n += up(r.rows, shift) * pieces(r.tiles);
    }
    if ((long long)block_sum(n, &s_sum[kSumTry + k]) * v.Hkv <= v.num_sms) break;
    per += 1 + per / 8;
    inv = 1.f / (float)per;
  }
  if (tid == 0) {
    w.ctl[kDrFew] = few;
    w.ctl[kDrChanges] = v.ctl[kCtlChanges];
    *reinterpret_cast<unsigned long long*>(w.ctl + kDrToken) = w.token;
  }
#pragma unroll 1
  for (;;) {
    mine = cnt > 0 ? pieces(tail) : 0;
    for (int k = 0; k < nd; ++k) mine += pieces(depth_tiles(k));
    base = block_exclusive_scan(mine, sm.tmp, &all);
    if (all <= w.rec_cap || per >= kLongest) break;
    per *= 2;
    inv = 1.f / (float)per;
  }
  int tail_rec = 0;
  if (b < cap) {
    w.nrec[b] = mine;
    w.rec_base[b] = base;
    for (int k = 0; k < nd; ++k) {
      w.rec_off[b * kRecOffs + k] = tail_rec;
      tail_rec += pieces(depth_tiles(k));
    }
    w.rec_off[b * kRecOffs + kTailRec] = tail_rec;
    w.depth[b] = nd;
  }
  // The beams' own sizes, for the list's other threads.
  __shared__ int s_rec[kMaxBeams];
  s_start[b] = start;
  s_len[b] = L;
  s_rec[b] = mine > 1 ? base + tail_rec : -1;
  __syncthreads();
  struct Piece {
    int tiles, splits, share, row_tiles, rows;
  };
  auto piece = [&](int src) {  // sources: the segments, then the slots
    Piece p;
    if (src >= nseg) {
      p.rows = s_cnt[src - nseg];
      p.tiles = p.rows > 0 ? tail_tiles(s_len[src - nseg] - s_start[src - nseg]) : 0;
    } else {
      const Source r = segment(src);
      p.rows = r.rows;
      p.tiles = r.tiles;
    }
    p.splits = pieces(p.tiles);
    p.share = p.splits > 1 ? (p.tiles + p.splits - 1) / p.splits : max(p.tiles, 1);
    p.row_tiles = up(p.rows, shift);
    return p;
  };
  const int n = emit_sorted(
      sm, nseg + cap,
      [&](int src) {
        const Piece p = piece(src);
        return p.splits * p.row_tiles;
      },
      [&](int src, int i) {
        const Piece p = piece(src);
        const int sp = p.row_tiles == 1 ? i : i / p.row_tiles, t = i - sp * p.row_tiles;
        const int rows = min(tokens, p.rows - t * tokens);
        return (min(p.share, p.tiles - sp * p.share) + 1) * (2 * rows > tokens ? 2 : 1);
      },
      [&](int src, int i, int at) {
        if (at >= w.max_units) return;
        const Piece p = piece(src);
        const int sp = p.row_tiles == 1 ? i : i / p.row_tiles, t = i - sp * p.row_tiles;
        const int rows = max(0, min(tokens, p.rows - t * tokens));
        DraftUnit u;
        u.ntok = rows;
        if (src < nseg) {
          const int len = v.seg_len[src] * v.P, first = v.seg_i0[src] * v.P;
          u.seg = src;
          u.beam = v.seg_rep[src];
          u.e0 = w.seg_list[src] + t * tokens;
          u.tok0 = first + sp * p.share * flash::kTok;
          u.tok1 = first + min((sp + 1) * p.share * flash::kTok, len);
          u.drafts = 0;
          u.rec = sp;
        } else {
          const int beam = src - nseg, n = s_len[beam];
          u.seg = -1;
          u.beam = beam;
          u.e0 = t * tokens;
          u.tok0 = min(s_start[beam] + sp * p.share * flash::kTok, n);
          u.tok1 = min(s_start[beam] + (sp + 1) * p.share * flash::kTok, n);
          u.drafts = sp == p.splits - 1 ? s_cnt[beam] : 0;
          u.rec = s_rec[beam] < 0 ? -1 : s_rec[beam] + sp;
        }
        w.units[at] = u;
      });
  if (tid == 0) w.ctl[kDrUnits] = min(n, w.max_units);
  if (cap <= kOneLaunch) {
    __threadfence_block();
    __syncthreads();
    draft_rows(v, w, parent, count, tid >> 5, kListThreads / 32);
  }
}

// A CTA for eight slots.  Latency: 7 us alone, about 3 behind the plan.
__global__ void __launch_bounds__(256) k_draft_rows(PoolView v, DraftView w, const int* parent, const int* count) {
  pdl_wait();
  pdl_launch_dependents();
  draft_rows(v, w, parent, count, blockIdx.x * 8 + (threadIdx.x >> 5), gridDim.x * 8);
}

// Where a row's result goes: the output itself when the beam has one record, else its record.
struct DraftRow {
  int beam, tok, rec;  // rec: the record, or -1 for the output
  bool valid;
};
// Row of entry e of a segment's token list, or of a beam's own token e.
__device__ __forceinline__ DraftRow draft_row(const DraftView& w, int seg, int beam, int e, int rec, bool valid) {
  if (!valid || seg < 0) return {beam, valid ? e : 0, rec, valid};
  const int2 x = w.list[e];  // a beam with a segment has a record of its own units too
  return {x.x & 1023, x.x >> 10, x.y + rec, true};
}

struct DraftJob {
  CUtensorMap tp, tk, tv;  // the pool's pages; the drafted keys and values
  PoolView v;
  DraftView w;
  int layer, oob;
  int page_shift, group0;   // log2 of the page size; the layer's first row group in the tensor map
  float qscale;
  const __nv_bfloat16 *q, *k, *vv;  // this layer's [max_beams][T][heads][128]
  __nv_bfloat16* o;

  static constexpr uint64_t kWaitNs = kWaitLimitNs;
  static constexpr bool kEarlyQ = true;
  // 64 traces x 4k 260 -> 240 us, 198 x 8k 295 -> 265; from two tiles on, 128 traces of 2 and 3 tiles a unit 1663 -> 1736 us.
  static constexpr int kLongPair = 4;
  static constexpr int kQArrivals = 4;
  // Tiles land as [16 groups of 8 tokens][half of D][8][64 dims].
  static constexpr int kKHalf = 1024, kKSbo = 2048, kVLbo = 1024, kVSbo = 2048, kVStep = 4096;
  static __device__ __forceinline__ int v_row(int row, int half) {
    return (row >> 3) * 2048 + half * 1024 + (row & 7) * 128;
  }

  struct Row : DraftRow {
    int gg;  // query head of the KV head
    unsigned long long anc;
  };

  __device__ __forceinline__ void error(int code) const { set_status(v.ctl, code); }
  struct Units {
    int count, few;
    __device__ __forceinline__ explicit Units(const DraftJob& j) : count(j.w.ctl[kDrUnits]), few(j.w.ctl[kDrFew]) {
      count = plan_holds(j.v, j.w) ? count : 0;
    }
  };
  // A warp that has nothing to do yet, once what came before has completed.
  __device__ __forceinline__ void begun() const {
    if (blockIdx.x == 0 && !plan_holds(v, w)) spoil_plan(v, w);
  }
  // Which rows share a unit, and where it stands in the list, follows the order in which segments were found, which may
  // differ from run to run: a row's result may not depend on it.  Where there are few units all of more than a tile are joint.
  __device__ __forceinline__ bool joins(const Units& all) const { return all.few != 0; }
  __device__ __forceinline__ int total(const Units& all) const { return all.count * v.Hkv; }
  __device__ __forceinline__ int capacity() const { return w.max_units * v.Hkv; }
  // Words of a unit, those of its loads first.
  enum { kBeam, kTok0, kTok1, kDrafts, kSeg, kE0, kNtok, kRec };
  __device__ __forceinline__ void unit(const Units&, int id, flash::Unit& x) const {
    const DraftUnit e = w.units[id / v.Hkv];
    const int n = e.tok1 - e.tok0;
    x.head = id % v.Hkv;
    x.nt = e.drafts ? tail_tiles(n) : (n + flash::kTok - 1) / flash::kTok;
    x.mode = e.ntok * v.G > flash::kRows ? flash::kDual : flash::kJoint;
    x.w[kSeg] = e.seg;
    x.w[kBeam] = e.beam;
    x.w[kE0] = e.e0;
    x.w[kNtok] = e.ntok;
    x.w[kTok0] = e.tok0;
    x.w[kTok1] = e.tok1;
    x.w[kDrafts] = e.drafts;
    x.w[kRec] = e.rec;
  }
  __device__ __forceinline__ bool draft_tile(const flash::Unit& x, int j) const { return x.w[kDrafts] && j == x.nt - 1; }
  // Rows of the context's last page past its end, and the drafted rows that are loaded (by eights) but lie past the count.
  __device__ __forceinline__ uint32_t stale_rows(const flash::Unit& x, int j) const {
    const int n = x.w[kTok1] - x.w[kTok0] - j * flash::kTok;
    const int page = n > 0 && n < flash::kTok ? -n & (v.P - 1) : 0;
    const int drafts = draft_tile(x, j) ? min(w.T - x.w[kDrafts], -x.w[kDrafts] & 7) : 0;
    return page + drafts > 0 ? flash::stale_word(n & 127, page, 64 + x.w[kDrafts], drafts) : 0;
  }
  // Evicted first: a layer's keys and values are read once or by units that run side by side, and should not push the records
  // that the join reads next out of the L2 (64 beams x 4k 284 -> 277 us, one beam of 20000 tokens 76 -> 70).
  static __device__ __forceinline__ void tma5(uint32_t dst, const CUtensorMap* tm, int c1, int c2, int c3, int c4,
                                              uint32_t bar) {
    uint64_t pol;
    asm("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(pol));
    asm volatile(
        "cp.async.bulk.tensor.5d.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1, {%2, %3, %4, %5, %6}], [%7], %8;" ::"r"(
            dst),
        "l"(tm), "r"(0), "r"(c1), "r"(c2), "r"(c3), "r"(c4), "r"(bar), "l"(pol)
        : "memory");
  }
  // The lane's page of tile j: its first row group in the pool's tensor map, or one past it (zeros).
  __device__ __forceinline__ int page(const flash::Unit& x, int j, int lane) const {
    const int pos = x.w[kTok0] + j * flash::kTok + (lane << page_shift);
    if ((lane << page_shift) >= flash::kTok || pos >= x.w[kTok1]) return oob;
    int p = v.tables[(size_t)x.w[kBeam] * v.max_pages + (pos >> page_shift)];
    if (p < 0 || p >= v.num_pages) {
      set_status(v.ctl, GB_ERR_INVALID);
      p = 0;
    }
    return group0 + x.head * (v.P / 8) + p * (2 * v.Hkv * v.P / 8);
  }
  // A page to a lane: the copies' issue overlaps.
  __device__ __forceinline__ void load_tile(const flash::Unit& x, int j, int kv, int page, uint32_t dst, uint32_t bar,
                                            int lane) const {
    const bool last = draft_tile(x, j);
    if ((lane << page_shift) < (last ? 64 : flash::kTok)) tma5(dst + (lane << (page_shift + 8)), &tp, 0, 0, kv, page, bar);
    if (last && lane >= 16 && lane < 24) {
      const int t = (lane - 16) * 8;
      tma5(dst + (lane - 8) * 2048, kv ? &tv : &tk, t < x.w[kDrafts] ? t : kMaxDraft, 0, x.head, x.w[kBeam], bar);
    }
  }
  __device__ __forceinline__ void find_row(const flash::Unit& x, int g, int r, Row& row) const {
    const int i = (x.mode == flash::kDual ? g * flash::kRows + r : r) / v.G;
    static_cast<DraftRow&>(row) = draft_row(w, x.w[kSeg], x.w[kBeam], x.w[kE0] + i, x.w[kRec], i < x.w[kNtok]);
    row.gg = r % v.G;
    row.anc = row.valid && x.w[kDrafts] ? w.anc[(size_t)row.beam * w.T + row.tok] : 0ull;
  }
  __device__ __forceinline__ void load_q(const flash::Unit& x, int g, int r, uint32_t dst, uint32_t bar,
                                         const Row& row) const {
    // Half a warp to a row, so that a copy of the warp meets four lines (a row to a thread met 32).
    const int lane = r & 31, c = lane & 15;
    const unsigned long long mine = reinterpret_cast<unsigned long long>(
        q + (((size_t)row.beam * w.T + row.tok) * v.Hq + x.head * v.G + row.gg) * flash::kD);
    const unsigned there = __ballot_sync(0xffffffffu, row.valid);
#pragma unroll
    for (int i = 0; i < 32; i += 2) {
      const int l = i + (lane >> 4);
      const char* src = reinterpret_cast<const char*>(__shfl_sync(0xffffffffu, mine, l)) + 16 * c;
      const uint32_t to = dst + (c >> 3) * 16384 + swz((r & ~31) + l, (c & 7) * 8);
      if ((there >> l) & 1)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(src) : "memory");
      else
        asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(to), "r"(0) : "memory");
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  }
  __device__ __forceinline__ void loaded_q(int r, uint32_t bar) const {
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    fence_proxy_async_smem();
    __syncwarp();
    if ((r & 31) == 0) mbar_arrive(bar);
  }
  __device__ __forceinline__ flash::Sees sees(const flash::Unit& x, const Row& row, int t) const {
    const int n = x.w[kTok1] - x.w[kTok0] - t * flash::kTok;
    const bool last = draft_tile(x, t);
    return {!last && n >= flash::kTok, last, n, row.anc};
  }
  template <class Done>
  __device__ __forceinline__ void out(const flash::Unit& x, const Row& row, uint32_t a, uint32_t b, bool two, float wa,
                                      float wb, float m, float l, Done done, volatile int* again) const {
    const bool final = row.rec < 0;
    const float inv = final ? 1.f / l : 1.f;
    const int head = x.head * v.G + row.gg;
    __nv_bfloat16* dst = o + (((size_t)row.beam * w.T + row.tok) * v.Hq + head) * flash::kD;
    const size_t rr = ((size_t)max(row.rec, 0) * v.Hkv + x.head) * w.rows + row.tok * v.G + row.gg;
    float* rec = w.rec + rr * flash::kD;
    bool fine = true;
    flash::walk_o(
        a, b, two, wa, wb,
        [&](int c, auto count, float* f) {
          constexpr int N = decltype(count)::value;
#pragma unroll
          for (int i = 0; i < N; ++i) {
            f[i] *= inv;
            fine = fine && isfinite(f[i]);
          }
          if (!row.valid) return;
          if (final) {
            uint32_t u[N / 2];
#pragma unroll
            for (int k = 0; k < N / 2; ++k) {
              const __nv_bfloat162 p = __floats2bfloat162_rn(f[2 * k], f[2 * k + 1]);
              u[k] = *reinterpret_cast<const uint32_t*>(&p);
            }
#pragma unroll
            for (int k = 0; k < N / 2; k += 8) flash::st32(dst + c + 2 * k, u + k);
          } else {
#pragma unroll
            for (int k = 0; k < N; k += 8) flash::st32(rec + c + k, reinterpret_cast<const uint32_t*>(f + k));
          }
        },
        done);
    if (row.valid && !final) w.ml[rr] = make_float2(m, l);
    if (row.valid && x.w[kDrafts] && !fine && isfinite(m) && isfinite(l)) *again = 1;
  }
  // Rows that only met a value that is not finite in drafted tokens off their path, which alone share a tile with what they
  // see; a row to a warp (see flash::one_row).
  __device__ __forceinline__ void again(const flash::Unit& x, int warp) const {
    if (!x.w[kDrafts]) return;
    const int lane = threadIdx.x & 31, nctx = x.w[kTok1] - x.w[kTok0];
    auto drafted_row = [&](const __nv_bfloat16* of, int i) {
      return of + (((size_t)x.w[kBeam] * w.T + i) * v.Hkv + x.head) * flash::kD;
    };
    unsigned long long odd = 0;  // tokens whose V is not finite
    bool looked = false;
#pragma unroll 1
    for (int i = warp; i < x.w[kNtok] * v.G; i += flash::kKWarp) {
      Row row;
      find_row(x, i / flash::kRows, i % flash::kRows, row);
      const size_t qo = (((size_t)row.beam * w.T + row.tok) * v.Hq + x.head * v.G + row.gg) * flash::kD;
      const size_t rr = ((size_t)max(row.rec, 0) * v.Hkv + x.head) * w.rows + row.tok * v.G + row.gg;
      bool bad;
      if (row.rec < 0) {
        const uint2 y = reinterpret_cast<const uint2*>(o + qo)[lane];
        bad = flash::not_finite(y.x) || flash::not_finite(y.y);
      } else {
        const float4 y = reinterpret_cast<const float4*>(w.rec + rr * flash::kD)[lane];
        bad = !(isfinite(y.x) && isfinite(y.y) && isfinite(y.z) && isfinite(y.w));
      }
      if (!__any_sync(0xffffffffu, bad)) continue;
      if (!looked) {
        looked = true;
        for (int t = 0; t < 64; t += 32)
          odd |= (unsigned long long)__ballot_sync(0xffffffffu, t + lane < x.w[kDrafts] && flash::not_finite(drafted_row(vv, t + lane))) << t;
      }
      if (!(odd & ~row.anc)) continue;
      float m, l, acc[4];
      if (!flash::one_row(
              q + qo, nctx + x.w[kDrafts],
              [&](int j, int kv, const __nv_bfloat16*& to) {
                if (j >= nctx) {
                  to = drafted_row(kv ? vv : k, j - nctx);
                  return ((row.anc >> (j - nctx)) & 1) != 0;
                }
                const int pos = x.w[kTok0] + j, page = v.tables[(size_t)x.w[kBeam] * v.max_pages + pos / v.P];
                to = reinterpret_cast<const __nv_bfloat16*>(v.kv) + kv_elem_offset(v, layer, page, kv, x.head, pos % v.P);
                return page >= 0 && page < v.num_pages;
              },
              qscale, m, l, acc))
        continue;
      if (row.rec < 0) {
        for (int c = 0; c < 4; ++c) o[qo + 4 * lane + c] = __float2bfloat16(acc[c] / l);
      } else {
        reinterpret_cast<float4*>(w.rec + rr * flash::kD)[lane] = make_float4(acc[0], acc[1], acc[2], acc[3]);
        if (lane == 0) w.ml[rr] = make_float2(m, l);
      }
    }
  }
  __device__ __forceinline__ void drain_q(uint32_t) const { asm volatile("cp.async.wait_all;" ::: "memory"); }
};

// A CTA per SM; what bounds it and its figures: the file's head, and flash.cuh for the split.
__global__ void __launch_bounds__(flash::kThreads, 1) k_draft(const __grid_constant__ DraftJob job) {
  extern __shared__ __align__(1024) unsigned char sm[];
  flash::body(job, sm);
}

// fp32: a CTA per (unit, KV head).
struct DraftTile {
  const PoolView& v;
  const DraftView& w;
  const DraftUnit& u;
  int layer, head, nctx;
  const float *qp, *kp, *vp;
  float* op;
  __device__ __forceinline__ int tok(int r) const { return u.e0 + r / v.G; }
  __device__ __forceinline__ bool valid(int r) const { return r / v.G < u.ntok; }
  __device__ __forceinline__ size_t row(int r) const {
    return (((size_t)u.beam * w.T + tok(r)) * v.Hq + head * v.G + r % v.G) * kTileD;
  }
  __device__ __forceinline__ const float* q(int r) const { return valid(r) ? qp + row(r) : nullptr; }
  __device__ __forceinline__ const float* token(int j, int kv) const {
    if (j >= nctx) return (kv ? vp : kp) + (((size_t)u.beam * w.T + j - nctx) * v.Hkv + head) * kTileD;
    const int pos = u.tok0 + j, page = v.tables[(size_t)u.beam * v.max_pages + pos / v.P];
    if (page < 0 || page >= v.num_pages) {
      set_status(v.ctl, GB_ERR_INVALID);
      return nullptr;
    }
    return reinterpret_cast<const float*>(v.kv) + kv_elem_offset(v, layer, page, kv, head, pos % v.P);
  }
  __device__ __forceinline__ const float* key(int j) const { return token(j, 0); }
  __device__ __forceinline__ const float* val(int j) const { return token(j, 1); }
  __device__ __forceinline__ TileSees sees(int r) const {
    return {nctx, nctx, valid(r) ? w.anc[(size_t)u.beam * w.T + tok(r)] : 0ull};
  }
  __device__ __forceinline__ void out(int r, int c, float4 x, float m, float l) const {
    if (!valid(r)) return;
    const DraftRow d = draft_row(w, -1, u.beam, tok(r), u.rec, true);
    if (d.rec < 0) {
      const float inv = 1.f / l;
      *reinterpret_cast<float4*>(op + row(r) + c) = make_float4(x.x * inv, x.y * inv, x.z * inv, x.w * inv);
    } else {
      const size_t rr = ((size_t)d.rec * v.Hkv + head) * w.rows + tok(r) * v.G + r % v.G;
      *reinterpret_cast<float4*>(w.rec + rr * kTileD + c) = x;
      if (c == 0) w.ml[rr] = make_float2(m, l);
    }
  }
};

__global__ void __launch_bounds__(kTileThreads, 1) k_draft_f32(PoolView v, DraftView w, int layer, const float* q,
                                                            const float* k, const float* vv, float* o, float qscale) {
  pdl_wait();
  pdl_launch_dependents();
  extern __shared__ __align__(16) unsigned char raw[];
  TileSmem& sm = *reinterpret_cast<TileSmem*>(raw);
  const bool holds = plan_holds(v, w);
  if (!holds && blockIdx.x == 0 && threadIdx.x < 32) spoil_plan(v, w);
  const int total = holds ? w.ctl[kDrUnits] * v.Hkv : 0;
  for (int id = blockIdx.x; id < total; id += gridDim.x) {
    const DraftUnit u = w.units[id / v.Hkv];
    const int nctx = u.tok1 - u.tok0;
    const DraftTile src{v, w, u, layer, id % v.Hkv, nctx, q, k, vv, o};
    tile_attention(sm, src, nctx + u.drafts, qscale);
    __syncthreads();
  }
}

// A CTA per (slot, token), or one for every 8 of its query heads where those are few, a warp per row: joins the row's
// records, sum 2^(m_k - m) (o_k, l_k), or writes the zeros of a row that holds no token; a row that has its result
// already is left.  Bound by the records' reads; many small CTAs (a third as many, looping: 128 beams of short contexts 46
// -> 51 us a layer).
// kBatch records at a time: 4 where there are many CTAs, whose registers then let more of them run (48 instead of 74; 64 beams
// x 4k 269 -> 260 us, a 36-layer round 1700 -> 1674), 8 where there are few (one beam of 20000 tokens 71 us, 74 with 4).
template <typename T, int D, int kBatch>
__global__ void __launch_bounds__(256) k_draft_merge(PoolView v, DraftView w, T* o) {
  pdl_wait();
  pdl_launch_dependents();
  constexpr int per = D / 32;
  using Vec = typename std::conditional<per == 4, float4, float2>::type;
  const int lane = threadIdx.x & 31, i = blockIdx.x, b = blockIdx.y;
  const int there = w.cnt[b], records = w.nrec[b];  // (loaded together)
  const int n = i < there ? records : 0;
  if (n == 1) return;
  const size_t step = (size_t)v.Hkv * w.rows;
  const size_t r1 = n > 0 ? (size_t)w.rec_base[b] * step + i * v.G : 0;
  for (int hq = blockIdx.z * 8 + (threadIdx.x >> 5); hq < v.Hq; hq += 8 * gridDim.z) {
    float acc[per] = {};
    if (n > 0) {
      const size_t r0 = r1 + (size_t)(hq / v.G) * w.rows + hq % v.G;
      float m = -INFINITY;
      for (int k = lane; k < n; k += 32) m = fmaxf(m, w.ml[r0 + k * step].x);
#pragma unroll
      for (int s = 16; s > 0; s >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, s));
      const float ref = m == -INFINITY ? 0.f : m;
      float l = 0.f;
      for (int k0 = 0; k0 < n; k0 += 32) {
        // Lane k has the weight of record k0 + k, so that the records' loads wait for nothing but their addresses.
        float2 ml = make_float2(-INFINITY, 0.f);
        if (k0 + lane < n) ml = w.ml[r0 + (k0 + lane) * step];
        const float f = exp2f(ml.x - ref);
        l = fmaf(ml.y, f, l);
        const int m32 = min(32, n - k0);
        const Vec* x = reinterpret_cast<const Vec*>(w.rec + (r0 + k0 * step) * D) + lane;
#pragma unroll 1
        for (int k = 0; k < m32; k += kBatch) {
          Vec y[kBatch];
#pragma unroll
          for (int e = 0; e < kBatch; ++e)
            if (k + e < m32) y[e] = x[(size_t)(k + e) * step * 32];
#pragma unroll
          for (int e = 0; e < kBatch; ++e) {
            const float g = __shfl_sync(0xffffffffu, f, (k + e) & 31);
            if (k + e < m32)
#pragma unroll
              for (int c = 0; c < per; ++c) acc[c] = fmaf(reinterpret_cast<const float*>(&y[e])[c], g, acc[c]);
          }
        }
      }
#pragma unroll
      for (int s = 16; s > 0; s >>= 1) l += __shfl_xor_sync(0xffffffffu, l, s);
      const float inv = 1.f / l;
#pragma unroll
      for (int c = 0; c < per; ++c) acc[c] *= inv;
      // The records are done with: lines still in the L2 need not reach memory (64 beams x 4k 277 -> 266 us, 198 x 8k 314 -> 300).
      __syncwarp();
      constexpr int lines = D * 4 / 128;
      const float* r = w.rec + (r0 + lane / lines * step) * D + lane % lines * 32;
#pragma unroll 1
      for (int k = lane / lines; k < n; k += 32 / lines, r += 32 / lines * step * D)
        asm volatile("discard.global.L2 [%0], 128;" ::"l"(r) : "memory");
    }
    T* dst = o + (((size_t)b * w.T + i) * v.Hq + hq) * D + lane * per;
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int c = 0; c < per; c += 2)
        *reinterpret_cast<__nv_bfloat162*>(dst + c) = __floats2bfloat162_rn(acc[c], acc[c + 1]);
    } else {
      *reinterpret_cast<Vec*>(dst) = *reinterpret_cast<const Vec*>(acc);
    }
  }
}

// ---------------------------------------------------------------------------
// Accepting a path
// ---------------------------------------------------------------------------

// One CTA, thread = slot.  The rule of a step that appends one token after another, each to the slots whose
// path is that long: lowest free page first, slots ascending; a partial tail page that others still hold is
// left to them and copied.  All or nothing.  Latency: 10 to 12 us for 16 to 128 slots.
__global__ void __launch_bounds__(1024) k_accept_plan(PoolView v, DraftView w, const int* parent, const int* count,
                                                      const int* accepted, int* n_out, int* path_out) {
  pdl_wait();
  pdl_launch_dependents();
  constexpr int kMaxNeeds = kMaxDraft / 16 + 1;  // pages a slot can need
  __shared__ int tmp[33];
  __shared__ unsigned long long s_path[kMaxBeams];
  __shared__ int s_tail[kMaxBeams];
  __shared__ unsigned s_bits[kMaxDraft][kMaxBeams / 32];  // slots that need a page with their k-th token
  __shared__ int s_first[kMaxDraft];                      // needs of earlier tokens
  __shared__ int s_pages[kMaxBeams * kMaxNeeds];
  const int tid = threadIdx.x, b = tid, lane = tid & 31;
  const int nodes = v.max_beams * w.T;
  const bool staged = nodes <= kMaxBeams * kMaxNeeds;
  if (staged) {  // the trees fit in shared memory (in s_pages, before its use): a thread walks its slot's path up
    for (int i = tid; i < nodes; i += 1024) s_pages[i] = parent[i];
    bool bad = false;
    const bool on = b < v.max_beams && v.active[b] != 0;
    const int n = b < v.max_beams ? drafted(count, b, w.T, on, &bad) : 0, to = on ? accepted[b] : -1;
    __syncthreads();
    unsigned long long p = 0;
    bool odd = to < -1 || to >= n;
    for (int i = 0; i < n; ++i) odd |= s_pages[b * w.T + i] < -1 || s_pages[b * w.T + i] >= i;
    for (int i = odd ? -1 : to; i >= 0; i = s_pages[b * w.T + i]) p |= 1ull << i;
    if (b < v.max_beams) s_path[b] = p;
    if (odd || bad) set_status(v.ctl, GB_ERR_INVALID);
  }
  // Larger ones: a warp per slot.
  for (int s = tid >> 5; s < (staged ? 0 : v.max_beams); s += 32) {
    bool bad = false, wrong;
    const int n = drafted(count, s, w.T, v.active[s] != 0, &bad), to = v.active[s] ? accepted[s] : -1;
    unsigned long long lo, hi;
    ancestors(parent + (size_t)s * w.T, w.T, n, &lo, &hi, &wrong);
    const bool odd = wrong || to < -1 || to >= n;
    const unsigned long long p = __shfl_sync(0xffffffffu, to < 32 ? lo : hi, max(to, 0) & 31);
    if (lane == 0) {
      s_path[s] = odd || to < 0 ? 0ull : p;
      if (odd || bad) set_status(v.ctl, GB_ERR_INVALID);
    }
  }
  for (int i = tid; i < kMaxDraft * (kMaxBeams / 32); i += 1024) (&s_bits[0][0])[i] = 0;
  __syncthreads();
  const bool act = b < v.max_beams && v.active[b] != 0;
  unsigned long long path = act ? s_path[b] : 0ull;
  int n = __popcll(path);
  const int L = act ? v.seq_len[b] : 0;
  // Copy-on-write: a slot that appends leaves a tail page that another still holds after the lower
  // slots have left it.
  int tail = -1;
  if (n > 0 && L % v.P && v.ctl[kCtlTailShared]) tail = v.tables[(size_t)b * v.max_pages + L / v.P];
  s_tail[b] = tail;
  __syncthreads();
  bool cow = false;
  if (tail >= 0) {
    int before = 0;
    const int R = v.refcnt[tail];
    if (R > 1)
      for (int s = 0; s < b; ++s) before += s_tail[s] == tail;
    cow = R - before > 1;
  }
  const int first_new = (L + v.P - 1) / v.P;
  const int fresh = n > 0 ? max(0, (L + n - 1) / v.P - first_new + 1) : 0;
  const int need = fresh + (cow ? 1 : 0);
  const bool too_long = n > 0 && (L + n - 1) / v.P >= v.max_pages;
  int total;
  block_exclusive_scan(need, tmp, &total);
  const bool fails = __syncthreads_or(too_long) || total > v.ctl[kCtlFree];
  if (fails) {
    if (tid == 0) set_status(v.ctl, GB_ERR_OOM);
    n = 0;
    path = 0;
    cow = false;
    total = 0;
  } else {
    if (cow) atomicOr(&s_bits[0][b >> 5], 1u << (b & 31));
    for (int j = 0; j < fresh; ++j) atomicOr(&s_bits[(first_new + j) * v.P - L][b >> 5], 1u << (b & 31));
  }
  __syncthreads();
  // The r-th need, token by token and slots ascending, gets the r-th lowest free page.
  {
    int c = 0;
    if (tid < kMaxDraft)
      for (int i = 0; i < kMaxBeams / 32; ++i) c += __popc(s_bits[tid][i]);
    int all;
    const int at = block_exclusive_scan(c, tmp, &all);
    if (tid < kMaxDraft) s_first[tid] = at;
  }
  int found = 0, w0 = max(v.ctl[kCtlCursor], 0);
  __syncthreads();
  while (found < total && w0 < v.words) {
    const int word = w0 + tid;
    unsigned bits = word < v.words ? v.free_bits[word] : 0u;
    if (word == v.words - 1 && (v.num_pages & 31)) bits &= (1u << (v.num_pages & 31)) - 1u;
    int here;
    int r = found + block_exclusive_scan(__popc(bits), tmp, &here);
    const unsigned before = bits;
    while (bits && r < total) {
      s_pages[r] = word * 32 + __ffs(bits) - 1;
      bits &= bits - 1u;
      if (++r == total) v.ctl[kCtlCursor] = word;
    }
    if (bits != before) v.free_bits[word] = (v.free_bits[word] & ~before) | bits;
    found += here;
    w0 += 1024;
  }
  __syncthreads();
  if (tid == 0 && total > 0) v.ctl[kCtlFree] -= total;
  auto page_of = [&](int k) {
    int r = s_first[k] + __popc(s_bits[k][b >> 5] & ((1u << (b & 31)) - 1u));
    for (int i = 0; i < (b >> 5); ++i) r += __popc(s_bits[k][i]);
    return s_pages[r];
  };
  if (!fails) {
    if (tid == 0) v.ctl[kCtlChanges] += 1;
    if (cow) {
      const int p = page_of(0);
      atomicSub(&v.refcnt[tail], 1);
      v.refcnt[p] = 1;
      v.tables[(size_t)b * v.max_pages + L / v.P] = p;
    }
    for (int j = 0; j < fresh; ++j) {
      const int p = page_of((first_new + j) * v.P - L);
      v.refcnt[p] = 1;
      v.tables[(size_t)b * v.max_pages + first_new + j] = p;
    }
  }
  if (b < v.max_beams) {
    w.acc_n[b] = n;
    w.acc_pos[b] = L;
    w.acc_old[b] = cow ? tail : -1;
    w.acc_path[b] = path;
    if (n > 0) {
      v.seq_len[b] = L + n;
      v.gen[b] += n;
    }
    if (n_out) n_out[b] = n;
    if (path_out) {
      int* to = path_out + (size_t)b * w.T;
      for (int i = 0; i < w.T; ++i) {
        to[i] = path ? __ffsll((long long)path) - 1 : -1;
        path &= path - 1;
      }
    }
  }
}

// A CTA per (slot, layer): the rows of a copied tail page, then the path's rows, 16 bytes a thread.  Bound by launch and latency
// for small rounds (8 us: 16 slots, 4 layers), by the copy for large ones (128 slots, 36 layers: 28 us).
__global__ void __launch_bounds__(256) k_accept_copy(PoolView v, DraftView w, const char* k, const char* vv) {
  pdl_wait();
  pdl_launch_dependents();
  __shared__ short s_tok[kMaxDraft];
  const int b = blockIdx.x, layer = blockIdx.y, tid = threadIdx.x;
  const int n = w.acc_n[b];
  if (n == 0) return;
  const int L = w.acc_pos[b], old = w.acc_old[b], rows = v.Hkv * 16;  // 16-byte pieces of a token's K (or V)
  if (tid < 64) {
    const unsigned long long path = w.acc_path[b];
    if ((path >> tid) & 1) s_tok[__popcll(path & ((1ull << tid) - 1))] = (short)tid;
  }
  const int* table = v.tables + (size_t)b * v.max_pages;
  if (old >= 0) {
    const int page = table[L / v.P], have = L % v.P;
    for (int i = tid; i < 2 * v.Hkv * have * 16; i += 256) {
      const int c = i & 15, row = (i >> 4) % have, kvh = (i >> 4) / have;
      const int kv = kvh / v.Hkv, h = kvh % v.Hkv;
      reinterpret_cast<uint4*>(v.kv + kv_elem_offset(v, layer, page, kv, h, row) * v.esize)[c] =
          reinterpret_cast<const uint4*>(v.kv + kv_elem_offset(v, layer, old, kv, h, row) * v.esize)[c];
    }
  }
  __syncthreads();
  const size_t src0 = ((size_t)layer * v.max_beams + b) * w.T * rows;
  for (int i = tid; i < 2 * n * rows; i += 256) {
    const int kv = i >= n * rows, j = kv ? i - n * rows : i, t = j / rows, c = j % rows, pos = L + t;
    const int page = table[pos / v.P];
    if (page < 0 || page >= v.num_pages) {
      set_status(v.ctl, GB_ERR_INVALID);
      continue;
    }
    const uint4 x = __ldcs(reinterpret_cast<const uint4*>(kv ? vv : k) + src0 + (size_t)s_tok[t] * rows + c);
    reinterpret_cast<uint4*>(v.kv + kv_elem_offset(v, layer, page, kv, c >> 4, pos % v.P) * v.esize)[c & 15] = x;
  }
}

// One CTA, thread = slot.  The pages past a slot's new length lose a reference.  A slot that is cut inside a page
// that others hold (theirs goes on, or was cut elsewhere) gets a copy, so that a shared page keeps one
// meaning for all its holders; slots decide in order against the current references, so when all of a page's
// holders are cut inside it the last one keeps it.  All or nothing: when there is not a free page for every
// slot cut inside a page that has several holders before the call, nothing changes.  Latency: 8 us.
__global__ void __launch_bounds__(1024) k_truncate(PoolView v, const int* lengths) {
  pdl_wait();
  pdl_launch_dependents();
  constexpr int kShort = 8;  // pages a thread drops by itself; longer runs go to a warp each
  __shared__ int tmp[33];
  __shared__ int s_tail[kMaxBeams], s_pages[kMaxBeams], s_long[kMaxBeams];
  __shared__ int s_nlong;
  const int tid = threadIdx.x, b = tid;
  const bool act = b < v.max_beams && v.active[b] != 0;
  const int L = act ? v.seq_len[b] : 0, want = act ? lengths[b] : -1;
  if (want > L) set_status(v.ctl, GB_ERR_INVALID);
  const bool cut = want >= 0 && want < L;
  const int* table = v.tables + (size_t)b * v.max_pages;
  const int tail = cut && want % v.P ? table[want / v.P] : -1;
  const bool shared = tail >= 0 && v.refcnt[tail] > 1;
  if (tid == 0) s_nlong = 0;
  s_tail[b] = tail;
  int need;
  block_exclusive_scan(shared ? 1 : 0, tmp, &need);
  if (need > v.ctl[kCtlFree]) {
    if (tid == 0) {
      set_status(v.ctl, GB_ERR_OOM);
      v.ctl[kCtlCowJobs] = 0;
      v.ctl[kCtlSegStale] = 0;
    }
    return;
  }
  __syncthreads();
  const int j0 = cut ? (want + v.P - 1) / v.P : 0, j1 = cut ? (L + v.P - 1) / v.P : 0;
  if (j1 - j0 <= kShort) {
    for (int j = j0; j < j1; ++j) unref_page(v, table[j]);
  } else {
    s_long[atomicAdd(&s_nlong, 1)] = b;
  }
  // Only pages of shared segments matter to them: those past a slot's cover are its own.
  const bool stale = __syncthreads_or(cut && v.grouped && want / v.P < v.seg_cover[b]);
  if (cut) {
    v.seq_len[b] = want;
    v.gen[b] = max(0, v.gen[b] - (L - want));
  }
  __syncthreads();
  s_pages[b] = j1;  // the run's end, for the warps that take the long ones
  __syncthreads();
  for (int i = tid >> 5; i < s_nlong; i += 32) {
    const int s = s_long[i], n = v.seq_len[s];
    for (int j = (n + v.P - 1) / v.P + (tid & 31); j < s_pages[s]; j += 32)
      unref_page(v, v.tables[(size_t)s * v.max_pages + j]);
  }
  __threadfence_block();
  __syncthreads();
  // Who copies: references as they are now, less the lower slots that copied before.
  bool cow = false;
  if (shared) {
    const int R = *reinterpret_cast<volatile int*>(&v.refcnt[tail]);
    int before = 0;
    if (R > 1)
      for (int s = 0; s < b; ++s) before += s_tail[s] == tail;
    cow = R - before > 1;
  }
  int total;
  const int rank = block_exclusive_scan(cow ? 1 : 0, tmp, &total);
  int found = 0, w0 = max(*reinterpret_cast<volatile int*>(&v.ctl[kCtlCursor]), 0);
  __syncthreads();
  while (found < total && w0 < v.words) {
    const int word = w0 + tid;
    unsigned bits = word < v.words ? *reinterpret_cast<volatile unsigned*>(&v.free_bits[word]) : 0u;
    if (word == v.words - 1 && (v.num_pages & 31)) bits &= (1u << (v.num_pages & 31)) - 1u;
    int here;
    int r = found + block_exclusive_scan(__popc(bits), tmp, &here);
    const unsigned before = bits;
    while (bits && r < total) {
      s_pages[r] = word * 32 + __ffs(bits) - 1;
      bits &= bits - 1u;
      if (++r == total) v.ctl[kCtlCursor] = word;
    }
    if (bits != before) v.free_bits[word] = (*reinterpret_cast<volatile unsigned*>(&v.free_bits[word]) & ~before) | bits;
    found += here;
    w0 += 1024;
  }
  __syncthreads();
  if (cow) {
    const int p = s_pages[rank];
    atomicSub(&v.refcnt[tail], 1);
    v.refcnt[p] = 1;
    v.tables[(size_t)b * v.max_pages + want / v.P] = p;
    v.cow[3 * rank] = tail;
    v.cow[3 * rank + 1] = p;
    v.cow[3 * rank + 2] = want % v.P;
  }
  if (tid == 0) {
    v.ctl[kCtlCowJobs] = total;
    v.ctl[kCtlSegStale] = stale;
    v.ctl[kCtlChanges] += 1;
    if (total > 0) atomicSub(&v.ctl[kCtlFree], total);
  }
}

// The rows of the pages that k_truncate replaced: a CTA per (layer, job).
__global__ void __launch_bounds__(256) k_cow_rows(PoolView v) {
  pdl_wait();
  pdl_launch_dependents();
  const int jobs = v.ctl[kCtlCowJobs], layer = blockIdx.y;
  for (int j = blockIdx.x; j < jobs; j += gridDim.x) {
    const int old = v.cow[3 * j], page = v.cow[3 * j + 1], have = v.cow[3 * j + 2];
    for (int i = threadIdx.x; i < 2 * v.Hkv * have * 16; i += 256) {
      const int c = i & 15, row = (i >> 4) % have, kvh = (i >> 4) / have;
      reinterpret_cast<uint4*>(v.kv + kv_elem_offset(v, layer, page, kvh / v.Hkv, kvh % v.Hkv, row) * v.esize)[c] =
          reinterpret_cast<const uint4*>(v.kv + kv_elem_offset(v, layer, old, kvh / v.Hkv, kvh % v.Hkv, row) * v.esize)[c];
    }
  }
}

bool on_device(const gb_pool* pool) {
  int d = -1;
  return cudaGetDevice(&d) == cudaSuccess && d == pool->device;
}

gb_status check_draft(gb_pool* pool, const gb_draft* d, const char* what) {
  if (!d || d->n_draft < 1 || d->n_draft > kMaxDraft || !d->parent_dev || !d->workspace_dev ||
      ((uintptr_t)d->workspace_dev & 255))
    return fail(pool, GB_ERR_INVALID, what);
  if (d->workspace_bytes < draft_layout(pool->cfg, pool->num_sms, d->n_draft).total)
    return fail(pool, GB_ERR_INVALID, "draft: the workspace is too small");
  if (!on_device(pool)) return fail(pool, GB_ERR_STATE, "draft: the pool is on another device than the current one");
  if (!pool->seeded) return fail(pool, GB_ERR_STATE, "pool not seeded");
  if (pool->next_layer != 0) return fail(pool, GB_ERR_STATE, "draft: inside an open step");
  return GB_OK;
}

bool meets(const void* a, size_t an, const void* b, size_t bn) {
  const char *x = static_cast<const char*>(a), *y = static_cast<const char*>(b);
  return x < y + bn && y < x + an;
}

// The round that a layer above 0 belongs to, or nullptr.
const gb_pool::DraftPlan* find_plan(const gb_pool* pool, const void* ws, int tokens, unsigned long long capture) {
  if (pool->draft_epoch != pool->epoch) return nullptr;
  for (const gb_pool::DraftPlan& p : pool->draft_plans)
    if (p.token && p.ws == ws && p.tokens == tokens && p.capture == capture) return &p;
  return nullptr;
}

// Takes the place of the plans whose memory it shares; where all entries are taken the oldest gives way.
void keep_plan(gb_pool* pool, const gb_pool::DraftPlan& plan) {
  gb_pool::DraftPlan* oldest = pool->draft_plans;  // (names grow; an entry without a plan has 0)
  for (gb_pool::DraftPlan& p : pool->draft_plans) {
    if (pool->draft_epoch != pool->epoch || meets(p.ws, p.bytes, plan.ws, plan.bytes)) p = {};
    if (p.token < oldest->token) oldest = &p;
  }
  *oldest = plan;
  pool->draft_epoch = pool->epoch;
}

}  // namespace
}  // namespace gb

using namespace gb;

extern "C" gb_status gb_draft_workspace_bytes(gb_pool* pool, int n_draft, size_t* bytes) {
  if (!pool || !bytes) return GB_ERR_INVALID;
  if (n_draft < 1 || n_draft > kMaxDraft) return fail(pool, GB_ERR_INVALID, "draft: 1 to 64 tokens");
  *bytes = draft_layout(pool->cfg, pool->num_sms, n_draft).total;
  return GB_OK;
}

extern "C" gb_status gb_draft_attention(gb_pool* pool, int layer, const gb_draft* d, const void* q_dev,
                                        const void* k_dev, const void* v_dev, float scale, void* out_dev,
                                        gb_stream_t stream) {
  if (!pool) return GB_ERR_INVALID;
  gb_status st = check_draft(pool, d, "draft: bad arguments");
  if (st != GB_OK) return st;
  if (layer < 0 || layer >= pool->cfg.num_layers || !q_dev || !k_dev || !v_dev || !out_dev || !(scale > 0.f) ||
      scale > 3e38f || (((uintptr_t)q_dev | (uintptr_t)k_dev | (uintptr_t)v_dev) & 15) || ((uintptr_t)out_dev & 31))
    return fail(pool, GB_ERR_INVALID, "draft: bad arguments");
  const PoolView& v = pool->view;
  const int T = d->n_draft;
  const size_t qb = (size_t)v.max_beams * T * v.Hq * v.D * v.esize, kb = qb / v.G;
  if (meets(out_dev, qb, q_dev, qb) || meets(out_dev, qb, k_dev, kb) || meets(out_dev, qb, v_dev, kb))
    return fail(pool, GB_ERR_INVALID, "draft: the output overlaps an input");
  const bool bf16 = v.dtype == GB_BF16;
  if (bf16 && !flash::launches_with(reinterpret_cast<const void*>(k_draft)))
    return fail(pool, GB_ERR_UNSUPPORTED, "draft: the kernel's registers");
  if (bf16 && !pool->have_tmap) return fail(pool, GB_ERR_UNSUPPORTED, "draft: no tensor map over the pool");
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  // A captured plan is made when its graph runs: it serves the calls of the same capture only.
  cudaStreamCaptureStatus capturing = cudaStreamCaptureStatusNone;
  unsigned long long capture = 0;
  if (const cudaError_t e = cudaStreamGetCaptureInfo(s, &capturing, &capture); e != cudaSuccess) {
    cudaGetLastError();
    return fail(pool, GB_ERR_CUDA, cudaGetErrorString(e));
  }
  if (capturing != cudaStreamCaptureStatusActive) capture = 0;
  const gb_pool::DraftPlan* planned = layer > 0 ? find_plan(pool, d->workspace_dev, T, capture) : nullptr;
  if (layer > 0 && !planned)
    return fail(pool, GB_ERR_STATE, "draft: layer 0 plans the round, on the pool as it is, in this workspace and graph");
  static std::atomic<unsigned long long> plans{0};
  const unsigned long long token = planned ? planned->token : ++plans;
  const DraftLayout layout = draft_layout(pool->cfg, pool->num_sms, T);
  const DraftView w = draft_view(pool, layout, T, d->workspace_dev, token);
  const float qscale = scale * 1.4426950408889634f;
  DraftJob job;
  if (bf16) {
    job.v = v;
    job.w = w;
    job.layer = layer;
    job.oob = pool->tmap_oob;
    job.page_shift = v.P == 16 ? 4 : v.P == 32 ? 5 : 6;
    job.group0 = (int)((long long)layer * v.num_pages * 2 * v.Hkv * v.P / 8);
    job.qscale = qscale;
    job.q = static_cast<const __nv_bfloat16*>(q_dev);
    job.k = static_cast<const __nv_bfloat16*>(k_dev);
    job.vv = static_cast<const __nv_bfloat16*>(v_dev);
    job.o = static_cast<__nv_bfloat16*>(out_dev);
    job.tp = *reinterpret_cast<const CUtensorMap*>(pool->tmap);
    const cuuint64_t dims[5] = {64, (cuuint64_t)T, 2, (cuuint64_t)v.Hkv, (cuuint64_t)v.max_beams};
    const cuuint64_t strides[4] = {(cuuint64_t)v.Hkv * 256, 128, 256, (cuuint64_t)T * v.Hkv * 256};
    const cuuint32_t box[5] = {64, 8, 2, 1, 1};
    if (!encode_tensor_map(&job.tk, k_dev, 5, dims, strides, box) ||
        !encode_tensor_map(&job.tv, v_dev, 5, dims, strides, box))
      return fail(pool, GB_ERR_CUDA, "draft: tensor map");
  }
  if (layer == 0) {
    const int tokens = (bf16 ? 2 * flash::kRows : kTileRows) / v.G;  // (G is a power of two)
    int shift = 0;
    while (1 << shift < tokens) ++shift;
    const long long tiles = (long long)v.max_pages * v.P / flash::kTok + 2;
    const long long dearest = 2 * v.max_beams * ((T + tokens - 1ll) / tokens) * (kTileCost * tiles + kUnitCost + kRecCost);
    int coarse = 0;
    while (dearest >> coarse >= 1 << 28) ++coarse;
    launch_pdl(k_draft_plan, 1, kListThreads, 0, s, v, w, d->parent_dev, d->count_dev, shift,
               bf16 ? shift - 1 : shift, bf16 ? 2 : 1, coarse, bf16 && v.grouped);
    pool->launches += 1;
    if (v.max_beams > kOneLaunch) {
      launch_pdl(k_draft_rows, (v.max_beams + 7) / 8, 256, 0, s, v, w, d->parent_dev, d->count_dev);
      pool->launches += 1;
    }
    if ((st = check_launch(pool, "draft_plan")) != GB_OK) return st;
    keep_plan(pool, {d->workspace_dev, layout.total, T, capture, token});
  }
  cudaError_t e;
  const bool sparse = (long long)T * v.max_beams < 2 * pool->num_sms;
  const dim3 merge(T, v.max_beams, sparse ? (v.Hq + 7) / 8 : 1);
  if (bf16) {
    e = set_max_dynamic_smem(reinterpret_cast<const void*>(k_draft), flash::kSmem);
    if (e == cudaSuccess) e = launch_pdl(k_draft, pool->num_sms, flash::kThreads, flash::kSmem, s, job);
    if (e == cudaSuccess)
      e = launch_pdl(sparse ? k_draft_merge<__nv_bfloat16, 128, 8> : k_draft_merge<__nv_bfloat16, 128, 4>, merge, 256, 0, s, v,
                     w, job.o);
  } else {
    e = set_max_dynamic_smem(reinterpret_cast<const void*>(k_draft_f32), (int)sizeof(TileSmem));
    if (e == cudaSuccess)
      e = launch_pdl(k_draft_f32, pool->num_sms, kTileThreads, sizeof(TileSmem), s, v, w, layer,
                     static_cast<const float*>(q_dev), static_cast<const float*>(k_dev), static_cast<const float*>(v_dev),
                     static_cast<float*>(out_dev), qscale);
    if (e == cudaSuccess)
      e = launch_pdl(sparse ? k_draft_merge<float, 64, 8> : k_draft_merge<float, 64, 4>, merge, 256, 0, s, v, w,
                     static_cast<float*>(out_dev));
  }
  pool->launches += 2;
  if (e != cudaSuccess) return fail(pool, GB_ERR_CUDA, cudaGetErrorString(e));
  return check_launch(pool, "draft");
}

extern "C" gb_status gb_accept_draft(gb_pool* pool, const gb_draft* d, const void* k_dev, const void* v_dev,
                                     const int32_t* accepted_dev, int32_t* count_out_dev, int32_t* path_out_dev,
                                     gb_stream_t stream) {
  if (!pool) return GB_ERR_INVALID;
  gb_status st = check_draft(pool, d, "accept: bad arguments");
  if (st != GB_OK) return st;
  if (!k_dev || !v_dev || !accepted_dev || (((uintptr_t)k_dev | (uintptr_t)v_dev) & 15))
    return fail(pool, GB_ERR_INVALID, "accept: bad arguments");
  const DraftView w =
      draft_view(pool, draft_layout(pool->cfg, pool->num_sms, d->n_draft), d->n_draft, d->workspace_dev, 0);
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  launch_pdl(k_accept_plan, 1, 1024, 0, s, pool->view, w, d->parent_dev, d->count_dev, accepted_dev, count_out_dev,
             path_out_dev);
  pool->launches += 1;
  if ((st = check_launch(pool, "accept_plan")) != GB_OK) return st;
  ++pool->epoch;
  launch_pdl(k_accept_copy, dim3(pool->cfg.max_beams, pool->cfg.num_layers), 256, 0, s, pool->view, w,
             static_cast<const char*>(k_dev), static_cast<const char*>(v_dev));
  pool->launches += 1;
  return check_launch(pool, "accept_copy");
}

extern "C" gb_status gb_truncate(gb_pool* pool, const int32_t* lengths_dev, gb_stream_t stream) {
  if (!pool) return GB_ERR_INVALID;
  if (!lengths_dev) return fail(pool, GB_ERR_INVALID, "truncate: null pointer");
  if (!on_device(pool)) return fail(pool, GB_ERR_STATE, "truncate: the pool is on another device than the current one");
  if (!pool->seeded) return fail(pool, GB_ERR_STATE, "pool not seeded");
  if (pool->next_layer != 0) return fail(pool, GB_ERR_STATE, "truncate inside an open step");
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  ++pool->epoch;
  launch_pdl(k_truncate, 1, 1024, 0, s, pool->view, lengths_dev);
  launch_pdl(k_cow_rows, dim3(std::min(pool->cfg.max_beams, 64), pool->cfg.num_layers), 256, 0, s, pool->view);
  pool->launches += 2;
  const gb_status st = check_launch(pool, "truncate");
  if (st != GB_OK) return st;
  if (rebuild_segments(pool, s, pool->view.ctl + kCtlSegStale) != cudaSuccess) return check_launch(pool, "segments");
  return GB_OK;
}
