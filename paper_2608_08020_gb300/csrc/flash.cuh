// Attention of up to 256 query rows over a run of keys on the tcgen05 tensor cores: bf16 inputs, 128
// dims, fp32 sums.  The pipeline shared by the prompt and the draft-tree kernels; a Job says which
// units of work there are, where their rows lie, which keys a row sees and where its result goes.
//
//   S = Q K^T (128 x 128, fp32 in tensor memory),  P = 2^(scale' S - m) (bf16),  O += P V
// with the running maximum m and sum l of each row's softmax, one pass over the keys.
//
// A unit has one head's query rows and nt tiles of 128 keys.  Two groups of four softmax warps each hold
// a Q tile of 128 rows, an accumulator O and an S tile in tensor memory (512 columns in all), so that two chains are in flight:
// while one group takes the exponentials of its S tile the tensor core works for the other.  A tile of each group is 2048
// cycles of products (128^3 x 2 each at 4096 multiply-adds a cycle); a long prompt takes some 3300 for it, since the chain from an
// S tile to the group's next one (scores read, maximum, 128 x 128 ex2 and their sums, P written, P.V, S) is longer than the
// other group's products, and what of it the two groups do not cover the tensor core waits.  What a group works on:
//   dual          129 to 256 rows: each group half of the rows, every K/V tile serves both
//   first, second up to 128 rows: two units of the CTA's list, a group each, their tiles coming by turns
//   joint         up to 128 rows and no second unit: the same rows in both groups, group g takes tiles g, g + 2, ...,
//                 and their sums are joined at the end
//   alone         the same with a single tile, or where the job does not allow joint units: group 0
// A row's sum goes over the keys in the same order in every mode but joint.
//
// P is rounded to bf16 for the tensor core: at most 2^-8 of each p, independent of one another, so a row's error is about that
// of its own rounding to bf16 (1.2 to 1.4 times a result's whose p are fp32).  A second term of 8 bits would be a P.V more for each
// tile, half as many products again.  The decode step's grouped role rounds the same way.  The sum l is of the unrounded values.
//
// Warp roles (512 threads):
//   warps 0-7    softmax: thread r of group g owns row r of its tile (tensor-memory lane r); also loads
//                the row's query; at the end they answer rows anew that met unseen values (one_row)
//   warp 8       takes the CTA's units from the sorted list, publishes them in a ring of eight and streams K
//   warp 11      streams V; both go through one ring of five 32 KiB stages (K0 V0 K1 V1 ..., of a pair K K V V)
//   warps 9-10   issue the products of a group each: S(i), then P.V(i) before S(i + 1), whose tile
//                P overwrites; a thread's products run in issue order
//   warps 12-15  write the results: while they read O the softmax groups are in the next unit
// CTA b takes entries b, 2 n - 1 - b, 2 n + b, ... of the list (n CTAs, longest first), so the shares come out even
// without a counter that every unit has to wait for.
// P overwrites the first half of its S tile.  O is rescaled by its own group, and only when a maximum
// grows by more than 8 (p <= 2^8 meanwhile): when S(i) is complete so is P.V(i - 1), issued before it.
//
// Every wait is bounded; when one runs out the CTA records the timeout, every role stops issuing and, once all have, waits
// (bounded) for its own copies and products, then the tensor memory is freed and the CTA leaves.
#pragma once
#include <cuda.h>
#include <mutex>
#include <set>
#include <type_traits>
#include <utility>

#include "internal.cuh"
#include "ptx.cuh"
#include "tc.cuh"

namespace gb {
namespace flash {

constexpr int kRows = 128, kTok = 128, kD = 128;
constexpr int kThreads = 512;          // four warpgroups: the two softmax groups, loads and products, results
constexpr int kLaunchRegs = 128;       // registers a thread at launch (65536 / 512); the softmax groups then hold a
constexpr int kSoftmaxRegs = 192, kOtherRegs = 64;  // tile's row of 128 scores, the others give theirs
static_assert(256 * (kSoftmaxRegs + kOtherRegs) <= kThreads * kLaunchRegs, "the shares come from the launch's total");
constexpr int kKWarp = 8, kMmaWarp = 9, kVWarp = 11, kOutWarp = 12;
constexpr int kStages = 5;
constexpr int kTile = 32768;           // Q, K or V tile: 128 x 128 bf16
constexpr int kRing = 2 * kTile;       // after the two Q tiles
constexpr int kBar = kRing + kStages * kTile;
constexpr int kXch = kBar + 1024;      // float2 [2 groups][128 rows]: (m, l) of a unit's groups
constexpr int kSmem = kXch + 2048;
static_assert(kSmem <= 232448, "shared memory per block");
constexpr uint32_t kTmemS = 0, kTmemO = 256;  // column of group 0; group 1 is 128 further

constexpr int kSlots = 8, kUnitWords = 12;  // units known ahead
enum Mode : int { kJoint, kDual, kFirst, kSecond, kAlone };
// Three "full" and three "empty" barriers a stage, used in turn (ring position mod 15), since the warps do not keep step: a wait
// on a barrier whose phase before last has not ended would pass at once.  For a group that waits for position p that phase is
// of p - 15.  It has ended if the load of p - 10 into its stage has been issued, and that follows from what the group has seen:
// the K and V of its tiles before, or that p's unit has begun (kBarBegin), so that every K before it is out.  Each warp loads in
// order, and a load at q says that q - 5 was consumed, hence landed, hence that all loads of its kind before it are out.  The
// blocks K V and K K V V, in any order, leave no p without such a chain (tests/test_ring_order.py goes through sequences of units);
// a loading warp's wait, for the consumption of p - 5, has p - 20 behind it in the same way.
constexpr int kFulls = 3 * kStages;
constexpr int kBarFull = 0;                       // [kFulls]
constexpr int kBarEmpty = kBarFull + 8 * kFulls;  // [kFulls]
constexpr int kBarQ = kBarEmpty + 8 * kFulls;     // [2] the group's query rows are in
constexpr int kBarS = kBarQ + 16;                 // [2] S of the group's next tile is complete
constexpr int kBarP = kBarS + 16;                 // [2 groups][2 halves] P of 64 of its keys is written (and O rescaled)
constexpr int kBarO = kBarP + 32;                 // [2] the unit's last P.V of the group is complete
constexpr int kBarOFree = kBarO + 16;             // [2] the group's O has been read
constexpr int kBarML = kBarOFree + 16;            // [2] the group's (m, l) are in
constexpr int kBarDrained = kBarML + 16;          // [2] all of the group's products are complete (given up)
constexpr int kBarPatch = kBarDrained + 16;       // a V tile that is mended before it is handed on
constexpr int kBarSched = kBarPatch + 8;          // [kSlots]
constexpr int kBarBegin = kBarSched + 8 * kSlots;  // [kSlots] K of the unit is on its way
constexpr int kBarSchedFree = kBarBegin + 8 * kSlots;
constexpr int kUnits = (kBarSchedFree + 8 * kSlots + 15) / 16 * 16;  // int [kSlots][kUnitWords]
// What the K and the V warp may have in flight at their end: the position loaded last, bit i of `seen` for the load i positions
// before it, and of a V tile that waits to be mended its full barrier (else 0) and the patch barrier's phase.
struct Flight {
  uint32_t last, seen, patched, patch_parity;
};
constexpr int kFlights = kUnits + 4 * kSlots * kUnitWords;  // Flight [2]
constexpr int kWordTmem = kFlights + 2 * (int)sizeof(Flight);
constexpr int kWordAbort = kWordTmem + 4;
constexpr int kWordAgain = kWordAbort + 4;  // some row was not finite
static_assert(kUnits % 16 == 0 && kWordAgain + 4 <= 1024, "control area");
constexpr int kSchedReaders = 15;  // eight softmax warps, two that issue products, one that loads V, four that write

// What every role knows of a unit; w is the job's own.
struct Unit {
  int nt;    // tiles of 128 keys; -1: no more units
  int mode;  // (the job says kDual or kJoint)
  int mate;  // tiles of the other unit of a first or second one
  int head;  // KV head
  int w[kUnitWords - 4];
};
static_assert(sizeof(Unit) == 4 * kUnitWords, "unit words");

__device__ __forceinline__ bool takes_part(int mode, int g) {
  return mode <= kDual || (g == 0) != (mode == kSecond);
}
// Group g's tiles of a unit.
__device__ __forceinline__ int group_tiles(int nt, int mode, int g) { return mode == kJoint ? (nt + 1 - g) / 2 : nt; }
__device__ __forceinline__ int group_tile(int mode, int g, int i) { return mode == kJoint ? 2 * i + g : i; }
// Ring positions of the K of a group's tiles i = 0, 1, ..., counted from where the unit (or the pair) begins; V follows its K.
__device__ __forceinline__ int tile_position(int mode, int mate, int g, int i) {
  if (mode == kFirst) return 2 * (i + min(i, mate));
  if (mode == kSecond) return 2 * (i + min(i + 1, mate));
  return 2 * group_tile(mode, g, i);
}
// The same for a job with long pairs (kLongPair tiles or more by turns): while both units of one have tiles they come as K K V V, so
// that a group's next K is in the ring a step before it is due.  Those of short ones come as K V K V, which puts the groups half
// a step apart from the start.
struct Places {
  int both, first, v_after;  // tiles that come by turns, the first's position, and how far behind its K a V lies meanwhile
  __device__ __forceinline__ int k(int i) const { return i < both ? 4 * i + first : 2 * (i + both); }
  __device__ __forceinline__ int v(int i) const { return k(i) + (i < both ? v_after : 1); }
};
// Of the first or second unit of a pair with that many tiles by turns (0: of a unit by itself).
template <class Job>
__device__ __forceinline__ Places places(int both, bool second) {
  const bool far = both >= Job::kLongPair;
  return {both, second ? (far ? 1 : 2) : 0, far ? 2 : 1};
}
// Ring positions of a unit, a pair's counted with its second.
__device__ __forceinline__ int positions(int nt, int mode, int mate) {
  return mode == kFirst ? 0 : mode == kSecond ? 2 * (nt + mate) : 2 * nt;
}

// The columns are handed out only after the wait: the registers pass through it.
__device__ __forceinline__ void ld32_issue(uint32_t taddr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
      "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
        "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
        "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr));
}
__device__ __forceinline__ void ld32_wait(uint32_t* r) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
                 "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]),
                 "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]),
                 "+r"(r[23]), "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]),
                 "+r"(r[30]), "+r"(r[31])
               :
               : "memory");
}

__device__ __forceinline__ void st16(uint32_t taddr, const uint32_t* u) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(
          taddr),
      "r"(u[0]), "r"(u[1]), "r"(u[2]), "r"(u[3]), "r"(u[4]), "r"(u[5]), "r"(u[6]), "r"(u[7]), "r"(u[8]), "r"(u[9]),
      "r"(u[10]), "r"(u[11]), "r"(u[12]), "r"(u[13]), "r"(u[14]), "r"(u[15])
      : "memory");
}
// Two fp32 operations in one instruction.
__device__ __forceinline__ uint64_t pack2(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void unpack2(uint64_t x, float& a, float& b) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(x));
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
template <int N>
__device__ __forceinline__ void regs_inc() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N>
__device__ __forceinline__ void regs_dec() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }
__device__ __forceinline__ void st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Products with the accumulate flag known (tc.cuh's take it as a value).
__device__ __forceinline__ void mma_set(uint32_t d, uint64_t a, uint64_t b, uint32_t id) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, 0, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
               "l"(a), "l"(b), "r"(id));
}
__device__ __forceinline__ void mma_add(uint32_t d, uint64_t a, uint64_t b, uint32_t id) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.eq.b32 p, 0, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
               "l"(a), "l"(b), "r"(id));
}
__device__ __forceinline__ void mma_ts_add(uint32_t d, uint32_t a, uint64_t b, uint32_t id) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.eq.b32 p, 0, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
               "r"(a), "l"(b), "r"(id));
}
// 32 bytes of a row.  A thread writes its own row, so a store of a warp meets 32 lines however wide it is: the wider, the
// fewer.
__device__ __forceinline__ void st32(void* p, const uint32_t* u) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(u[0]), "r"(u[1]), "r"(u[2]),
               "r"(u[3]), "r"(u[4]), "r"(u[5]), "r"(u[6]), "r"(u[7])
               : "memory");
}
// Whether a kernel of this pipeline has the registers at launch that its warps then share out (fewer, and they would wait for ever).
inline bool launches_with(const void* kernel) try {
  static std::mutex mu;
  static std::set<std::pair<const void*, int>> fine;  // (kernel, device)
  int device = 0;
  if (cudaGetDevice(&device) != cudaSuccess) return false;
  std::lock_guard<std::mutex> lock(mu);
  if (fine.count({kernel, device})) return true;
  cudaFuncAttributes a{};
  if (cudaFuncGetAttributes(&a, kernel) != cudaSuccess || a.numRegs * kThreads < 256 * (kSoftmaxRegs + kOtherRegs))
    return false;
  fine.insert({kernel, device});
  return true;
} catch (...) {
  return false;
}
// warp_wait (tc.cuh) with the lanes apart meanwhile, for the warps that write (8192 tokens when it was chosen: 384 us so, 388 with
// the other here too, 391 with this one for the softmax too).
template <class Job>
__device__ __forceinline__ bool lanes_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag) {
  return __all_sync(0xffffffffu, wait_or_abort(bar, parity, abort_flag, Job::kWaitNs));
}
// One lane of the warp, the same each time.
__device__ __forceinline__ bool elect_one() {
  uint32_t p;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
  return p != 0;
}

__device__ __forceinline__ void ld16_issue(uint32_t taddr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr));
}
__device__ __forceinline__ void ld16_wait(uint32_t* r) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
                 "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])
               :
               : "memory");
}
// Columns of a row's result, N = 16 or 32 of one group's O, or 16 of both with their weights.
template <int N>
__device__ __forceinline__ void read_o(uint32_t a, float* o) {
  uint32_t u[N];
#pragma unroll
  for (int c = 0; c < N; c += 16) ld16_issue(a + c, u + c);
#pragma unroll
  for (int c = 0; c < N; c += 16) ld16_wait(u + c);
#pragma unroll
  for (int c = 0; c < N; ++c) o[c] = __uint_as_float(u[c]);
}
__device__ __forceinline__ void read_both(uint32_t a, uint32_t b, float wa, float wb, float* o) {
  uint32_t u[16], v[16];
  ld16_issue(a, u);
  ld16_issue(b, v);
  ld16_wait(u);
  ld16_wait(v);
  // A weight of 0 belongs to a group that saw no key of the row: what it summed is 0 x V.
#pragma unroll
  for (int c = 0; c < 16; ++c)
    o[c] = (wa == 0.f ? 0.f : wa * __uint_as_float(u[c])) + (wb == 0.f ? 0.f : wb * __uint_as_float(v[c]));
}
// The 128 columns in turn, 32 at a time (16 of a joint unit): use(c, N, values).  done() once all have been read.
template <class Use, class Done>
__device__ __forceinline__ void walk_o(uint32_t a, uint32_t b, bool two, float wa, float wb, Use use, Done done) {
  if (two) {
#pragma unroll 1
    for (int c = 0; c < kD; c += 16) {
      float f[16];
      read_both(a + c, b + c, wa, wb, f);
      if (c + 16 == kD) done();
      use(c, std::integral_constant<int, 16>{}, f);
    }
  } else {
#pragma unroll 1
    for (int c = 0; c < kD; c += 32) {
      float f[32];
      read_o<32>(a + c, f);
      if (c + 32 == kD) done();
      use(c, std::integral_constant<int, 32>{}, f);
    }
  }
}

// Rows of a V tile that hold no token but whatever their memory did, up to 127 of them: `first` rows from row a on, then `second`
// from row b on.  One word, 0: none.
__device__ __forceinline__ uint32_t stale_word(int a, int first, int b, int second) {
  return (uint32_t)a | (uint32_t)first << 8 | (uint32_t)b << 16 | (uint32_t)(first + second) << 24;
}

// Keys of a tile a row sees: all of them, the first `limit`, or the first `limit` (up to 64) and those of `bits`.
struct Sees {
  bool all;                 // (the same for the warp)
  bool by_bits;             // (the same for the warp)
  int limit;                // columns below this
  unsigned long long bits;  // column 64 + i for bit i
};

// A product with P takes every key of a tile, with p = 0 for those the row does not see, and 0 x inf is NaN: a row whose result is
// not finite although the maximum and the sum of its softmax are may only have met a value that it does not see.  The warps that
// write make a note, and the softmax warps, once all else is done and nobody waits for them but the CTA's end, look through the
// CTA's rows for those and answer them anew over the keys they see (Job::again).

// One row's softmax over the keys that key(j, kv, row) says are seen (row: k_j or v_j), by a warp: lane l gets columns 4 l on of the
// unnormalised sum.  32 keys at a time, a score to a lane, then eight values' loads at once (256 rows over 32768 keys by a CTA's eight
// warps: 135 ms; by the four that write, with the registers they have, 280 to 700, and their units waited).  False where a score
// seen is not finite.
template <class Key>
__device__ __forceinline__ bool one_row(const __nv_bfloat16* q, int nkeys, Key key, float qscale, float& m, float& l, float* acc) {
  const int lane = threadIdx.x & 31;
  constexpr int kAtOnce = 8;
  m = -INFINITY;
  l = 0.f;
  for (int i = 0; i < 4; ++i) acc[i] = 0.f;
#pragma unroll 1
  for (int j0 = 0; j0 < nkeys; j0 += 32) {
    const __nv_bfloat16* row;
    const bool on = j0 + lane < nkeys && key(j0 + lane, 0, row);
    float s = -INFINITY;
    if (on) {
      float part[4] = {};
#pragma unroll 4
      for (int c = 0; c < kD; c += 8) {
        const uint4 a = *reinterpret_cast<const uint4*>(q + c), b = *reinterpret_cast<const uint4*>(row + c);
        const uint32_t x[4] = {a.x, a.y, a.z, a.w}, y[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          part[i] = fmaf(__uint_as_float(x[i] << 16), __uint_as_float(y[i] << 16), part[i]);
          part[i] = fmaf(__uint_as_float(x[i] & 0xffff0000u), __uint_as_float(y[i] & 0xffff0000u), part[i]);
        }
      }
      s = ((part[0] + part[1]) + (part[2] + part[3])) * qscale;
    }
    float mx = s;
#pragma unroll
    for (int w = 16; w > 0; w >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, w));
    if (mx > m) {
      const float f = exp2f(m - mx);
      l *= f;
      for (int i = 0; i < 4; ++i) acc[i] *= f;
      m = mx;
    }
    const float p = on ? exp2f(s - (m == -INFINITY ? 0.f : m)) : 0.f;  // (scores of -inf alone so far: every p is 0)
    l += p;
    const unsigned there = __ballot_sync(0xffffffffu, on);
#pragma unroll 1
    for (int e0 = 0; e0 < 32; e0 += kAtOnce) {
      uint2 x[kAtOnce];
#pragma unroll
      for (int e = 0; e < kAtOnce; ++e)
        if ((there >> (e0 + e)) & 1) {
          key(j0 + e0 + e, 1, row);
          x[e] = reinterpret_cast<const uint2*>(row)[lane];
        }
#pragma unroll
      for (int e = 0; e < kAtOnce; ++e) {
        const float f = __shfl_sync(0xffffffffu, p, e0 + e);
        if ((there >> (e0 + e)) & 1) {
          acc[0] = fmaf(f, __uint_as_float(x[e].x << 16), acc[0]);
          acc[1] = fmaf(f, __uint_as_float(x[e].x & 0xffff0000u), acc[1]);
          acc[2] = fmaf(f, __uint_as_float(x[e].y << 16), acc[2]);
          acc[3] = fmaf(f, __uint_as_float(x[e].y & 0xffff0000u), acc[3]);
        }
      }
    }
  }
#pragma unroll
  for (int w = 16; w > 0; w >>= 1) l += __shfl_xor_sync(0xffffffffu, l, w);
  return isfinite(m) && isfinite(l);
}
// Whether two bf16 values, or a row of V (this lane's answer), are not all finite.
__device__ __forceinline__ bool not_finite(uint32_t x) { return (x & 0x7f80u) == 0x7f80u || (x & 0x7f800000u) == 0x7f800000u; }
__device__ __forceinline__ bool not_finite(const __nv_bfloat16* v) {
  bool bad = false;
#pragma unroll 4
  for (int c = 0; c < kD; c += 8) {
    const uint4 a = *reinterpret_cast<const uint4*>(v + c);
    bad = bad || not_finite(a.x) || not_finite(a.y) || not_finite(a.z) || not_finite(a.w);
  }
  return bad;
}

// Entry of the list that is the CTA's u-th: b, 2 n - 1 - b, 2 n + b, ...
__device__ __forceinline__ int unit_id(int u) {
  return u * (int)gridDim.x + ((u & 1) ? (int)gridDim.x - 1 - (int)blockIdx.x : (int)blockIdx.x);
}

template <class Job>
__device__ __forceinline__ void body(const Job& job, unsigned char* sm) {
  // (the warp by a shuffle: what follows from it is then known to be the same in every lane)
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  const uint32_t sbase = smem_addr(sm), ctl = sbase + kBar;
  volatile int* abort_flag = reinterpret_cast<volatile int*>(sm + kBar + kWordAbort);
  volatile int* again = reinterpret_cast<volatile int*>(sm + kBar + kWordAgain);
  Unit* units = reinterpret_cast<Unit*>(sm + kBar + kUnits);
  Flight* flight = reinterpret_cast<Flight*>(sm + kBar + kFlights);
  if (sbase & 1023) {  // the swizzled layouts need a 1024-byte aligned base
    pdl_wait();
    if (tid == 0) job.error(GB_ERR_UNSUPPORTED);
    return;
  }
  if (warp == 0) {  // a barrier to a lane
    if (lane < kFulls) {
      mbar_init(ctl + kBarFull + 8 * lane, 1);
      mbar_init(ctl + kBarEmpty + 8 * lane, 2);
    } else if (lane < kFulls + 2) {
      const int i = lane - kFulls;
      mbar_init(ctl + kBarQ + 8 * i, Job::kQArrivals);
      mbar_init(ctl + kBarS + 8 * i, 1);
      mbar_init(ctl + kBarP + 16 * i, 4);
      mbar_init(ctl + kBarP + 16 * i + 8, 4);
      mbar_init(ctl + kBarO + 8 * i, 1);
      mbar_init(ctl + kBarOFree + 8 * i, 4);
      mbar_init(ctl + kBarML + 8 * i, 4);
      mbar_init(ctl + kBarDrained + 8 * i, 1);
    } else if (lane < kFulls + 2 + kSlots) {
      const int i = lane - kFulls - 2;
      mbar_init(ctl + kBarSched + 8 * i, 1);
      mbar_init(ctl + kBarBegin + 8 * i, 1);
      mbar_init(ctl + kBarSchedFree + 8 * i, kSchedReaders);
    } else if (lane == 31) {
      mbar_init(ctl + kBarPatch, 1);
      *abort_flag = 0;
      *reinterpret_cast<volatile int*>(sm + kBar + kWordAgain) = 0;
    }
    static_assert(kFulls + 2 + kSlots <= 31, "a lane each");
    fence_mbar_init();
  }
  if (warp == kMmaWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(ctl + kWordTmem), "r"(512));
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(sm + kBar + kWordTmem);
  pdl_wait();
  pdl_launch_dependents();

  // The warpgroups share out the launch's registers; the others give theirs at once, so the groups' waits for them end.
  if (warp >= kKWarp) {
    regs_dec<kOtherRegs>();
    if (warp == kKWarp) {
      // ---------------------------------------------------------------- units and K tiles
      const typename Job::Units all(job);
      const int total = job.total(all), cap = job.capacity();
      uint32_t from = 0;            // ring position of the unit's (or pair's) first tile; without long pairs, of the next
      uint32_t last = 0, seen = 0;  // position loaded last; bit i: so was the one i before it
      bool ok = true;
      auto find = [&](int u, Unit& x) {
        x.nt = -1;
        x.mate = 0;
        const int id = unit_id(u);
        if (id < cap) job.unit(all, id, x);  // (before the count of units is in: the list is there to its capacity)
        if (id >= total) x.nt = -1;
      };
      auto publish = [&](int u, const Unit& x) {
        const int slot = u & (kSlots - 1);
        if (u >= kSlots) ok = warp_wait<Job::kWaitNs>(ctl + kBarSchedFree + 8 * slot, (u / kSlots - 1) & 1, abort_flag);
        if (ok && lane == 0) {
          units[slot] = x;
          mbar_arrive(ctl + kBarSched + 8 * slot);
        }
        __syncwarp();
      };
      auto begin = [&](int u) {
        if (lane == 0) mbar_arrive(ctl + kBarBegin + 8 * (u & (kSlots - 1)));
      };
      auto load = [&](const Unit& z, const Places& at, int j, int page) {
        const uint32_t n = Job::kLongPair > 0 ? from + at.k(j) : from, st = n % kStages;
        if (n >= (uint32_t)kStages)
          ok = warp_wait<Job::kWaitNs>(ctl + kBarEmpty + 8 * ((n - kStages) % kFulls), ((n - kStages) / kFulls) & 1, abort_flag);
        if (!ok) return;
        const uint32_t bar = ctl + kBarFull + 8 * (n % kFulls);
        if (lane == 0) mbar_arrive_expect_tx(bar, kTile);
        __syncwarp();
        job.load_tile(z, j, 0, page, sbase + kRing + st * kTile, bar, lane);
        if (Job::kLongPair > 0) {
          seen = seen << (n - last) | 1;
          last = n;
        } else {
          from += 2;
        }
      };
      // Modes of a unit and the one after it: two of up to 128 rows make a pair.
      auto match = [&](Unit& p, Unit& q) {
        if (p.nt < 0 || p.mode == kDual) return false;
        if (q.nt < 0 || q.mode == kDual) {
          if (p.nt == 1 || !job.joins(all)) p.mode = kAlone;
          return false;
        }
        p.mode = kFirst;
        p.mate = q.nt;
        q.mode = kSecond;
        q.mate = p.nt;
        return true;
      };
      // x, and y where they are a pair, are known to all and next to be loaded; what follows is looked up meanwhile.
      Unit x, y, a, c;
      find(0, x);
      find(1, y);
      bool pair = match(x, y);
      publish(0, x);
      if (pair && ok) publish(1, y);
      int page_x = x.nt >= 0 ? job.page(x, 0, lane) : 0, page_y = pair ? job.page(y, 0, lane) : 0;  // the lane's pages
      for (int u = 0; ok && x.nt >= 0;) {
        const int step = pair ? 2 : 1, tiles = pair ? max(x.nt, y.nt) : x.nt, both = pair ? min(x.nt, y.nt) : 0;
        const Places at_x = places<Job>(both, false), at_y = places<Job>(both, true);
        bool next_pair = false;
        begin(u);
        if (pair) begin(u + 1);
        for (int j = 0; j < tiles && ok; ++j) {
#pragma unroll 1
          for (int e = 0; e < (pair ? 2 : 1) && ok; ++e) {  // (one copy of a load's code)
            const Unit z = e ? y : x;
            if (j >= z.nt) continue;
            load(z, e ? at_y : at_x, j, e ? page_y : page_x);
            const int next = j + 1 < z.nt ? job.page(z, j + 1, lane) : 0;
            if (e) page_y = next;
            else page_x = next;
          }
          if (j == 0 && ok) {
            if (pair) find(u + 2, a);
            else a = y;
            find(u + step + 1, c);
            next_pair = match(a, c);
            publish(u + step, a);
            if (next_pair && ok) publish(u + step + 1, c);
          }
        }
        if (Job::kLongPair > 0) from += 2 * (x.nt + (pair ? y.nt : 0));
        u += step;
        pair = next_pair;
        x = a;
        y = c;
        page_x = ok && x.nt >= 0 ? job.page(x, 0, lane) : 0;
        page_y = ok && pair ? job.page(y, 0, lane) : 0;
      }
      if (Job::kLongPair == 0) {
        last = from - 2;
        seen = 0x155u & ((1u << min(from, 31u)) - 1);
      }
      if (lane == 0) flight[0] = {last, seen, 0, 0};
    } else if (warp == kVWarp) {
      // ---------------------------------------------------------------- V tiles
      uint32_t from = 0, last = 0, seen = 0;  // as above
      uint32_t patches = 0;
      uint32_t p_dst = 0, p_full = 0, stale = 0;  // the V tile that waits to be mended, and its rows (0: none waits)
      bool ok = true;
      auto fetch = [&](int u, Unit& to) {
        const int slot = u & (kSlots - 1);
        to.nt = -1;
        if (!(ok = warp_wait<Job::kWaitNs>(ctl + kBarSched + 8 * slot, (u / kSlots) & 1, abort_flag))) return;
        to = units[slot];
        __syncwarp();
        if (lane == 0) mbar_arrive(ctl + kBarSchedFree + 8 * slot);
      };
      // Whatever lies in the rows of a V tile that hold no token is made 0, since 0 x NaN is NaN.
      auto mend = [&]() {
#pragma unroll 1
        for (int i = lane; i < (int)(stale >> 24) * 16; i += 32) {
          const int first = (stale >> 8) & 255, n = i >> 4, row = n < first ? (stale & 255) + n : ((stale >> 16) & 255) + n - first;
          *reinterpret_cast<uint4*>(sm + (p_dst - sbase) + Job::v_row(row, (i >> 3) & 1) + (i & 7) * 16) = make_uint4(0, 0, 0, 0);
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(p_full);
        ++patches;
        stale = 0;
      };
      // A stage's release, or with `landed` only the tile to be mended, which meanwhile is mended as soon as it is in.
      auto wait = [&](uint32_t bar, uint32_t parity, bool landed) {
        if (!stale) return warp_wait<Job::kWaitNs>(bar, parity, abort_flag);  // (a suspended wait leaves the issue slots to others)
        uint64_t t0 = 0;
        for (uint32_t it = 1;; ++it) {
          int f = 0;
          if (lane == 0) {
            if (stale && mbar_test(ctl + kBarPatch, patches & 1)) f = 2;
            else if (!landed && mbar_test(bar, parity)) f = 1;
            else if ((it & 63) == 0) {
              const uint64_t now = globaltimer_ns();
              if (t0 == 0) t0 = now;
              if (*abort_flag || now - t0 > Job::kWaitNs) {
                *abort_flag = 1;
                f = 3;
              }
            }
          }
          f = __shfl_sync(0xffffffffu, f, 0);
          if (f == 3) return false;
          if (f == 2) mend();
          if (f == 1 || (landed && f == 2)) return true;
        }
      };
      auto load = [&](const Unit& now, const Places& at, int j, int page) {
        const uint32_t n = Job::kLongPair > 0 ? from + at.v(j) : from + 1;
        const uint32_t st = n % kStages, dst = sbase + kRing + st * kTile, full = ctl + kBarFull + 8 * (n % kFulls);
        const uint32_t rows = job.stale_rows(now, j);
        // The stage's release, then, since one tile waits at a time, the one before (one wait in the code: it is inlined).
#pragma unroll 1
        for (int landed = n < (uint32_t)kStages; ok && landed < (rows && stale ? 2 : 1); ++landed)
          ok = wait(ctl + kBarEmpty + 8 * ((n - kStages) % kFulls), ((n - kStages) / kFulls) & 1, landed != 0);
        if (!ok) return;
        uint32_t bar = full;
        if (rows) {
          stale = rows;
          p_dst = dst;
          p_full = full;
          bar = ctl + kBarPatch;
        }
        if (lane == 0) mbar_arrive_expect_tx(bar, kTile);
        __syncwarp();
        job.load_tile(now, j, 1, page, dst, bar, lane);
        if (Job::kLongPair > 0) {
          seen = seen << (n - last) | 1;
          last = n;
        } else {
          from += 2;
        }
      };
      Unit x, y;
      fetch(0, x);
      bool pair = ok && x.nt >= 0 && x.mode == kFirst;
      if (pair) fetch(1, y);
      int page_x = ok && x.nt >= 0 ? job.page(x, 0, lane) : 0, page_y = ok && pair ? job.page(y, 0, lane) : 0;
      for (int u = 0; ok && x.nt >= 0;) {
        const int tiles = pair ? max(x.nt, y.nt) : x.nt, both = pair ? min(x.nt, y.nt) : 0;
        const Places at_x = places<Job>(both, false), at_y = places<Job>(both, true);
        for (int j = 0; j < tiles && ok; ++j) {
#pragma unroll 1
          for (int e = 0; e < (pair ? 2 : 1) && ok; ++e) {  // (one copy of a load's code)
            const Unit z = e ? y : x;
            if (j >= z.nt) continue;
            load(z, e ? at_y : at_x, j, e ? page_y : page_x);
            const int next = j + 1 < z.nt ? job.page(z, j + 1, lane) : 0;
            if (e) page_y = next;
            else page_x = next;
          }
        }
        if (!ok) break;
        if (Job::kLongPair > 0) from += 2 * (x.nt + (pair ? y.nt : 0));
        u += pair ? 2 : 1;
        fetch(u, x);
        if (!ok) break;
        pair = x.nt >= 0 && x.mode == kFirst;
        if (pair) fetch(u + 1, y);
        if (!ok) break;
        page_x = x.nt >= 0 ? job.page(x, 0, lane) : 0;
        page_y = pair ? job.page(y, 0, lane) : 0;
      }
      if (ok && stale) ok = wait(0, 0, true);
      if (Job::kLongPair == 0) {
        last = from - 1;
        seen = 0x155u & ((1u << min(from, 31u)) - 1);
      }
      if (lane == 0) flight[1] = {last, seen, stale ? p_full : 0, patches & 1};
    } else if (warp >= kOutWarp) {
      // ---------------------------------------------------------------- results
      const int r = tid & 127;
      const uint32_t o_addr = tmem + kTmemO + ((uint32_t)((warp & 3) * 32) << 16);
      const float2* xch = reinterpret_cast<const float2*>(sm + kXch);
      uint32_t c[2] = {0, 0};  // each group's units so far
      if (warp == kOutWarp) job.begun();
      for (int u = 0;; ++u) {
        const int slot = u & (kSlots - 1);
        if (!lanes_wait<Job>(ctl + kBarSched + 8 * slot, (u / kSlots) & 1, abort_flag)) break;
        const Unit& x = units[slot];
        const int mode = x.mode;
        if (x.nt < 0) break;
        bool ok = true;
        typename Job::Row row;
        if (mode == kJoint) {  // the two groups' sums
          job.find_row(x, 0, r, row);
          for (int g = 0; g < 2 && ok; ++g)
            ok = lanes_wait<Job>(ctl + kBarML + 8 * g, c[g] & 1, abort_flag) && lanes_wait<Job>(ctl + kBarO + 8 * g, c[g] & 1, abort_flag);
          if (!ok) break;
          const float2 p = xch[r], q = xch[128 + r];
          const float m = fmaxf(p.x, q.x), ref = m == -INFINITY ? 0.f : m, wp = exp2f(p.x - ref), wq = exp2f(q.x - ref);
          tc_fence_after();
          job.out(x, row, o_addr, o_addr + 128, true, wp, wq, m, p.y * wp + q.y * wq, [&]() {
            tc_fence_before();
            __syncwarp();
            if (lane < 2) mbar_arrive(ctl + kBarOFree + 8 * lane);
          }, again);
          ++c[0];
          ++c[1];
        } else {
          for (int g = 0; g < 2; ++g) {
            if (!takes_part(mode, g)) continue;
            job.find_row(x, g, r, row);
            ok = lanes_wait<Job>(ctl + kBarML + 8 * g, c[g] & 1, abort_flag) && lanes_wait<Job>(ctl + kBarO + 8 * g, c[g] & 1, abort_flag);
            if (!ok) break;
            const float2 p = xch[g * 128 + r];
            tc_fence_after();
            job.out(x, row, o_addr + g * 128, 0, false, 1.f, 0.f, p.x, p.y, [&]() {
              tc_fence_before();
              __syncwarp();
              if (lane == 0) mbar_arrive(ctl + kBarOFree + 8 * g);
            }, again);
            ++c[g];
          }
          if (!ok) break;
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(ctl + kBarSchedFree + 8 * slot);
      }
      __threadfence_block();
      asm volatile("bar.arrive 1, %0;" ::"n"(32 * (kKWarp + 4)) : "memory");
    } else if (warp == kMmaWarp || warp == kMmaWarp + 1) {
      // ---------------------------------------------------------------- products, a warp per group
      // The whole warp walks the group's tiles and one lane issues: operands that are the same in every lane
      // stay in uniform registers, where the instruction takes them from.
      constexpr uint32_t ID_S = idesc(kRows, kTok, false), ID_PV = idesc(kRows, kD, true);
      const int g = warp - kMmaWarp;
      const bool leader = elect_one();
      const uint32_t base = __shfl_sync(0xffffffffu, sbase, 0), tm = __shfl_sync(0xffffffffu, tmem, 0);
      const uint32_t bars = base + kBar, s_t = tm + kTmemS + g * 128, o_t = tm + kTmemO + g * 128;
      const uint64_t q0 = sdesc(base + g * kTile, 16, 1024);
      uint32_t ring = 0;        // stage count of the unit's first tile
      uint32_t n = 0, c = 0;    // the group's tiles, and units in which it had any
      bool ok = true;
      auto wait = [&](uint32_t bar, uint32_t parity) {
        ok = warp_wait<Job::kWaitNs>(bar, parity, abort_flag);
        return ok;
      };
      for (int u = 0; ok; ++u) {
        const int slot = u & (kSlots - 1);
        if (!wait(bars + kBarSched + 8 * slot, (u / kSlots) & 1)) break;
        const int nt = __shfl_sync(0xffffffffu, units[slot].nt, 0), mode = __shfl_sync(0xffffffffu, units[slot].mode, 0),
                  mate = __shfl_sync(0xffffffffu, units[slot].mate, 0);
        if (leader) mbar_arrive(bars + kBarSchedFree + 8 * slot);
        if (nt < 0) break;
        const uint32_t from = ring;
        ring += positions(nt, mode, mate);
        if (!takes_part(mode, g)) continue;
        if (!wait(bars + kBarBegin + 8 * slot, (u / kSlots) & 1)) break;
        const int mine = group_tiles(nt, mode, g);
        Places at = places<Job>(mode == kFirst || mode == kSecond ? min(nt, mate) : 0, mode == kSecond);
        if (mode == kJoint) at = {mine, 2 * g, 1};  // every other tile
        // A stage is free after both groups' use of it; a tile of one group's alone counts twice.
        auto done_with = [&](uint32_t bar) {
          mma_commit(bar);
          if (mode != kDual) mma_commit(bar);
        };
        for (int i = -1; i < mine && ok; ++i) {  // P.V of tile i, then S of tile i + 1
          const uint32_t v_pos = from + (Job::kLongPair > 0 ? at.v(i) : tile_position(mode, mate, g, i) + 1);
          const uint32_t k_pos = from + (Job::kLongPair > 0 ? at.k(i + 1) : tile_position(mode, mate, g, i + 1));
          const uint32_t v_st = v_pos % kStages, k_st = k_pos % kStages;
          const uint32_t v_done = bars + kBarEmpty + 8 * (v_pos % kFulls), k_done = bars + kBarEmpty + 8 * (k_pos % kFulls);
          // The tiles first: once P is there nothing else is waited for between it and the next S.
          if (i + 1 < mine && !wait(bars + kBarFull + 8 * (k_pos % kFulls), (k_pos / kFulls) & 1)) break;
          if (i < 0) {
            if (!wait(bars + kBarQ + 8 * g, c & 1)) break;
          } else {
            if (!wait(bars + kBarFull + 8 * (v_pos % kFulls), (v_pos / kFulls) & 1)) break;
            if (i == 0 && c > 0 && !wait(bars + kBarOFree + 8 * g, (c - 1) & 1)) break;
            const uint64_t v0 = sdesc(base + kRing + v_st * kTile, Job::kVLbo, Job::kVSbo);
            if (!wait(bars + kBarP + 16 * g, (n - 1) & 1)) break;
            tc_fence_after();
            if (leader) {
              mma_ts(o_t, s_t, v0, ID_PV, i > 0 ? 1u : 0u);
#pragma unroll
              for (int kk = 1; kk < kTok / 32; ++kk) mma_ts_add(o_t, s_t + kk * 8, v0 + ((kk * Job::kVStep) >> 4), ID_PV);
            }
            __syncwarp();
            if (!wait(bars + kBarP + 16 * g + 8, (n - 1) & 1)) break;
            tc_fence_after();
            if (leader) {
#pragma unroll
              for (int kk = kTok / 32; kk < kTok / 16; ++kk)
                mma_ts_add(o_t, s_t + kk * 8, v0 + ((kk * Job::kVStep) >> 4), ID_PV);
              done_with(v_done);
              if (i + 1 == mine) mma_commit(bars + kBarO + 8 * g);
            }
            __syncwarp();
          }
          if (i + 1 < mine) {
            ++n;
            tc_fence_after();
            if (leader) {
              const uint64_t k0 = sdesc(base + kRing + k_st * kTile, 16, Job::kKSbo);
              mma_set(s_t, q0, k0, ID_S);
#pragma unroll
              for (int kk = 1; kk < kD / 16; ++kk)
                mma_add(s_t, q0 + (((kk >> 2) * 16384 + (kk & 3) * 32) >> 4),
                        k0 + (((kk >> 2) * Job::kKHalf + (kk & 3) * 32) >> 4), ID_S);
              mma_commit(bars + kBarS + 8 * g);
              done_with(k_done);
            }
            __syncwarp();
          }
        }
        ++c;
      }
    }
  } else {
    regs_inc<kSoftmaxRegs>();
    // ---------------------------------------------------------------- softmax
    const int g = warp >> 2, r = tid & 127;
    const uint32_t lane_base = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t s_addr = tmem + kTmemS + g * 128 + lane_base, o_addr = tmem + kTmemO + lane_base;
    float2* xch = reinterpret_cast<float2*>(sm + kXch);
    const float qscale = job.qscale;
    uint32_t n = 0, c_done = 0;   // tiles of this group, units it is done with
    int u_next = 0;               // the unit read next
    bool alive = true;
    typename Job::Row row, row_y;
    // The group's next unit: its words stay in shared memory until the group is done with it.
    bool known = false;  // the next unit has been found (the same in a warp)
    auto next_unit = [&](int& slot, bool patient) {
      for (;; ++u_next) {
        slot = u_next & (kSlots - 1);
        const uint32_t bar = ctl + kBarSched + 8 * slot, parity = (u_next / kSlots) & 1;
        if (!patient) {
          if (!__all_sync(0xffffffffu, mbar_test(bar, parity))) return true;
        } else if (!warp_wait<Job::kWaitNs>(bar, parity, abort_flag)) {
          return false;
        }
        if (units[slot].nt < 0) break;
        if (takes_part(units[slot].mode, g)) {
          ++u_next;
          break;
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(ctl + kBarSchedFree + 8 * slot);
      }
      known = true;
      return true;
    };
    int sx = 0, sy = 0;
    alive = next_unit(sx, true);
    if (alive && units[sx].nt >= 0) {
      job.find_row(units[sx], g, r, row);
      job.load_q(units[sx], g, r, sbase + g * kTile, ctl + kBarQ + 8 * g, row);
      job.loaded_q(r, ctl + kBarQ + 8 * g);
    }
    // The group's last S of a unit is complete: the next unit's query rows may come.  While P of that tile is due the
    // group does not wait for the unit: where others without the group come first, it is made known only when they are
    // loaded, to which the ring may need the stage of this tile's V.
    auto begin_next = [&](bool patient) {
      if (known) return true;
      if (!next_unit(sy, patient)) return false;
      if (known && units[sy].nt >= 0) {
        job.find_row(units[sy], g, r, row_y);
        job.load_q(units[sy], g, r, sbase + g * kTile, ctl + kBarQ + 8 * g, row_y);
      }
      return true;
    };
    while (alive && units[sx].nt >= 0) {
      const Unit& x = units[sx];
      const int mode = x.mode, mine = group_tiles(x.nt, mode, g);
      float m_ref = -INFINITY, l = 0.f;
      known = false;
      for (int i = 0; i < mine; ++i, ++n) {
        const int t = group_tile(mode, g, i);
        if (!warp_wait<Job::kWaitNs>(ctl + kBarS + 8 * g, n & 1, abort_flag)) { alive = false; break; }
        if (Job::kEarlyQ && i + 1 == mine && !(alive = begin_next(false))) break;
        tc_fence_after();
        uint32_t su[128];
#pragma unroll
        for (int c = 0; c < 128; c += 32) ld32_issue(s_addr + c, su + c);
#pragma unroll
        for (int c = 0; c < 128; c += 32) ld32_wait(su + c);
        float* s = reinterpret_cast<float*>(su);
        const Sees see = job.sees(x, row, t);
        if (!see.all) {
#pragma unroll
          for (int c = 0; c < 64; ++c) s[c] = c < see.limit ? s[c] : -INFINITY;
          if (see.by_bits) {
            const uint32_t half[2] = {(uint32_t)see.bits, (uint32_t)(see.bits >> 32)};
#pragma unroll
            for (int c = 64; c < 128; ++c) s[c] = (half[(c - 64) >> 5] & (1u << (c & 31))) ? s[c] : -INFINITY;
          } else {
#pragma unroll
            for (int c = 64; c < 128; ++c) s[c] = c < see.limit ? s[c] : -INFINITY;
          }
        }
        float mx[4] = {fmaxf(s[0], s[1]), fmaxf(s[2], s[3]), fmaxf(s[4], s[5]), fmaxf(s[6], s[7])};
#pragma unroll
        for (int c = 8; c < 128; c += 8)
#pragma unroll
          for (int k = 0; k < 4; ++k) mx[k] = max3(mx[k], s[c + 2 * k], s[c + 2 * k + 1]);
        const float mt = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * qscale;
        const bool raise = mt > m_ref + 8.f;
        if (i > 0 && __any_sync(0xffffffffu, raise)) {
          const float alpha = raise ? exp2f(m_ref - mt) : 1.f;
#pragma unroll 1
          for (int c0 = 0; c0 < 128; c0 += 32) {
            float o[32];
            tmem_ld32(o_addr + g * 128 + c0, o);
#pragma unroll
            for (int c = 0; c < 32; ++c) o[c] *= alpha;
            tmem_st32(o_addr + g * 128 + c0, o);
          }
          l *= alpha;
        }
        if (raise) m_ref = mt;
        const float neg_m = m_ref == -INFINITY ? 0.f : -m_ref;  // no key seen yet: every p is 0
        const uint64_t sc2 = pack2(qscale, qscale), nm2 = pack2(neg_m, neg_m);
        uint64_t ls[4] = {0ull, 0ull, 0ull, 0ull};  // pairs of fp32 sums
#pragma unroll
        for (int c = 0; c < 128; c += 32) {
          uint32_t pw[16];
#pragma unroll
          for (int k = 0; k < 32; k += 2) {
            float p0, p1;
            unpack2(fma2(pack2(s[c + k], s[c + k + 1]), sc2, nm2), p0, p1);
            p0 = ex2_approx(p0);
            p1 = ex2_approx(p1);
            ls[(k >> 1) & 3] = add2(ls[(k >> 1) & 3], pack2(p0, p1));
            const __nv_bfloat162 a = __floats2bfloat162_rn(p0, p1);
            pw[k / 2] = *reinterpret_cast<const uint32_t*>(&a);
          }
          st16(s_addr + c / 2, pw);
          if (c == 32 || c == 96) {  // half of the tile's keys: the tensor core may begin on them
            st_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(ctl + kBarP + 16 * g + (c == 96 ? 8 : 0));
          }
        }
        float l0, l1;
        unpack2(add2(add2(ls[0], ls[1]), add2(ls[2], ls[3])), l0, l1);
        l += l0 + l1;
      }
      if (!alive) break;
      if (!(alive = begin_next(true))) break;
      if (units[sy].nt >= 0) job.loaded_q(r, ctl + kBarQ + 8 * g);
      // (m, l) go to the warps that write, once they have those of the group's unit before.
      if (c_done > 0 && !(alive = warp_wait<Job::kWaitNs>(ctl + kBarOFree + 8 * g, (c_done - 1) & 1, abort_flag))) break;
      ++c_done;
      xch[g * 128 + r] = make_float2(m_ref, l);
      __syncwarp();
      if (lane == 0) mbar_arrive(ctl + kBarML + 8 * g);
      __syncwarp();
      if (lane == 0) mbar_arrive(ctl + kBarSchedFree + 8 * sx);
      sx = sy;
      row = row_y;
    }
    // All rows are written (see one_row).
    asm volatile("bar.sync 1, %0;" ::"n"(32 * (kKWarp + 4)) : "memory");
    if (*again && !*abort_flag) {
      const typename Job::Units all(job);
      const int total = job.total(all);
#pragma unroll 1
      for (int u = 0; unit_id(u) < total; ++u) {
        Unit x;
        job.unit(all, unit_id(u), x);
        job.again(x, warp);
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  // Given up: no role issues anything more.  What each has in flight ends before the tensor memory is freed and the CTA leaves
  // (bounded).  (Only here does every role know: one that came to its end before another gave up would have looked too early.)
  if (*abort_flag) {
    if (tid == 0) job.error(GB_ERR_TIMEOUT);
    if (warp < kKWarp) {
      job.drain_q(ctl + kBarQ + 8 * (warp >> 2));
    } else if ((warp == kKWarp || warp == kVWarp) && lane == 0) {
      const Flight f = flight[warp == kVWarp];
      if (f.patched) mbar_wait_bounded(ctl + kBarPatch, f.patch_parity, Job::kWaitNs / 8);
      for (uint32_t i = 0; i < 2 * kStages; ++i) {
        const uint32_t bar = ctl + kBarFull + 8 * ((f.last - i) % kFulls);
        if (((f.seen >> i) & 1) && bar != f.patched) mbar_wait_bounded(bar, ((f.last - i) / kFulls) & 1, Job::kWaitNs / 8);
      }
    } else if (warp == kMmaWarp || warp == kMmaWarp + 1) {
      // (a commit by the lane that issued them stands for all its products, S and P.V)
      const uint32_t bar = ctl + kBarDrained + 8 * (warp - kMmaWarp);
      if (elect_one()) {
        mma_commit(bar);
        mbar_wait_bounded(bar, 0, Job::kWaitNs / 8);
      }
      __syncwarp();
    }
    __syncthreads();
  }
  tc_fence_after();
  if (warp == kMmaWarp) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512));
}

}  // namespace flash
}  // namespace gb
