// The next token of each row of logits, from a given random number.
//
// With max the row's largest logit and w_i = exp((x_i - max) / T), the tokens are taken in descending order of (x, -index):
//   top-k   keeps the first k of them,
//   min-p   of these the ones with w_i >= min_p,
//   top-p   of these the shortest head whose mass reaches top_p of theirs,
// so what is kept is always a head of that order: the tokens with x > K, and those with x = K up to some index.  The token is
// the first, by index, at which the kept tokens' mass passes u times its total.
//
// A token is compared against sums over the whole vocabulary, so masses are whole numbers: w in units of 2^-44, right to 2^-28 of
// itself (weights_of) and half a unit, summed in 64 bits.  Sums are then the same in any order, and no draw depends on how the row
// was split.  (Tokens below 2^-24 of the largest enter top-p's total by exp2f of an fp32 exponent: right to 2^-17 of themselves, as
// the exponent, up to 46, has three roundings of 2^-24.)
//
// A cluster of CTAs a row, which reads it two to four times; all but the first time from L2:
//   1. the largest logit; with top-k a value that at least k tokens reach, of the threads' largest,
//   2. for top-p, the row's mass and the masses of 1024 slices of the exponent (slice_masses),
//   3. a list of the tokens that can be kept, for the first CTA, which orders, cuts and draws in it (draw_listed).
// Where more than kCap tokens stay, pass 3 sums the mass of runs of 32 pieces instead and lists only the slices that hold the
// cut (top_p_runs), and the draw finds its run, then its token.  What has no bound of either kind goes a digit of the key at a
// time over the whole row (cut).
//
// What bounds it: at many rows the weights (36 issue slots a token, and a shared atomic in pass 2), not the bytes: 512 rows of
// 128000 bf16 take 141 us for 19 us of reading (0.93 TB/s), 64 rows of 151000 fp32 65 us for 6; at few, a chain of passes and
// cluster barriers of 1-4 us each: 8 rows of 32000 with top-k take 11 us, greedy rows 3.
#include <cuda_bf16.h>
#include <math.h>

#include <algorithm>

#include "internal.cuh"

namespace gb {
namespace {

constexpr int kThreads = 512;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxVocab = 1 << 19;      // masses stay under 2^63
constexpr int kUnit = 44;               // a weight of one is 2^44
constexpr int kBins = 256, kDigits = 4, kDigitBits = 12;
constexpr int kMaxCluster = 8;
constexpr float kFar = 46.f;            // weights of 2^-46 and less count as none
constexpr int kCap = 4096;              // tokens of the first CTA's list, in which a row is decided
constexpr int kRanked = 256;            // lists up to this long are ranked by comparing every two entries
constexpr int kSlices = 1024;           // of the weights' exponents, 22 to a power of two
constexpr int kPerPower = 22;
static_assert(kFar * kPerPower < kSlices, "every weight has a slice");
typedef unsigned long long u64;

// 2^(-j/256) in units of 2^-31: the power series of exp in 64 bits, as the compiler evaluates it.
struct PowerTable {
  uint32_t t[kBins];
  constexpr PowerTable() : t() {
    for (int j = 0; j < kBins; ++j) {
      const double x = -0.69314718055994530942 * j / kBins;
      double term = 1, sum = 0;
      for (int n = 1; n < 30; ++n) {
        sum += term;
        term *= x / n;
      }
      t[j] = (uint32_t)(sum * (double)(1u << 31) + 0.5);
    }
  }
};
__device__ const PowerTable kPowers;

struct Job {
  const void* logits;
  long long stride;
  int rows, vocab, cluster;
  const float *u, *temperature, *top_p, *min_p;
  const int* top_k;
  float all_temperature, all_top_p, all_min_p;
  int all_top_k;
  int* token;
  float* logprob;
};

// ---- clusters ----------------------------------------------------------------------------------
__device__ __forceinline__ unsigned cluster_rank() {
  unsigned r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t peer_addr(const void* p, unsigned rank) {
  uint32_t a;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
  return a;
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ uint32_t peer_load(uint32_t a) {
  uint32_t x;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(x) : "r"(a) : "memory");
  return x;
}
__device__ __forceinline__ void peer_store32(uint32_t a, uint32_t x) {
  asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(a), "r"(x) : "memory");
}
__device__ __forceinline__ void peer_store64(uint32_t a, u64 x) {
  asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(a), "l"(x) : "memory");
}

// ---- keys and weights ----------------------------------------------------------------------------

// Larger x, larger key; the two zeros are one; what is not a number comes below everything.
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);
  return x != x ? 0u : (b & 0x80000000u) ? ~b : b | 0x80000000u;
}

struct Row {
  float max, ch, cl;  // log2(e) / T in two terms
};

// y = (max - x) log2(e) / T to fp32, which alone says a token's slice.
__device__ __forceinline__ float exponent(const Row& row, float x) { return __fmul_rn(__fsub_rn(row.max, x), row.ch); }

// exp((x - max) / T) = m 2^-31 2^-n with m in (2^30, 2^31], for a logit with exponent() below kFar; j = floor(256 y), n = j >> 8.
// y is taken to 2^-40 of itself or better; m is the table's 2^(-(j & 255)/256) less its share 1 - 2^-r, 0 <= r < 2^-8, to the
// third order and in units of 2^-31.  Together within 3 units: half of one in the table, one that the product's floor cuts off, half
// in q and as much in its terms' roundings; 2^-29.0 of the weight is the most that 40 million of them were off.
// Two at a time, as the fp32 units take them; of other logits something without meaning.
struct Weight {
  uint32_t m;
  int j;
};
__device__ __forceinline__ float2 two(float x) { return make_float2(x, x); }
__device__ __forceinline__ float2 minus(float2 x) { return make_float2(-x.x, -x.y); }
__device__ __forceinline__ void weights_of(const Row& row, const uint32_t* table, float2 x, Weight (&w)[2]) {
  const float2 top = two(row.max), ch = two(row.ch), nx = minus(x);
  const float2 d = __fadd2_rn(top, nx), b = __fadd2_rn(d, minus(top));
  const float2 e = __fadd2_rn(__fadd2_rn(top, __fadd2_rn(b, minus(d))), __fadd2_rn(nx, minus(b)));
  const float2 yh = __fmul2_rn(d, ch);
  const float2 yl = __fadd2_rn(__ffma2_rn(d, ch, minus(yh)), __ffma2_rn(d, two(row.cl), __fmul2_rn(e, ch)));
  const float2 z = __fadd2_rd(yh, two(49152.f));           // down to a multiple of 2^-8
  const float2 r = __fadd2_rn(__fadd2_rn(yh, minus(__fadd2_rn(z, two(-49152.f)))), yl);
  constexpr float kLn2 = 0.69314718055994530942f, k31 = 0x1p31f, kBase = 0x1.4p23f;
  float2 q = __ffma2_rn(r, two(k31 * kLn2 * kLn2 * kLn2 / 6), two(-k31 * kLn2 * kLn2 / 2));
  q = __fadd2_rn(__fmul2_rn(r, __ffma2_rn(r, q, two(k31 * kLn2))), two(kBase));  // rounds; q < 0 where yl pulls y under its multiple
  const float zs[2] = {z.x, z.y}, qs[2] = {q.x, q.y};
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int less = 2 * (__float_as_int(qs[i]) - __float_as_int(kBase));
    w[i].j = __float_as_int(zs[i]) - __float_as_int(49152.f);
    const uint32_t t = table[w[i].j & 255];
    w[i].m = t + (uint32_t)__mulhi(-(int)t, less);         // (-t: at least -2^31)
  }
}
// The same in units of 2^-44.
__device__ __forceinline__ u64 mass_of(const Weight& w) {
  const int n = w.j >> 8, sh = max(n - (kUnit - 31), 0);
  const uint32_t m = (w.m + ((1u << sh) >> 1)) >> sh;      // (sh <= 32: a shift by 32 gives 0 on the GPU)
  return (u64)m << max(kUnit - 31 - n, 0);
}
__device__ __forceinline__ u64 weight(const Row& row, const uint32_t* table, float x) {
  if (!(x > -INFINITY)) return 0;
  if (x == row.max) return 1ull << kUnit;
  if (!(exponent(row, x) < kFar)) return 0;
  Weight w[2];
  weights_of(row, table, two(x), w);
  return mass_of(w[0]);
}

// Slices of the exponent, kPerPower to a power of two: floor(kPerPower j / 256).  Their masses are summed in units of
// 2^slice_shift, 12 bits of a weight.
__device__ __forceinline__ int slice_of(const Weight& w) { return w.j * kPerPower >> 8; }
__device__ __forceinline__ uint32_t slice_part(const Weight& w) { return w.m >> max(19, (w.j >> 8) - (kUnit - 31)); }
__device__ __forceinline__ int slice_shift(int b) { return max(0, 32 - b / kPerPower); }
// The exponent that slice b begins at: tokens with exponent() below it are in the slices before.
__device__ __forceinline__ float slice_begin(int b) { return (float)((b * 256 + kPerPower - 1) / kPerPower) * (1.f / 256); }

__device__ __forceinline__ unsigned value(const float* p) { return __float_as_uint(*p); }
__device__ __forceinline__ unsigned value(const __nv_bfloat16* p) { return __bfloat16_as_ushort(*p); }
__device__ __forceinline__ void values(const uint4& v, float (&x)[4]) {
  x[0] = __uint_as_float(v.x);
  x[1] = __uint_as_float(v.y);
  x[2] = __uint_as_float(v.z);
  x[3] = __uint_as_float(v.w);
}
__device__ __forceinline__ void values(const uint4& v, float (&x)[8]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}

// A row in pieces of 16 bytes from the 16-byte boundary at or before its start on: piece v holds the tokens
// v * N - off ..; a lane's piece.  Where a piece passes the row's ends its missing values are -infinity.
template <typename T>
struct Pieces {
  static constexpr int N = 16 / (int)sizeof(T);
  const T* x;
  int vocab, off, count;
  __device__ Pieces(const T* row, int n) : x(row), vocab(n) {
    off = (int)(((uintptr_t)row & 15) / sizeof(T));
    count = (off + n + N - 1) / N;
  }
  __device__ __forceinline__ uint4 bits(int v) const {
    const int i0 = v * N - off;
    if (v < count && i0 >= 0 && i0 + N <= vocab) return __ldg(reinterpret_cast<const uint4*>(x + i0));
    constexpr unsigned kNone = sizeof(T) == 4 ? 0xff800000u : 0xff80u;  // -infinity
    uint32_t w[4] = {};
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const bool in = v < count && i0 + e >= 0 && i0 + e < vocab;
      w[e * (int)sizeof(T) / 4] |= (in ? value(x + i0 + e) : kNone) << (e * (int)sizeof(T) % 4 * 8);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
  __device__ __forceinline__ void load(int v, float (&f)[N]) const { values(bits(v), f); }
  // f(v, its values) of the pieces v = first, first + step, ... below `end`, the same number for every lane of a warp (end: for
  // lane 0); `Ahead` loads at a time.
  template <int Ahead, class F>
  __device__ __forceinline__ void scan(int first, int end, int step, F f) const {
    const int lane = threadIdx.x & 31;
    for (int v0 = first; v0 < end; v0 += Ahead * step) {
      uint4 b[Ahead];
#pragma unroll
      for (int a = 0; a < Ahead; ++a) b[a] = bits(v0 + a * step + lane);
#pragma unroll
      for (int a = 0; a < Ahead; ++a) {
        if (v0 + a * step >= end) break;
        float y[N];
        values(b[a], y);
        f(v0 + a * step + lane, y);
      }
    }
  }
};

// ---- the row's CTAs ----------------------------------------------------------------------------------

struct Entry {
  float x;
  int i;
};

// What is kept: the tokens with key > k, and those with key = k and index <= i.
struct Head {
  uint32_t k;
  int i;
};
__device__ __forceinline__ bool kept(const Head& h, uint32_t key, int i) { return key > h.k || (key == h.k && i <= h.i); }

struct Top {
  float max;
  int arg;
  uint32_t bound;
  uint32_t pad;
};

struct Smem {
  uint32_t table[kBins];
  Entry list[kCap];
  union {
    u64 weights[kCap];                   // of the list, once it is whole
    u64 runs[(kMaxVocab / 4 + 2 + 31) / 32];  // the first CTA's: mass of each run of 32 pieces
  };
  float queue[kWarps][64 + 32 * 8];      // logits that wait for their weights
  u64 order[kRanked];                    // tokens to be ranked, (key from above, index), and their weights
  u64 ranked[kRanked];
  Entry places[kRanked];                 // a short list in order
  uint32_t slice[kSlices];               // masses by slice, see top_p_list
  uint32_t hist[1 + kDigits][kBins];     // counts, then the masses' digits
  u64 total[kBins];
  Top tops[kMaxCluster];                 // of the row's CTAs
  Head head;
  double ahead;                          // T ln(min_p)
  float least;
  int listed, ranks, token;
  int lo, hi, many;                      // top-p: the slices that its cut can lie in, whether it keeps more than a list holds
  float red[kWarps];
  int redi[kWarps];
  u64 red64[kWarps];
  u64 before;                            // of the bin chosen
  int bin;
  u64 sum;
};

// (The GPU's 64-bit floating point runs at a sixtieth of its 32-bit rate, so what every thread needs is in whole numbers.)
// floor(f n) of 0 <= f < 1, exactly, and whether f n is more.
__device__ __forceinline__ bool product(float f, u64 n, u64* below) {
  const uint32_t b = __float_as_uint(f);
  const int e = (int)(b >> 23), shift = 150 - (e ? e : 1);   // f = m 2^-shift
  const u64 m = e ? (b & 0x7fffffu) | 0x800000u : b & 0x7fffffu;
  const u64 lo = n * m, hi = __umul64hi(n, m);
  if (shift >= 128) {
    *below = 0;
    return (lo | hi) != 0;
  }
  if (shift >= 64) {
    *below = hi >> (shift - 64);
    return lo != 0 || (hi & ((1ull << (shift - 64)) - 1)) != 0;
  }
  *below = (lo >> shift) | (hi << (64 - shift));
  return (lo & ((1ull << shift) - 1)) != 0;
}
// The token drawn is the first at which the kept mass passes this.
__device__ __forceinline__ u64 draw_at(float u, u64 total) {
  if (!(u > 0.f)) return 0;
  if (u >= 1.f) return total - 1;
  u64 t;
  product(u, total, &t);
  return t;
}
// ln(w / total)
__device__ __forceinline__ float log_share(float x, float m, float temperature, u64 total) {
  const double y = x == m ? 0.0 : ((double)x - (double)m) / (double)temperature;
  return (float)(y - log((double)total * 0x1p-44));
}

// A warp's queue of values.
struct Queue {
  float* at;
  int n;
  // Elements e of x where bit e of `mine` is set, lane after lane.
  template <int N>
  __device__ __forceinline__ void put(const float (&x)[N], unsigned mine) {
    const int lane = threadIdx.x & 31, own = __popc(mine);
    int inc = own;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += y;
    }
    int to = n + inc - own;
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (mine >> e & 1) at[to++] = x[e];
    n += __shfl_sync(0xffffffffu, inc, 31);
    __syncwarp();
  }
  // f of the last `some` <= 64, two at a time: f(two values, which of them).
  template <class F>
  __device__ __forceinline__ void take(int some, F f) {
    const int lane = threadIdx.x & 31;
    const float* from = at + n - some;
    if (lane < some) {
      const bool both = lane + 32 < some;
      const float x = from[lane];
      f(make_float2(x, both ? from[lane + 32] : x), both ? 3u : 1u);
    }
    n -= some;
    __syncwarp();
  }
};

// The kernel's shared memory, by its name: through a pointer that a function was given, the accesses of a function that is not
// inlined are generic ones, whose atomics are ten times slower.
extern __shared__ __align__(16) unsigned char sample_smem[];
#define sm (*reinterpret_cast<Smem*>(sample_smem))

template <typename T>
struct RowCtas {
  const Pieces<T> pieces;
  const Row row;
  const unsigned rank, ctas;
  static constexpr int N = Pieces<T>::N;

  // f(value, token) of every token, spread over the row's CTAs.
  template <class F>
  __device__ __forceinline__ void each(F f) const {
    const int step = (int)(ctas * kThreads);
#pragma unroll 2
    for (int v = (int)(rank * kThreads + threadIdx.x); v < pieces.count; v += step) {
      float x[N];
      pieces.load(v, x);
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const int i = v * N - pieces.off + e;
        if (i >= 0 && i < pieces.vocab) f(x[e], i);
      }
    }
  }
  // The same of the first n tokens of this CTA's list.
  template <class F>
  __device__ __forceinline__ void each_listed(int n, F f) const {
    for (int j = threadIdx.x; j < n; j += kThreads) f(sm.list[j].x, sm.list[j].i);
  }
  // f(value, token, weight), of those with a weight in sm.weights.
  template <class F>
  __device__ __forceinline__ void each_weighed(int n, F f) const {
    for (int j = threadIdx.x; j < n; j += kThreads) {
      const u64 w = sm.weights[j];
      if (w) f(sm.list[j].x, sm.list[j].i, w);
    }
  }

  // One digit of a selection among the row's tokens (n < 0) or this CTA's first n listed ones: the bin in which the running
  // total (of counts or masses, by bin in ascending order) reaches `target` > 0, and the total before it.  bin(x, i): a token's
  // bin, or -1; weigh: by mass.
  template <class B>
  __device__ void digit(int n, bool weigh, u64 target, B bin) {
    for (int t = threadIdx.x; t < (1 + kDigits) * kBins; t += kThreads) (&sm.hist[0][0])[t] = 0;
    __syncthreads();
    auto count = [&](float x, int i) {
      const int b = bin(x, i);
      if (b < 0) return;
      if (!weigh) {
        atomicAdd(&sm.hist[0][b], 1u);
        return;
      }
      const u64 w = weight(row, sm.table, x);
#pragma unroll
      for (int d = 0; d < kDigits; ++d) {
        const uint32_t part = (uint32_t)(w >> (d * kDigitBits)) & ((1u << kDigitBits) - 1);
        if (part) atomicAdd(&sm.hist[1 + d][b], part);
      }
    };
    if (n < 0) {
      each(count);
      cluster_sync();
    } else {
      each_listed(n, count);
      __syncthreads();
    }
    for (int b = threadIdx.x; b < kBins; b += kThreads) {
      u64 t = 0;
      const unsigned first = n < 0 ? 0 : rank, last = n < 0 ? ctas : rank + 1;
      for (unsigned c = first; c < last; ++c) {
        if (!weigh) {
          t += peer_load(peer_addr(&sm.hist[0][b], c));
        } else {
          for (int d = 0; d < kDigits; ++d) t += (u64)peer_load(peer_addr(&sm.hist[1 + d][b], c)) << (d * kDigitBits);
        }
      }
      sm.total[b] = t;
    }
    if (n < 0) cluster_sync();
    else __syncthreads();
    if (threadIdx.x < 32) {
      const int lane = threadIdx.x;
      u64 own = 0;
      for (int b = 0; b < kBins / 32; ++b) own += sm.total[lane * (kBins / 32) + b];
      u64 inc = own;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const u64 y = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += y;
      }
      const unsigned past = __ballot_sync(0xffffffffu, inc >= target);
      const int l = past ? __ffs(past) - 1 : 31;
      if (lane == l) {
        u64 before = inc - own;
        int b = lane * (kBins / 32);
        const int last = b + kBins / 32 - 1;
        while (b < last && before + sm.total[b] < target) before += sm.total[b++];
        sm.bin = b;
        sm.before = before;
      }
    }
    __syncthreads();
  }

  // Cut the head where its running total (counts, or masses) reaches `target`, 1 <= target <= the head's total.  n: digit()'s.
  __device__ Head cut(const Head& h, int n, bool weigh, u64 target) {
    const uint32_t top = key_of(row.max);
    uint32_t at = 0;                       // of top - key, the digits chosen so far
    u64 of = 0;                            // the last one's bin's total
    for (int s = 24; s >= 0; s -= 8) {
      digit(n, weigh, target, [&](float x, int i) {
        const uint32_t key = key_of(x), rel = top - key;
        return kept(h, key, i) && (s == 24 || rel >> (s + 8) == at >> (s + 8)) ? (int)(rel >> s & 255u) : -1;
      });
      at |= (uint32_t)sm.bin << s;
      target -= sm.before;
      of = sm.total[sm.bin];
      __syncthreads();
    }
    if (at > top || top - at < h.k) return h;   // (the total stays below the target: all of the head)
    // The key is chosen; of its tokens, all of one weight, the first ones by index.
    Head to = {top - at, h.k == top - at ? h.i : 0x7fffffff};
    if (target >= of) return to;
    u64 most = target;
    if (weigh) {
      const u64 w = weight(row, sm.table, key_value(to.k));
      most = (target + w - 1) / w;
      if (most * w >= of) return to;
    }
    to.i = min(to.i, by_index(n, false, most, [&](float x, int i) { return key_of(x) == to.k && i <= to.i; }));
    return to;
  }

  // The order of this CTA's sm.ranks <= kRanked tokens in sm.order: f(token's number, the mass of those before it, its own),
  // for each by one thread, which compares it with all the others, together with its neighbours.
  template <class F>
  __device__ __forceinline__ void rank_each(F f) const {
    const int n = sm.ranks, shift = n <= kRanked / 4 ? 3 : n <= kRanked / 2 ? 2 : 1, ways = 1 << shift;
    const int j = threadIdx.x >> shift, way = threadIdx.x & (ways - 1);
    const u64 own = sm.order[j < n ? j : 0];
    u64 before = 0;
#pragma unroll 4
    for (int z = way; z < n; z += ways) {
      const u64 w = sm.ranked[z];
      before += sm.order[z] < own ? w : 0;
    }
    for (int o = 1; o < ways; o <<= 1) before += __shfl_xor_sync(0xffffffffu, before, o);
    if (j < n && way == 0) f(j, before, sm.ranked[j]);
  }
  __device__ __forceinline__ void to_rank(u64 order, u64 w) const {
    const int at = atomicAdd(&sm.ranks, 1);
    if (at < kRanked) {
      sm.order[at] = order;
      sm.ranked[at] = w;
    }
  }

  // cut() by mass of the head h of this CTA's list (each(f): f(value, token, weight) of its tokens in h) where the tokens with
  // an exponent below `begin` are known to stay.
  template <class Each>
  __device__ Head cut_listed(const Head& h, int n, float begin, u64 target, Each each_of) {
    if (threadIdx.x == 0) {
      sm.ranks = 0;
      sm.head = h;
    }
    __syncthreads();
    u64 above = 0;
    each_of([&](float x, int i, u64 w) {
      if (exponent(row, x) < begin) above += w;
      else to_rank((u64)~key_of(x) << 32 | (unsigned)i, w);
    });
    above = block_sum(above);
    if (sm.ranks > kRanked) return cut(h, n, true, target);
    rank_each([&](int j, u64 before, u64 w) {
      before += above;
      if (before < target && target <= before + w) sm.head = {~(uint32_t)(sm.order[j] >> 32), (int)(uint32_t)sm.order[j]};
    });
    __syncthreads();
    return sm.head;
  }

  // The index at which the running total of the tokens that in(x, i) says, taken by index, reaches `target`.
  template <class In>
  __device__ int by_index(int n, bool weigh, u64 target, In in) {
    int index = 0;
    for (int s = 16; s >= 0; s -= 8) {     // (indexes are below 2^19)
      digit(n, weigh, target, [&](float x, int i) {
        return in(x, i) && (s == 16 || i >> (s + 8) == index >> (s + 8)) ? i >> s & 255 : -1;
      });
      index |= sm.bin << s;
      target -= sm.before;
      __syncthreads();
    }
    return index;
  }

  // This CTA's sum, in every thread.
  __device__ u64 block_sum(u64 s) {
#pragma unroll
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if ((threadIdx.x & 31) == 0) sm.red64[threadIdx.x >> 5] = s;
    __syncthreads();
    u64 t = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) t += sm.red64[w];
    __syncthreads();
    return t;
  }

  // The sum of the threads' before this one, and of all.
  __device__ u64 block_before(u64 s, u64* all) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    u64 inc = s;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const u64 y = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += y;
    }
    if (lane == 31) sm.red64[warp] = inc;
    __syncthreads();
    u64 before = inc - s, t = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const u64 x = sm.red64[w];
      before += w < warp ? x : 0;
      t += x;
    }
    *all = t;
    __syncthreads();
    return before;
  }

  // Room for the warp's `mine` entries each in this CTA's list.
  __device__ __forceinline__ int reserve(int mine) const {
    const int lane = threadIdx.x & 31;
    int inc = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += y;
    }
    int at = 0;
    if (lane == 31) at = atomicAdd(&sm.listed, inc);
    return __shfl_sync(0xffffffffu, at, 31) + inc - mine;
  }
  __device__ __forceinline__ void put(int at, float x, int i) const {
    if (at < kCap) sm.list[at] = {x, i};
  }
  // The row's tokens that in(x, i) says into the lists of the CTAs that read them, in no order.
  template <class In>
  __device__ __forceinline__ void gather(In in) const {
    pieces.template scan<4>((int)(rank * kThreads) + (int)(threadIdx.x & ~31u), pieces.count, (int)(ctas * kThreads), [&](int v, const float (&x)[N]) {
      unsigned mine = 0;
#pragma unroll
      for (int e = 0; e < N; ++e) mine |= x[e] > -INFINITY && in(x[e], v * N - pieces.off + e) ? 1u << e : 0u;
      if (!__any_sync(0xffffffffu, mine != 0)) return;
      int at = reserve(__popc(mine));
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (mine >> e & 1) put(at++, x[e], v * N - pieces.off + e);
    });
  }
  // The CTAs' lists behind the first one's.  Their length together, and where it is above kCap only that.
  __device__ int join_lists() const {
    cluster_sync();
    int n = 0, own = 0, at = 0;
    for (unsigned c = 0; c < ctas; ++c) {
      const int there = (int)peer_load(peer_addr(&sm.listed, c));
      if (c < rank) at += there;
      if (c == rank) own = there;
      n += there;
    }
    if (rank != 0 && n <= kCap) {
      const uint32_t to = peer_addr(&sm.list[at], 0);
      for (int j = threadIdx.x; j < own; j += kThreads)
        peer_store64(to + j * (uint32_t)sizeof(Entry), (u64)__float_as_uint(sm.list[j].x) | (u64)(unsigned)sm.list[j].i << 32);
    }
    cluster_sync();
    return n;
  }

  // Sums the weights of the tokens with x >= least, and those that top-p can keep by slices of their exponent, to 12 bits
  // each.  Tokens below 2^-24 (`far`) are only summed, from the 22 bits of exp2f.  The others' weights take 36 issue slots, so a warp
  // puts their logits in a queue of its own and takes 64 at a time from it: as they lie in the row, most turns of a warp would have
  // only a few.  Tokens so light that all of them together could not be the share 1 - p that goes need no slice (`can`).
  __device__ u64 slice_masses(float p, float least, float own_max) {
    for (int b = threadIdx.x; b < kSlices; b += kThreads) sm.slice[b] = 0;
    // From below, log2 of all's mass: that of the threads' largest tokens.  (Each CTA has bounds of its own.)
    float some = own_max >= least ? exp2f(-exponent(row, own_max)) : 0.f;
#pragma unroll
    for (int o = 16; o; o >>= 1) some += __shfl_xor_sync(0xffffffffu, some, o);
    if ((threadIdx.x & 31) == 0) sm.red[threadIdx.x >> 5] = some;
    __syncthreads();
    some = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) some += sm.red[w];
    const float there = log2f(fmaxf(some, 1.f)) - 0.01f;
    const float can = log2f((float)pieces.vocab / fmaxf(1.f - p, 5e-8f)) + 0.1f;
    const float far = fminf(fmaxf(can, 24.f), kFar);   // (the same for every CTA, and however many there are)
    const int reach = min((int)(fmaxf(can - there, 0.1f) * (float)kPerPower) + 1, kSlices - 1);
    uint32_t light = 0;   // of 1024 tokens at most
    u64 s = 0;
    const int step = (int)(ctas * kThreads);
    Queue queue{sm.queue[threadIdx.x >> 5], 0};
    auto add = [&](float2 x, unsigned which) {
      Weight w[2];
      weights_of(row, sm.table, x, w);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if (!(which >> i & 1)) continue;
        s += mass_of(w[i]);
        const int b = slice_of(w[i]);
        if (b <= reach) atomicAdd(&sm.slice[b], slice_part(w[i]));
      }
    };
    pieces.template scan<2>((int)(rank * kThreads) + (int)(threadIdx.x & ~31u), pieces.count, step, [&](int, const float (&x)[N]) {
      unsigned mine = 0;
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float y = exponent(row, x[e]);
        const bool in = x[e] >= least;
        if (in && y < far) mine |= 1u << e;
        else if (in && y < kFar) light += __float_as_uint(exp2f(-y) + 0x1p-21f) - __float_as_uint(0x1p-21f);  // 2^-44 each
      }
      const unsigned some = __reduce_add_sync(0xffffffffu, __popc(mine));
      if (some == 0) return;
      if (some >= 16 * N) {
#pragma unroll
        for (int e = 0; e < N; e += 2) add(make_float2(x[e], x[e + 1]), mine >> e);
        return;
      }
      queue.put(x, mine);
      while (queue.n >= 64) queue.take(64, add);
    });
    queue.take(queue.n, add);
    return s + light;
  }

  // What top-p keeps of the tokens with x >= least.  The slices' running total is short of the true one by 2^-11 of itself at
  // most, so the cut lies in a slice from the one in which it reaches p of all with 2^-10 on top (sm.lo) to the one in which it
  // does as it is (sm.hi).  Where few tokens lie that far they go into the first CTA's list, and all of their mass to *all: true.
  __device__ bool top_p_list(float p, float least, float own_max, u64* all) {
    u64 s = block_sum(slice_masses(p, least, own_max));
    if (threadIdx.x == 0) sm.sum = s;
    cluster_sync();
    if (rank == 0) {
      u64 t = 0;
      for (unsigned c = 0; c < ctas; ++c) {
        const uint32_t a = peer_addr(&sm.sum, c);
        t += (u64)peer_load(a) | (u64)peer_load(a + 4) << 32;
      }
      *all = t;
      window(share(p, t));
    }
    cluster_sync();
    if (rank != 0 && threadIdx.x == 0) {
      sm.lo = (int)peer_load(peer_addr(&sm.lo, 0));
      sm.hi = (int)peer_load(peer_addr(&sm.hi, 0));
      sm.many = (int)peer_load(peer_addr(&sm.many, 0));
    }
    __syncthreads();
    if (sm.many) return false;
    const float end = slice_begin(sm.hi + 1);
    gather([&](float x, int) { return x >= least && exponent(row, x) < end; });
    return true;
  }
  // By the first CTA: sm.lo, sm.hi, and sm.many, whether more than kCap tokens lie so far: at least a slice's mass over the most
  // that one of it weighs.
  __device__ void window(u64 target) {
    constexpr int per = kSlices / kThreads;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    u64 mass[per], m = 0;
    unsigned count[per], n = 0;
#pragma unroll
    for (int i = 0; i < per; ++i) {
      const int b = threadIdx.x * per + i;
      u64 t = 0;
      for (unsigned c = 0; c < ctas; ++c) t += peer_load(peer_addr(&sm.slice[b], c));
      t <<= slice_shift(b);
      mass[i] = m += t;
      count[i] = n += (unsigned)(t >> max(kUnit - b / kPerPower, 0));
    }
    const u64 own = m;
    const unsigned owned = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const u64 x = __shfl_up_sync(0xffffffffu, m, o);
      const unsigned y = __shfl_up_sync(0xffffffffu, n, o);
      if (lane >= o) {
        m += x;
        n += y;
      }
    }
    if (lane == 31) {
      sm.red64[warp] = m;
      sm.redi[warp] = (int)n;
    }
    if (threadIdx.x == 0) {
      sm.lo = sm.hi = kSlices - 1;
      sm.many = 0;
    }
    __syncthreads();
    m -= own;
    n -= owned;
    for (int w = 0; w < warp; ++w) {
      m += sm.red64[w];
      n += (unsigned)sm.redi[w];
    }
    u64 before = m;
#pragma unroll
    for (int i = 0; i < per; ++i) {
      const u64 with = m + mass[i];
      if (before + (before >> 10) < target && with + (with >> 10) >= target) sm.lo = threadIdx.x * per + i;
      if (before < target && with >= target) {
        sm.hi = threadIdx.x * per + i;
        sm.many = n + count[i] > kCap;
      }
      before = with;
    }
  }

  // The cut where that list would be too long: a pass that sums what lies before slice sm.lo, by runs of 32 pieces, and lists
  // the slices up to sm.hi, in which the first CTA finds it.  (all: as from top_p_list; from: the head of
  // the tokens with x >= least.)  It adds what the list keeps to the
  // runs.  The other CTAs get no head; false where the list is too long even so (a long run of equal weights).
  __device__ bool top_p_runs(float p, float least, const Head& from, u64 all, Head* head) {
    if (threadIdx.x == 0) sm.listed = 0;
    cluster_sync();
    const float begin = slice_begin(sm.lo), end = slice_begin(sm.hi + 1);
    const int runs = (pieces.count + 31) / 32, lane = threadIdx.x & 31;
    Queue queue{sm.queue[threadIdx.x >> 5], 0};
    pieces.template scan<2>((int)(rank * kThreads) + (int)(threadIdx.x & ~31u), pieces.count, (int)(ctas * kThreads), [&](int v, const float (&x)[N]) {
      const int g = v >> 5;
      unsigned above = 0, window = 0;
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float y = exponent(row, x[e]);
        const bool in = x[e] >= least && y < end;
        above |= in && y < begin ? 1u << e : 0u;
        window |= in && y >= begin ? 1u << e : 0u;
      }
      u64 s = 0;
      const unsigned some = __reduce_add_sync(0xffffffffu, __popc(above));
      if (some != 0) {
        auto add = [&](float2 y, unsigned which) {
          Weight w[2];
          weights_of(row, sm.table, y, w);
          s += (which & 1 ? mass_of(w[0]) : 0) + (which & 2 ? mass_of(w[1]) : 0);
        };
        if (some >= 16 * N) {
#pragma unroll
          for (int e = 0; e < N; e += 2) add(make_float2(x[e], x[e + 1]), above >> e);
        } else {
          queue.put(x, above);
          while (queue.n > 0) queue.take(min(queue.n, 64), add);
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
      }
      if (lane == 0) peer_store64(peer_addr(&sm.runs[g], 0), s);
      if (__any_sync(0xffffffffu, window != 0)) {
        int at = reserve(__popc(window));
#pragma unroll
        for (int e = 0; e < N; ++e)
          if (window >> e & 1) put(at++, x[e], v * N - pieces.off + e);
      }
    });
    const int n = join_lists();
    if (n > kCap) return false;
    if (rank == 0) {
      u64 s = 0;
      for (int g = threadIdx.x; g < runs; g += kThreads) s += sm.runs[g];
      s = block_sum(s);
      const Head to = cut_listed(from, n, -1.f, share(p, all) - s, [&](auto f) {
        each_listed(n, [&](float x, int i) { f(x, i, weight(row, sm.table, x)); });
      });
      each_listed(n, [&](float x, int i) {
        if (kept(to, key_of(x), i)) atomicAdd(&sm.runs[(i + pieces.off) / (32 * N)], weight(row, sm.table, x));
      });
      __syncthreads();
      *head = to;
    }
    return true;
  }

  // The CTAs' sums added up.
  __device__ u64 row_sum(u64 s) {
    if (threadIdx.x == 0) sm.sum = s;
    cluster_sync();
    u64 t = 0;
    for (unsigned c = 0; c < ctas; ++c) {
      const uint32_t a = peer_addr(&sm.sum, c);
      t += (u64)peer_load(a) | (u64)peer_load(a + 4) << 32;
    }
    cluster_sync();
    return t;
  }

  // The mass at which top-p's head ends.
  __device__ static u64 share(float p, u64 all) {
    u64 below;
    const bool more = product(fmaxf(p, 0.f), all, &below);
    return max(1ull, min(below + (more ? 1 : 0), all));
  }

  // The token drawn, by the first CTA, whose list of n tokens holds every one that is kept: the first k of them (k < 1: all), of
  // these top-p's head (p >= 1: all).  all: the mass that p is a share of, 0: that of the first k.  Every thread gets it, and the
  // mass of what is kept.
  __device__ int draw_listed(int n, int k, float p, u64 all, float u, u64* mass) {
    if (n <= kRanked) {
      // Every entry's rank, by comparing every two, puts it in its place; the masses before the places say what is kept.
      if (threadIdx.x < n) {
        const Entry e = sm.list[threadIdx.x];
        sm.order[threadIdx.x] = (u64)~key_of(e.x) << 32 | (unsigned)e.i;
      }
      if (threadIdx.x == 0) {
        sm.ranks = 0;
        sm.token = -1;
      }
      __syncthreads();
      const int shift = n <= kRanked / 4 ? 3 : n <= kRanked / 2 ? 2 : 1, ways = 1 << shift;
      const int j = threadIdx.x >> shift, way = threadIdx.x & (ways - 1);
      const u64 own = sm.order[j < n ? j : 0];
      int place = 0;
#pragma unroll 8
      for (int z = way; z < n; z += ways) place += sm.order[z] < own ? 1 : 0;
      for (int o = 1; o < ways; o <<= 1) place += __shfl_xor_sync(0xffffffffu, place, o);
      if (j < n && way == 0) sm.places[place] = sm.list[j];
      __syncthreads();
      const int some = k < 1 ? n : min(n, k);
      const bool there = (int)threadIdx.x < some;
      const Entry e = sm.places[there ? threadIdx.x : 0];
      const u64 w = there ? weight(row, sm.table, e.x) : 0;
      u64 sum;
      const u64 before = block_before(w, &sum);
      if (p < 1.f) {
        const u64 to = share(p, all ? all : sum);
        const bool in = there && before < to;
        if (in) to_rank((u64)(unsigned)e.i, w);
        sum = block_sum(in ? w : 0);
      } else {
        if (there) to_rank((u64)(unsigned)e.i, w);
        __syncthreads();
      }
      const u64 at = draw_at(u, sum);
      rank_each([&](int z, u64 passed, u64 own_w) {
        if (passed <= at && at < passed + own_w) sm.token = (int)sm.order[z];
      });
      __syncthreads();
      *mass = sum;
      return sm.token;
    }
    Head head = {0u, 0x7fffffff};
    if (k > 0 && n > k) head = cut(head, n, false, (u64)k);
    u64 total = weigh_listed(n, head);
    auto weighed = [&](auto f) { each_weighed(n, f); };
    if (p < 1.f) {
      head = cut_listed(head, n, k > 0 ? -1.f : slice_begin(sm.lo), share(p, all ? all : total), weighed);
      total = weigh_listed(n, head);
    }
    *mass = total;
    // A digit of the index, then the tokens that share it.
    const u64 at = draw_at(u, total);
    const int shift = max(0, 24 - __clz(pieces.vocab));
    if (threadIdx.x == 0) sm.ranks = 0;
    digit(n, true, at + 1, [&](float x, int i) { return kept(head, key_of(x), i) ? i >> shift : -1; });
    const int bin = sm.bin;
    const u64 rest = at - sm.before;
    each_weighed(n, [&](float, int i, u64 w) {
      if (i >> shift == bin) to_rank((u64)(unsigned)i, w);
    });
    __syncthreads();
    if (sm.ranks > kRanked) return by_index(n, true, at + 1, [&](float x, int i) { return kept(head, key_of(x), i); });
    rank_each([&](int j, u64 before, u64 w) {
      if (before <= rest && rest < before + w) sm.token = (int)sm.order[j];
    });
    __syncthreads();
    return sm.token;
  }
  // The weights of the list's tokens, 0 where the head does not keep them, and their sum.
  __device__ u64 weigh_listed(int n, const Head& h) {
    u64 s = 0;
    for (int j = threadIdx.x; j < n; j += kThreads) {
      const Entry e = sm.list[j];
      const u64 w = kept(h, key_of(e.x), e.i) ? weight(row, sm.table, e.x) : 0;
      sm.weights[j] = w;
      s += w;
    }
    return block_sum(s);
  }
  __device__ static float key_value(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }

};

template <typename T>
__global__ void __launch_bounds__(kThreads, 2) k_sample(const __grid_constant__ Job job) {
  pdl_wait();
  pdl_launch_dependents();
  constexpr int N = Pieces<T>::N;
  const int r = (int)blockIdx.x / job.cluster, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const unsigned rank = cluster_rank(), ctas = (unsigned)job.cluster;
  cluster_arrive();
  const Pieces<T> pieces(static_cast<const T*>(job.logits) + (size_t)r * job.stride, job.vocab);
  const float temperature = job.temperature ? job.temperature[r] : job.all_temperature;
  const int top_k = job.top_k ? job.top_k[r] : job.all_top_k;
  const float top_p = job.top_p ? job.top_p[r] : job.all_top_p, min_p = job.min_p ? job.min_p[r] : job.all_min_p;
  const bool by_k = top_k > 0 && top_k < job.vocab, greedy = !(temperature > 0.f) || top_k == 1;
  for (int j = tid; j < kBins; j += kThreads) sm.table[j] = kPowers.t[j];
  if (tid == 0) sm.listed = 0;

  if (min_p > 0.f && tid == kThreads - 1)  // (an endless temperature makes every weight one, and times ln 1 it is no number)
    sm.ahead = temperature < INFINITY ? (double)temperature * log(fmin((double)min_p, 1.0)) : -INFINITY;

  // The largest logit, and the piece that has it first.
  float m = -INFINITY;
  int at = 0x7fffffff;
#pragma unroll 4
  for (int v = (int)(rank * kThreads + tid); v < pieces.count; v += (int)(ctas * kThreads)) {
    float x[N];
    pieces.load(v, x);
    float p = x[0];
#pragma unroll
    for (int e = 1; e < N; ++e) p = fmaxf(p, x[e]);
    if (p > m) {
      m = p;
      at = v;
    }
  }
  // Where the first k tokens are asked for: a value that at least k of the threads' largest reach (to 14 bits of its key, a
  // bit of it at a time).
  uint32_t bound = 0;
  if (by_k && !greedy && top_k <= kThreads) {
    const uint32_t key = key_of(m);
    for (int b = 31; b >= 18; --b)
      if (__syncthreads_count(key >= (bound | 1u << b)) >= top_k) bound |= 1u << b;
  }
  const float own_max = m;
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    const float y = __shfl_xor_sync(0xffffffffu, m, o);
    const int z = __shfl_xor_sync(0xffffffffu, at, o);
    if (y > m || (y == m && z < at)) {
      m = y;
      at = z;
    }
  }
  if (lane == 0) {
    sm.red[warp] = m;
    sm.redi[warp] = at;
  }
  __syncthreads();
  cluster_wait();  // every CTA of the row runs
  if (warp == 0) {
    m = lane < kWarps ? sm.red[lane] : -INFINITY;
    at = lane < kWarps ? sm.redi[lane] : 0x7fffffff;
#pragma unroll
    for (int o = 16; o; o >>= 1) {
      const float y = __shfl_xor_sync(0xffffffffu, m, o);
      const int z = __shfl_xor_sync(0xffffffffu, at, o);
      if (y > m || (y == m && z < at)) {
        m = y;
        at = z;
      }
    }
    if ((unsigned)lane < ctas) {
      const uint32_t to = peer_addr(&sm.tops[rank], lane);
      peer_store64(to, (u64)__float_as_uint(m) | (u64)(unsigned)at << 32);
      peer_store32(to + 8, bound);
    }
  }
  cluster_sync();
  m = -INFINITY;
  at = 0x7fffffff;
  for (unsigned c = 0; c < ctas; ++c) {
    const Top& t = sm.tops[c];
    if (t.max > m || (t.max == m && t.arg < at)) {
      m = t.max;
      at = t.arg;
    }
    bound = max(bound, t.bound);
  }
  if (m == -INFINITY || greedy) {   // nothing to draw from, or the likeliest token
    if (rank == 0 && tid == 0) {
      int token = -1;
      if (m > -INFINITY) {
        float x[N];
        pieces.load(at, x);
        for (int e = N - 1; e >= 0; --e)
          if (x[e] == m) token = at * N - pieces.off + e;
      }
      job.token[r] = token;
      if (job.logprob) job.logprob[r] = token < 0 ? -INFINITY : 0.f;
    }
    return;
  }
  // log2(e) / T in two terms: the quotient, and its remainder's.
  Row row;
  row.max = m;
  row.ch = fminf(1.44269502f / temperature, 3e38f);   // (0 times it stays 0)
  row.cl = row.ch < 1e30f && temperature < 1e30f ? (__fmaf_rn(-row.ch, temperature, 1.44269502f) + 1.92596299e-8f) / temperature : 0.f;
  RowCtas<T> ctx{pieces, row, rank, ctas};
  float least = -INFINITY;  // min-p's: w >= min_p where x >= max + T ln(min_p), the least fp32 value that is
  if (min_p > 0.f) {
    if (tid == 0) {
      const double from = (double)m + sm.ahead;
      least = (float)from;
      if ((double)least < from) least = nextafterf(least, INFINITY);
      sm.least = least;
    }
    __syncthreads();
    least = sm.least;
  }
  // Where few tokens can be kept the first CTA decides in a list of them.
  const Head from = least > -INFINITY ? Head{key_of(least) - 1, -1} : Head{0u, 0x7fffffff};  // x >= least: a key above its own less one
  Head head = from;
  bool summed = false;  // the kept tokens' mass lies in the first CTA's runs
  if (m < INFINITY) {
    u64 all = 0;
    bool listed = true;
    if (by_k && top_k <= kThreads) {
      const float from = fmaxf(least, ctx.key_value(bound));  // (a NaN where the bound is below every number)
      ctx.gather([&](float x, int) { return x >= from; });
    } else if (!by_k && top_p < 1.f) {
      listed = ctx.top_p_list(top_p, least, own_max, &all);
    } else if (!by_k && min_p > 0.f) {
      ctx.gather([&](float x, int) { return x >= least; });
    } else {
      listed = false;
    }
    if (listed) {
      const int n = ctx.join_lists();
      if (n <= kCap) {
        if (rank == 0) {
          u64 total;
          const int token = ctx.draw_listed(n, by_k ? top_k : 0, top_p, all, job.u[r], &total);
          if (tid == 0) job.token[r] = token;
          if (job.logprob)
            ctx.each_listed(n, [&](float x, int i) {
              if (i == token) job.logprob[r] = log_share(x, m, temperature, total);
            });
        }
        return;
      }
    }
    if (!by_k && top_p < 1.f) summed = ctx.top_p_runs(top_p, least, from, all, &head);
  }
  const int runs = (pieces.count + 31) / 32;
  if (!summed) {
    head = by_k ? ctx.cut({0u, 0x7fffffff}, -1, false, (u64)top_k) : from;
    if (least > -INFINITY && from.k >= head.k) head = from;  // (of one key, min-p's: it keeps none of that key's tokens)
    if (top_p < 1.f) {
      u64 s = 0;
      ctx.each([&](float x, int i) { s += kept(head, key_of(x), i) ? weight(row, sm.table, x) : 0; });
      head = ctx.cut(head, -1, true, ctx.share(top_p, ctx.row_sum(ctx.block_sum(s))));
    }
    // The kept tokens' mass by runs of 32 pieces, to the first CTA.
    pieces.template scan<2>(((int)rank * kWarps + warp) * 32, pieces.count, (int)(ctas * kThreads), [&](int v, const float (&x)[N]) {
      u64 s = 0;
#pragma unroll
      for (int e = 0; e < N; e += 2) {
        Weight w[2];
        weights_of(row, sm.table, make_float2(x[e], x[e + 1]), w);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const bool in = kept(head, key_of(x[e + i]), v * N - pieces.off + e + i);
          s += in && x[e + i] == m ? 1ull << kUnit : in && exponent(row, x[e + i]) < kFar ? mass_of(w[i]) : 0;
        }
      }
#pragma unroll
      for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
      if (lane == 0) peer_store64(peer_addr(&sm.runs[v >> 5], 0), s);
    });
    cluster_sync();
  }
  if (rank != 0 || warp != 0) return;
  // Its first warp finds the run, then the token.
  const int per = (runs + 31) / 32;
  u64 own = 0;
  for (int g = lane * per; g < min(runs, (lane + 1) * per); ++g) own += sm.runs[g];
  u64 inc = own;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const u64 y = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += y;
  }
  const u64 total = __shfl_sync(0xffffffffu, inc, 31);
  const u64 target = draw_at(job.u[r], total);
  const int l = __ffs(__ballot_sync(0xffffffffu, inc > target)) - 1;
  int run = l * per;
  u64 before = __shfl_sync(0xffffffffu, inc - own, l);
  while (before + sm.runs[run] <= target) before += sm.runs[run++];
  const int v = run * 32 + lane;
  float x[N];
  pieces.load(v, x);
  u64 w[N];
  own = 0;
#pragma unroll
  for (int e = 0; e < N; ++e) {
    w[e] = kept(head, key_of(x[e]), v * N - pieces.off + e) ? weight(row, sm.table, x[e]) : 0;
    own += w[e];
  }
  inc = own;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const u64 y = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += y;
  }
  inc += before;
  if (lane != __ffs(__ballot_sync(0xffffffffu, inc > target)) - 1) return;
  u64 sum = inc - own;
  bool found = false;
#pragma unroll
  for (int e = 0; e < N; ++e) {
    sum += w[e];
    if (!found && sum > target) {
      found = true;
      job.token[r] = v * N - pieces.off + e;
      if (job.logprob) job.logprob[r] = log_share(x[e], m, temperature, total);
    }
  }
}

#undef sm

}  // namespace
}  // namespace gb

using namespace gb;

extern "C" gb_status gb_sample(const gb_sample_args* a, gb_stream_t stream) {
  if (!a || a->rows < 0 || a->vocab < 1 || (a->dtype != GB_F32 && a->dtype != GB_BF16)) return GB_ERR_INVALID;
  if (a->rows == 0) return GB_OK;
  const int es = a->dtype == GB_F32 ? 4 : 2;
  if (!a->logits || !a->u || !a->token || a->row_stride < a->vocab || ((uintptr_t)a->logits % es) != 0 ||
      (((uintptr_t)a->u | (uintptr_t)a->token | (uintptr_t)a->logprob | (uintptr_t)a->temperature | (uintptr_t)a->top_k |
        (uintptr_t)a->top_p | (uintptr_t)a->min_p) & 3) != 0)
    return GB_ERR_INVALID;
  if (a->vocab > kMaxVocab) return GB_ERR_UNSUPPORTED;
  int device = 0, sms = 0;
  if (cudaGetDevice(&device) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device) != cudaSuccess)
    return GB_ERR_CUDA;
  // CTAs a row: as many as keep the GPU's SMs busy, some also of many rows, whose times differ sixfold: 512 rows of 128000 take
  // 189 us with one, 142 with two.  At least a few pieces for each thread.
  constexpr int kLeast = 2;
  int cluster = 1;
  while (cluster < kMaxCluster && (cluster < kLeast || (long long)a->rows * cluster * 2 <= 2ll * sms) && a->vocab / (cluster * 2) >= kThreads * 4)
    cluster *= 2;
  if ((long long)a->rows * cluster > 0x7fffffffll) return GB_ERR_TOO_LARGE;
  Job job = {a->logits, a->row_stride, a->rows, a->vocab, cluster, a->u, a->temperature, a->top_p, a->min_p, a->top_k,
             a->all_temperature, a->all_top_p, a->all_min_p, a->all_top_k, a->token, a->logprob};
  void (*kernel)(const Job) = a->dtype == GB_F32 ? k_sample<float> : k_sample<__nv_bfloat16>;
  if (set_max_dynamic_smem(reinterpret_cast<const void*>(kernel), (int)sizeof(Smem)) != cudaSuccess)
    return GB_ERR_CUDA;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(a->rows * cluster));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = sizeof(Smem);
  cfg.stream = reinterpret_cast<cudaStream_t>(stream);
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)cluster;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  if (cudaLaunchKernelEx(&cfg, kernel, job) != cudaSuccess) {
    cudaGetLastError();
    return GB_ERR_CUDA;
  }
  return GB_OK;
}
