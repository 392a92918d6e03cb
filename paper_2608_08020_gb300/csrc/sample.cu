// The next token of each row of logits, from a given random number.
//
// With max the row's largest logit and w_i = exp((x_i - max) / T), the tokens are taken in descending order of (x, -index):
//   top-k   keeps the first k of them,
//   min-p   of these the ones with w_i >= min_p,
//   top-p   of these the shortest head whose mass reaches top_p of theirs,
// so what is kept is always a head of that order: the tokens with x > K, and those with x = K up to some index.  The token is
// the first, by index, at which the kept tokens' mass passes u times its total.
//
// A token is compared against sums over the whole vocabulary, so masses are whole numbers: w in units of 2^-44, right to about
// 2^-33 of itself, summed in 64 bits.  Sums are then the same in any order, and no draw depends on how the row was split.
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
constexpr int kCap = 4096;              // tokens of a list
constexpr int kSlices = 1024;           // of the weights' exponents, 22 to a power of two
constexpr float kPerPower = 22.f;
static_assert(kFar * kPerPower < kSlices, "every weight has a slice");
typedef unsigned long long u64;

// 2^(-j/256) in units of 2^-44: the power series of exp in 64 bits, as the compiler evaluates it.
struct PowerTable {
  u64 t[kBins];
  constexpr PowerTable() : t() {
    for (int j = 0; j < kBins; ++j) {
      const double x = -0.69314718055994530942 * j / kBins;
      double term = 1, sum = 0;
      for (int n = 1; n < 30; ++n) {
        sum += term;
        term *= x / n;
      }
      t[j] = (u64)(sum * (double)(1ull << kUnit) + 0.5);
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
__device__ __forceinline__ uint32_t peer_load(uint32_t a) {
  uint32_t x;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(x) : "r"(a) : "memory");
  return x;
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

// exp((x - max) / T) in units of 2^-44.  y = (max - x) log2(e) / T to 2^-40 of itself or better; 2^-y is the table's
// 2^(-j/256) times 1 + p, with p the third-order series of 2^-r, |r| <= 2^-9.
__device__ __forceinline__ u64 weight(const Row& row, const u64* table, float x) {
  if (!(x > -INFINITY)) return 0;
  if (x == row.max) return 1ull << kUnit;
  const float d = __fsub_rn(row.max, x), b = __fsub_rn(d, row.max);
  const float e = __fadd_rn(__fsub_rn(row.max, __fsub_rn(d, b)), __fsub_rn(-x, b));
  const float yh = __fmul_rn(d, row.ch);
  if (!(yh < kFar)) return 0;
  const float yl = __fadd_rn(__fmaf_rn(d, row.ch, -yh), __fmaf_rn(d, row.cl, __fmul_rn(e, row.ch)));
  const float z = __fadd_rn(yh, 49152.f);                  // rounds to multiples of 2^-8
  const int j = __float_as_int(z) - __float_as_int(49152.f);
  const float r = __fadd_rn(__fsub_rn(yh, __fsub_rn(z, 49152.f)), yl);
  constexpr float kLn2 = 0.69314718055994530942f;
  const float p = r * __fmaf_rn(r, __fmaf_rn(r, -kLn2 * kLn2 * kLn2 / 6, kLn2 * kLn2 / 2), -kLn2);
  const u64 t = table[j & 255];
  const u64 w = t + (u64)(((long long)(int)(t >> 14) * __float2int_rn(p * 0x1p40f)) >> 26);
  const int n = j >> 8;
  return (w + ((1ull << n) >> 1)) >> n;
}

// The slice of a weight: y in steps of 1 / 22 (in a lower slice the weight is larger).
__device__ __forceinline__ int slice_of(const Row& row, float x) {
  if (x == row.max) return 0;
  const float y = __fmul_rn(__fsub_rn(row.max, x), row.ch);
  return y < kFar ? (int)(y * kPerPower) : kSlices - 1;
}
// Masses are summed in units of 2^shift by slice: 12 bits of a weight's 45.
__device__ __forceinline__ int slice_shift(int b) { return max(0, 32 - b / (int)kPerPower); }

__device__ __forceinline__ float value(const float* p) { return *p; }
__device__ __forceinline__ float value(const __nv_bfloat16* p) { return __bfloat162float(*p); }
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
  __device__ __forceinline__ void load(int v, float (&f)[N]) const {
    const int i0 = v * N - off;
    if (v < count && i0 >= 0 && i0 + N <= vocab) {
      values(__ldg(reinterpret_cast<const uint4*>(x + i0)), f);
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e) f[e] = v < count && i0 + e >= 0 && i0 + e < vocab ? value(x + i0 + e) : -INFINITY;
    }
  }
};

// ---- the row's CTAs ----------------------------------------------------------------------------------

struct Entry {
  float x;
  int i;
};

struct Smem {
  u64 table[kBins];
  Entry list[kCap];                      // the first CTA's holds all
  uint32_t slice[kSlices];               // masses by slice, see top_p_cut
  u64 slice_total[kSlices];
  int listed, window[2];
  uint32_t head_k;
  int head_i;
  uint32_t hist[1 + kDigits][kBins];     // counts, then the masses' digits
  u64 total[kBins];
  float red[kWarps];
  int redi[kWarps];
  u64 red64[kWarps];
  u64 before;                            // of the bin chosen
  int bin;
  float max;                             // this CTA's, read by its peers
  int arg;
  u64 sum;
};

// What is kept: the tokens with key > k, and those with key = k and index <= i.
struct Head {
  uint32_t k;
  int i;
};
__device__ __forceinline__ bool kept(const Head& h, uint32_t key, int i) { return key > h.k || (key == h.k && i <= h.i); }

template <typename T>
struct RowCtas {
  Smem& sm;
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
    for (int s = 24; s >= 0; s -= 8) {
      digit(n, weigh, target, [&](float x, int i) {
        const uint32_t key = key_of(x), rel = top - key;
        return kept(h, key, i) && (s == 24 || rel >> (s + 8) == at >> (s + 8)) ? (int)(rel >> s & 255u) : -1;
      });
      at |= (uint32_t)sm.bin << s;
      target -= sm.before;
      __syncthreads();
    }
    // The key is chosen; of its tokens, all of one weight, the first ones by index.
    Head to = {top - at, h.k == top - at ? h.i : 0x7fffffff};
    u64 most = target;
    if (weigh) {
      const u64 w = weight(row, sm.table, key_value(to.k));
      most = w ? (target + w - 1) / w : target;
    }
    to.i = min(to.i, by_index(n, false, most, [&](float x, int i) { return key_of(x) == to.k && i <= to.i; }));
    return to;
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

  // Puts the tokens that in(x, i) says into this CTA's list; then the first CTA's holds all of the row's (in no order).
  // Returns how many there are: lists of more than kCap hold no more, and are none.
  template <class In>
  __device__ int gather(In in) {
    if (threadIdx.x == 0) sm.listed = 0;
    __syncthreads();
    const int step = (int)(ctas * kThreads);
    for (int v0 = (int)(rank * kThreads) + (int)(threadIdx.x & ~31u); v0 < pieces.count; v0 += step) {
      const int v = v0 + (int)(threadIdx.x & 31);
      float x[N];
      pieces.load(v, x);
      unsigned mine = 0;
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const int i = v * N - pieces.off + e;
        if (v < pieces.count && i >= 0 && i < pieces.vocab && in(x[e], i)) mine |= 1u << e;
      }
      if (!__any_sync(0xffffffffu, mine != 0)) continue;
      if (mine) {
        int at = atomicAdd(&sm.listed, __popc(mine));
#pragma unroll
        for (int e = 0; e < N; ++e)
          if (mine >> e & 1) {
            if (at < kCap) sm.list[at] = {x[e], v * N - pieces.off + e};
            ++at;
          }
      }
    }
    cluster_sync();
    int n = 0, before = 0;
    for (unsigned c = 0; c < ctas; ++c) {
      const int own = (int)peer_load(peer_addr(&sm.listed, c));
      if (c < rank) before += own;
      n += own;
    }
    if (n <= kCap && rank > 0) {
      const int own = sm.listed;
      for (int j = threadIdx.x; j < own; j += kThreads)
        peer_store64(peer_addr(&sm.list[before + j], 0), (u64)__float_as_uint(sm.list[j].x) | (u64)(unsigned)sm.list[j].i << 32);
    }
    cluster_sync();
    return n;
  }

  // The head that the first CTA has found, to all.
  __device__ Head share(const Head& h) {
    if (rank == 0 && threadIdx.x == 0) {
      sm.head_k = h.k;
      sm.head_i = h.i;
    }
    cluster_sync();
    const Head to = {peer_load(peer_addr(&sm.head_k, 0)), (int)peer_load(peer_addr(&sm.head_i, 0))};
    cluster_sync();
    return to;
  }

  // The k-th largest of the threads' largest tokens, of k <= kThreads: at least k of the row's tokens are as large.
  __device__ uint32_t bound_of_top(int k, uint32_t key) {
    uint32_t at = 0;  // the largest value that at least k keys reach
    for (int b = 31; b >= 0; --b)
      if (__syncthreads_count(key >= (at | 1u << b)) >= k) at |= 1u << b;
    if (threadIdx.x == 0) sm.head_k = at;
    cluster_sync();
    for (unsigned c = 0; c < ctas; ++c) at = max(at, peer_load(peer_addr(&sm.head_k, c)));
    cluster_sync();
    return at;
  }

  // Cut the head where its mass reaches the share p of its total.  One pass sums the weights exactly, and by slices of their
  // exponent to 12 bits each: the running total of the slices is then known from below, and from above within 2^-10 of itself,
  // which leaves a slice or two in which the cut must lie.  A second pass sums what lies before them exactly and lists their
  // tokens, among which the cut is found.  Tokens so light that all of them together could not be the share 1 - p that goes
  // need no slice.
  __device__ Head top_p_cut(const Head& h, float p) {
    for (int b = threadIdx.x; b < kSlices; b += kThreads) sm.slice[b] = 0;
    __syncthreads();
    const float far = log2f((float)pieces.vocab / fmaxf(1.f - p, 5e-8f)) + 0.01f;
    const int last = min(kSlices - 1, (int)(far * kPerPower) + 1);
    u64 s = 0;
    each([&](float x, int i) {
      if (!kept(h, key_of(x), i)) return;
      const u64 w = weight(row, sm.table, x);
      s += w;
      const int b = slice_of(row, x);
      if (b <= last) atomicAdd(&sm.slice[b], (uint32_t)(w >> slice_shift(b)));
    });
    s = block_sum(s);
    if (threadIdx.x == 0) sm.sum = s;
    cluster_sync();
    u64 all = 0;
    for (unsigned c = 0; c < ctas; ++c) {
      const uint32_t a = peer_addr(&sm.sum, c);
      all += (u64)peer_load(a) | (u64)peer_load(a + 4) << 32;
    }
    for (int b = threadIdx.x; b < kSlices; b += kThreads) {
      u64 t = 0;
      for (unsigned c = 0; c < ctas; ++c) t += peer_load(peer_addr(&sm.slice[b], c));
      sm.slice_total[b] = t << slice_shift(b);
    }
    cluster_sync();
    const u64 target = max(1ull, min((u64)ceil(fmax((double)p, 0.0) * (double)all), all));
    if (threadIdx.x < 32) {
      constexpr int per = kSlices / 32;
      const int lane = threadIdx.x;
      u64 own = 0;
      for (int b = 0; b < per; ++b) own += sm.slice_total[lane * per + b];
      u64 inc = own;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const u64 y = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += y;
      }
      // First slice whose running total, from above, or from below, reaches the target.
      u64 before = inc - own;
      int lo = kSlices, hi = kSlices;
      for (int b = lane * per; b < (lane + 1) * per; ++b) {
        before += sm.slice_total[b];
        if (lo == kSlices && before + (before >> 10) >= target) lo = b;
        if (hi == kSlices && before >= target) hi = b;
      }
      lo = (int)__reduce_min_sync(0xffffffffu, (unsigned)lo);
      hi = (int)__reduce_min_sync(0xffffffffu, (unsigned)hi);
      if (lane == 0) {
        sm.window[0] = min(lo, last);
        sm.window[1] = min(hi, last);
      }
    }
    __syncthreads();
    const int lo = sm.window[0], hi = sm.window[1];
    u64 above = 0;
    const int n = gather([&](float x, int i) {
      if (!kept(h, key_of(x), i)) return false;
      const int b = slice_of(row, x);
      if (b < lo) above += weight(row, sm.table, x);
      return b >= lo && b <= hi;
    });
    above = block_sum(above);
    if (threadIdx.x == 0) sm.sum = above;
    cluster_sync();
    above = 0;
    for (unsigned c = 0; c < ctas; ++c) {
      const uint32_t a = peer_addr(&sm.sum, c);
      above += (u64)peer_load(a) | (u64)peer_load(a + 4) << 32;
    }
    cluster_sync();
    if (n > kCap || above >= target) return cut(h, -1, true, target);   // (a run of equal weights)
    Head to = h;
    if (rank == 0) to = cut(h, n, true, target - above);
    return share(to);
  }
  __device__ static float key_value(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }

  // The sum of f over the row's tokens, in every thread.
  template <class F>
  __device__ u64 sum(F f) {
    u64 s = 0;
    each([&](float x, int i) { s += f(x, i); });
#pragma unroll
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if ((threadIdx.x & 31) == 0) sm.red64[threadIdx.x >> 5] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
      u64 t = 0;
      for (int w = 0; w < kWarps; ++w) t += sm.red64[w];
      sm.sum = t;
    }
    cluster_sync();
    u64 t = 0;
    for (unsigned c = 0; c < ctas; ++c) {
      const uint32_t a = peer_addr(&sm.sum, c);
      t += (u64)peer_load(a) | (u64)peer_load(a + 4) << 32;
    }
    cluster_sync();
    return t;
  }
};

// The token drawn is the first at which the kept mass passes this.
__device__ __forceinline__ u64 draw_at(float u, u64 total) {
  const u64 t = u > 0.f ? (u64)fmin((double)u * (double)total, 9e18) : 0;
  return min(t, total - 1);
}
// ln(w / total)
__device__ __forceinline__ float share_of(float x, float m, float temperature, u64 total) {
  const double y = x == m ? 0.0 : ((double)x - (double)m) / (double)temperature;
  return (float)(y - log((double)total * 0x1p-44));
}

template <typename T>
__global__ void __launch_bounds__(kThreads) k_sample(const __grid_constant__ Job job) {
  pdl_wait();
  pdl_launch_dependents();
  extern __shared__ __align__(16) unsigned char raw[];
  Smem& sm = *reinterpret_cast<Smem*>(raw);
  u64* chunk = reinterpret_cast<u64*>(raw + sizeof(Smem));  // the first CTA's: mass of each run of 32 pieces
  constexpr int N = Pieces<T>::N;
  const int r = (int)blockIdx.x / job.cluster, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const unsigned rank = cluster_rank(), ctas = (unsigned)job.cluster;
  const Pieces<T> pieces(static_cast<const T*>(job.logits) + (size_t)r * job.stride, job.vocab);
  for (int j = tid; j < kBins; j += kThreads) sm.table[j] = kPowers.t[j];

  // The largest logit, and the piece that has it first.
  float m = -INFINITY;
  int at = 0x7fffffff;
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
  const uint32_t own_key = key_of(m);
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
  if (tid == 0) {
    for (int w = 1; w < kWarps; ++w)
      if (sm.red[w] > m || (sm.red[w] == m && sm.redi[w] < at)) {
        m = sm.red[w];
        at = sm.redi[w];
      }
    sm.max = m;
    sm.arg = at;
  }
  cluster_sync();
  m = -INFINITY;
  at = 0x7fffffff;
  for (unsigned c = 0; c < ctas; ++c) {
    const float y = __uint_as_float(peer_load(peer_addr(&sm.max, c)));
    const int z = (int)peer_load(peer_addr(&sm.arg, c));
    if (y > m || (y == m && z < at)) {
      m = y;
      at = z;
    }
  }
  cluster_sync();
  float temperature = job.temperature ? job.temperature[r] : job.all_temperature;
  const int top_k = job.top_k ? job.top_k[r] : job.all_top_k;
  const float top_p = job.top_p ? job.top_p[r] : job.all_top_p, min_p = job.min_p ? job.min_p[r] : job.all_min_p;
  if (m == -INFINITY || !(temperature > 0.f) || top_k == 1) {   // nothing to draw from, or the likeliest token
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
  const double c = 1.4426950408889634074 / (double)temperature;
  Row row;
  row.max = m;
  row.ch = (float)c;
  row.cl = (float)(c - (double)row.ch);
  RowCtas<T> ctx{sm, pieces, row, rank, ctas};
  Head head = {0u, 0x7fffffff};
  Head least = head;  // min-p's
  if (min_p > 0.f) {
    // w >= min_p where x >= max + T ln(min_p): the least fp32 value that is.
    const double from = (double)m + (double)temperature * log(fmin((double)min_p, 1.0));
    float f = (float)from;
    if ((double)f < from) f = nextafterf(f, INFINITY);
    least.k = key_of(f);
    if (least.k > 0) {  // x >= f: key > key(f) - 1
      --least.k;
      least.i = -1;
    }
  }
  const bool by_k = top_k > 0 && top_k < job.vocab;
  if (by_k && top_k <= kThreads) {
    // The few tokens that can be among the first k, in one list.
    const uint32_t bound = ctx.bound_of_top(top_k, own_key);
    const int n = ctx.gather([&](float x, int i) { return key_of(x) >= bound && kept(least, key_of(x), i); });
    if (n <= kCap) {
      if (rank != 0) return;
      if (n > top_k) head = ctx.cut(head, n, false, (u64)top_k);
      u64 total = 0;
      ctx.each_listed(n, [&](float x, int i) { total += kept(head, key_of(x), i) ? weight(row, sm.table, x) : 0; });
      total = ctx.block_sum(total);
      if (top_p < 1.f) {
        const u64 target = (u64)ceil(fmax((double)top_p, 0.0) * (double)total);
        head = ctx.cut(head, n, true, max(1ull, min(target, total)));
        total = 0;
        ctx.each_listed(n, [&](float x, int i) { total += kept(head, key_of(x), i) ? weight(row, sm.table, x) : 0; });
        total = ctx.block_sum(total);
      }
      const int token = ctx.by_index(n, true, draw_at(job.u[r], total) + 1, [&](float x, int i) { return kept(head, key_of(x), i); });
      if (tid == 0) job.token[r] = token;
      if (job.logprob)
        ctx.each_listed(n, [&](float x, int i) {
          if (i == token) job.logprob[r] = share_of(x, m, temperature, total);
        });
      return;
    }
  }
  if (by_k) head = ctx.cut(head, -1, false, (u64)top_k);
  if (least.k > head.k || (least.k == head.k && least.i < head.i)) head = least;
  if (top_p < 1.f) head = ctx.top_p_cut(head, top_p);
  // The kept tokens' mass by runs of 32 pieces, to the first CTA.
  const int runs = (pieces.count + 31) / 32;
  for (int g = (int)rank * kWarps + warp; g < runs; g += (int)ctas * kWarps) {
    const int v = g * 32 + lane;
    float x[N];
    pieces.load(v, x);
    u64 s = 0;
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (kept(head, key_of(x[e]), v * N - pieces.off + e)) s += weight(row, sm.table, x[e]);
#pragma unroll
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (lane == 0) peer_store64(peer_addr(&chunk[g], 0), s);
  }
  cluster_sync();
  if (rank != 0 || warp != 0) return;
  // Its first warp finds the run, then the token.
  const int per = (runs + 31) / 32;
  u64 own = 0;
  for (int g = lane * per; g < min(runs, (lane + 1) * per); ++g) own += chunk[g];
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
  while (before + chunk[run] <= target) before += chunk[run++];
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
      if (job.logprob) job.logprob[r] = share_of(x[e], m, temperature, total);
    }
  }
}

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
  // CTAs a row: as many as keep the GPU's SMs busy, and at least a few pieces for each thread.
  int cluster = 1;
  while (cluster < kMaxCluster && (long long)a->rows * cluster * 2 <= 2ll * sms && a->vocab / (cluster * 2) >= kThreads * 4) cluster *= 2;
  if ((long long)a->rows * cluster > 0x7fffffffll) return GB_ERR_TOO_LARGE;
  Job job = {a->logits, a->row_stride, a->rows, a->vocab, cluster, a->u, a->temperature, a->top_p, a->min_p, a->top_k,
             a->all_temperature, a->all_top_p, a->all_min_p, a->all_top_k, a->token, a->logprob};
  const int n = 16 / es, runs = ((a->vocab + n - 1 + n - 1) / n + 31) / 32;
  const size_t smem = sizeof(Smem) + (size_t)runs * sizeof(u64);
  void (*kernel)(const Job) = a->dtype == GB_F32 ? k_sample<float> : k_sample<__nv_bfloat16>;
  if (set_max_dynamic_smem(reinterpret_cast<const void*>(kernel), (int)(sizeof(Smem) + (kMaxVocab / 128 + 2) * sizeof(u64))) != cudaSuccess)
    return GB_ERR_CUDA;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(a->rows * cluster));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
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
