// Causal attention over whole prompts, packed one after the other (gb_prompt_attention).
//
//   out[i][h] = sum_{j <= i} p_j v[j][h / G],  p = softmax_j(scale q[i][h] . k[j][h / G])
// for the tokens i, j of one sequence.  The rows of one KV head are (token, query head of the group), token
// by token, so a tile of 128 rows has 128 / G tokens and all G heads that read the same K and V.
//
// Bound by the tensor cores from a few hundred tokens on (2 D Hq n^2 flops against 4 D (Hq + Hkv) n bytes).
// A planner CTA lists the units (sequence, run of tokens), longest first; a CTA per SM takes its (unit, KV head) pairs
// in turn.  One prompt's units need no list.  bf16: flash.cuh; fp32: tile.cuh.
// Measured (32 query heads, 8 KV heads, bf16): 8192 tokens 379 us, 1.45 PFLOP/s of the 1.88 of a large library product; 16384
// tokens of 16 and 2 heads 716 us, 1.54 PFLOP/s; 24 packed prompts of up to 2048 tokens 73 us; 333 tokens 11 us, of which the
// host's call is 9 to 10.
#include <algorithm>
#include <mutex>

#include "flash.cuh"
#include "tile.cuh"
#include "worklist.cuh"

namespace gb {
namespace {

// Workspace: control words, the units, then a word per sequence.
enum PromptCtl : int { kPrStatus = 0, kPrUnits = 1, kPrWords = 64 };

struct PromptUnit {
  int start, len;   // the sequence's first row and length
  int t0, ntok;     // its tokens [t0, t0 + ntok)
};

// `tokens` of a unit, or where that makes `few` units at most `small_tokens`.  lens: a word per sequence, used only when some
// bounds are out of order or range: then a sequence counts if its own bounds are in range, in order and not before an
// earlier one that is in range, so no row belongs to two and the list has room for all units.
__global__ void __launch_bounds__(kListThreads) k_prompt_plan(const int* cu, int num_seqs, int num_tokens, int tokens,
                                                              int small_tokens, int few, int max_units, int* ctl, int* lens) {
  pdl_wait();
  pdl_launch_dependents();
  __shared__ ListSmem sm;
  PromptUnit* units = reinterpret_cast<PromptUnit*>(ctl + kPrWords);
  const int tid = threadIdx.x, lane = tid & 31;
  auto in_range = [&](int x) { return x >= 0 && x <= num_tokens; };
  bool bad = false;
  for (int s = tid; s < num_seqs; s += kListThreads) bad |= !in_range(cu[s]) || !in_range(cu[s + 1]) || cu[s] > cu[s + 1];
  bad = __syncthreads_or(bad);
  if (tid == 0) ctl[kPrStatus] = bad ? GB_ERR_INVALID : GB_OK;
  for (int base = 0, top = 0; bad && base < num_seqs; base += kListThreads) {  // top: the highest bound so far
    const int s = base + tid, x = s < num_seqs && in_range(cu[s]) ? cu[s] : 0;
    int high = max(x, top);  // of the bounds up to this one
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, high, o);
      if (lane >= o) high = max(high, y);
    }
    if (lane == 31) sm.tmp[tid >> 5] = high;
    __syncthreads();
    for (int w = 0; w < tid >> 5; ++w) high = max(high, sm.tmp[w]);
    if (s < num_seqs) lens[s] = in_range(cu[s]) && in_range(cu[s + 1]) && cu[s] >= high ? max(cu[s + 1] - cu[s], 0) : 0;
    __syncthreads();
    if (tid == kListThreads - 1) sm.tmp[0] = high;
    __syncthreads();
    top = sm.tmp[0];
    __syncthreads();
  }
  auto length = [&](int s) { return bad ? lens[s] : cu[s + 1] - cu[s]; };
  int mine = 0, all;
  for (int s = tid; s < num_seqs; s += kListThreads) mine += (length(s) + tokens - 1) / tokens;
  block_exclusive_scan(mine, sm.tmp, &all);
  const int per = all <= few ? small_tokens : tokens;
  const int n = emit_sorted(
      sm, num_seqs, [&](int s) { return (length(s) + per - 1) / per; },
      [&](int s, int i) { return (min((i + 1) * per, length(s)) + flash::kTok - 1) / flash::kTok; },
      [&](int s, int i, int at) {
        if (at >= max_units) return;
        const int len = length(s);
        units[at] = {cu[s], len, i * per, min(per, len - i * per)};
      });
  if (tid == 0) ctl[kPrUnits] = min(n, max_units);
}

struct PromptView {
  int* ctl;
  const int* cu;
  int most_units;                           // entries of the list
  int num_seqs, tokens, small_tokens, few;  // tokens of a unit, where there are at most `few` of them small_tokens
  int Hkv, G, num_tokens;
  float qscale;
  long long q_stride, k_stride, v_stride, out_stride;  // elements between tokens
};

// The units.  One prompt's are known from its bounds, longest first, without the planner's launch (a call of 333 tokens took
// 5 us more with it).
struct PromptUnits {
  int start, len, per, count;
  __device__ __forceinline__ explicit PromptUnits(const PromptView& p) {
    if (p.num_seqs != 1) {
      count = p.ctl[kPrUnits];
      return;
    }
    start = p.cu[0];
    const int end = p.cu[1];
    len = start >= 0 && start <= end && end <= p.num_tokens ? end - start : 0;
    per = (len + p.tokens - 1) / p.tokens <= p.few ? p.small_tokens : p.tokens;
    count = (len + per - 1) / per;
  }
  // The planner's part of the status, where there is none: by one thread, once.
  static __device__ __forceinline__ void status(const PromptView& p) {
    if (p.num_seqs != 1) return;
    const int start = p.cu[0], end = p.cu[1];
    p.ctl[kPrStatus] = start >= 0 && start <= end && end <= p.num_tokens ? GB_OK : GB_ERR_INVALID;
  }
  __device__ __forceinline__ PromptUnit operator()(const PromptView& p, int i) const {
    if (p.num_seqs != 1) return reinterpret_cast<const PromptUnit*>(p.ctl + kPrWords)[i];
    const int t0 = (count - 1 - i) * per;
    return {start, len, t0, min(per, len - t0)};
  }
};

struct PromptJob : PromptView {
  CUtensorMap tq, tk, tv;
  const __nv_bfloat16 *q, *k, *v;
  __nv_bfloat16* o;

  static constexpr uint64_t kWaitNs = kWaitLimitNs;
  static constexpr bool kEarlyQ = false;
  static constexpr int kLongPair = 0;  // none: K and V come from the L2 in time (24 packed prompts 78.2 us, with 4 tiles 79.4)
  static constexpr int kQArrivals = 1;
  // Tiles land as [half of D][128 tokens][64 dims].
  static constexpr int kKHalf = 16384, kKSbo = 1024, kVLbo = 16384, kVSbo = 1024, kVStep = 2048;
  static __device__ __forceinline__ int v_row(int row, int half) { return half * 16384 + row * 128; }

  struct Row {
    int tok;        // row r's token in its sequence
    int head;       // its query head
    int first;      // the warp's first token
    bool valid;
  };

  __device__ __forceinline__ void error(int code) const { atomicCAS(&ctl[kPrStatus], GB_OK, code); }
  __device__ __forceinline__ void begun() const {
    if (blockIdx.x == 0 && threadIdx.x % 32 == 0) PromptUnits::status(*this);
  }
  using Units = PromptUnits;  // what the warp that takes the units holds
  __device__ __forceinline__ int total(const Units& all) const { return all.count * Hkv; }
  __device__ __forceinline__ int capacity() const { return most_units * Hkv; }
  __device__ __forceinline__ bool joins(const Units&) const { return true; }  // (the list is the same each time)
  __device__ __forceinline__ void unit(const Units& all, int id, flash::Unit& x) const {
    const PromptUnit e = all(*this, id / Hkv);
    x.head = id % Hkv;
    x.nt = (e.t0 + e.ntok + flash::kTok - 1) / flash::kTok;
    x.mode = e.ntok * G > flash::kRows ? flash::kDual : flash::kJoint;
    x.w[0] = e.start;
    x.w[1] = e.t0;
    x.w[2] = e.ntok;
    x.w[3] = e.len;
  }
  // A tile's rows past the sequence are another one's or nobody's (past the tensor: zeros).
  __device__ __forceinline__ uint32_t stale_rows(const flash::Unit& x, int j) const {
    const int n = x.w[3] - j * flash::kTok;  // of the sequence, in the tile
    const int rows = min(flash::kTok - n, num_tokens - x.w[0] - x.w[3]);
    return n < flash::kTok && rows > 0 ? flash::stale_word(n, rows, 0, 0) : 0;
  }
  __device__ __forceinline__ int page(const flash::Unit&, int, int) const { return 0; }
  __device__ __forceinline__ void load_tile(const flash::Unit& x, int j, int kv, int, uint32_t dst, uint32_t bar,
                                            int lane) const {
    if (lane == 0) tma4(dst, kv ? &tv : &tk, 0, x.w[0] + j * flash::kTok, 0, x.head, bar);
  }
  static __device__ __forceinline__ void tma4(uint32_t dst, const CUtensorMap* tm, int c0, int c1, int c2, int c3,
                                              uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(
            dst),
        "l"(tm), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(bar)
        : "memory");
  }
  __device__ __forceinline__ int first_token(const flash::Unit& x, int g) const {
    return x.w[1] + (x.mode == flash::kDual ? g * (flash::kRows / G) : 0);
  }
  __device__ __forceinline__ void find_row(const flash::Unit& x, int g, int r, Row& row) const {
    const int base = first_token(x, g);
    row.tok = base + r / G;
    row.head = x.head * G + r % G;
    row.first = base + (r & ~31) / G;
    row.valid = row.tok < x.w[1] + x.w[2];
  }
  __device__ __forceinline__ void load_q(const flash::Unit& x, int g, int r, uint32_t dst, uint32_t bar,
                                         const Row&) const {
    if (r == 0) {
      mbar_arrive_expect_tx(bar, flash::kTile);
      tma4(dst, &tq, 0, x.head * G, x.w[0] + first_token(x, g), 0, bar);
    }
  }
  __device__ __forceinline__ void loaded_q(int, uint32_t) const {}
  __device__ __forceinline__ flash::Sees sees(const flash::Unit&, const Row& row, int t) const {
    const int k0 = t * flash::kTok;
    return {k0 + flash::kTok - 1 <= row.first, false, row.tok - k0 + 1, 0ull};
  }
  template <class Done>
  __device__ __forceinline__ void out(const flash::Unit& x, const Row& row, uint32_t a, uint32_t b, bool two, float wa,
                                      float wb, float m, float l, Done done, volatile int* again) const {
    const float inv = 1.f / l;
    __nv_bfloat16* dst = o + (x.w[0] + row.tok) * out_stride + row.head * flash::kD;
    bool fine = true;
    flash::walk_o(
        a, b, two, wa, wb,
        [&](int c, auto count, const float* f) {
          constexpr int N = decltype(count)::value;
          uint32_t u[N / 2];
#pragma unroll
          for (int i = 0; i < N; i += 2) {
            const float f0 = f[i] * inv, f1 = f[i + 1] * inv;
            fine = fine && isfinite(f0) && isfinite(f1);
            const __nv_bfloat162 p = __floats2bfloat162_rn(f0, f1);
            u[i / 2] = *reinterpret_cast<const uint32_t*>(&p);
          }
          if (row.valid)
#pragma unroll
            for (int i = 0; i < N / 2; i += 4)
              *reinterpret_cast<uint4*>(dst + c + 2 * i) = make_uint4(u[i], u[i + 1], u[i + 2], u[i + 3]);
        },
        done);
    if (row.valid && !fine && isfinite(m) && isfinite(l)) *again = 1;
  }
  // Rows that only met a value that is not finite in tokens they do not see, a row to a warp (see flash::one_row): those before
  // the last such token of the unit's tiles.
  __device__ __forceinline__ void again(const flash::Unit& x, int warp) const {
    const int lane = threadIdx.x & 31, end = min(x.nt * flash::kTok, x.w[3]);  // (rows behind the sequence were made zero)
    const long long s0 = x.w[0];
    int last = -2;  // not looked for yet
#pragma unroll 1
    for (int i = warp; i < (x.mode == flash::kDual ? 2 : 1) * flash::kRows; i += flash::kKWarp) {
      Row row;
      find_row(x, i / flash::kRows, i % flash::kRows, row);
      if (!row.valid) continue;
      __nv_bfloat16* dst = o + (s0 + row.tok) * out_stride + row.head * flash::kD;
      const uint2 y = reinterpret_cast<const uint2*>(dst)[lane];
      if (!__any_sync(0xffffffffu, flash::not_finite(y.x) || flash::not_finite(y.y))) continue;
      if (last == -2) {
        last = -1;
        for (int j = first_token(x, 0) + 1 + lane; j < end; j += 32)
          if (flash::not_finite(v + (s0 + j) * v_stride + x.head * flash::kD)) last = j;
        last = __reduce_max_sync(0xffffffffu, last);
      }
      if (row.tok >= last) continue;
      float m, l, acc[4];
      if (!flash::one_row(
              q + (s0 + row.tok) * q_stride + row.head * flash::kD, row.tok + 1,
              [&](int j, int kv, const __nv_bfloat16*& to) {
                to = (kv ? v + (s0 + j) * v_stride : k + (s0 + j) * k_stride) + x.head * flash::kD;
                return true;
              },
              qscale, m, l, acc))
        continue;
      for (int c = 0; c < 4; ++c) dst[4 * lane + c] = __float2bfloat16(acc[c] / l);
    }
  }
  __device__ __forceinline__ void drain_q(uint32_t bar) const {
    // A copy in flight lands before the CTA leaves; without one the barrier's last phase passes at once and the other runs out.
    if ((threadIdx.x & 127) == 0) {
      mbar_wait_bounded(bar, 0, kWaitLimitNs / 16);
      mbar_wait_bounded(bar, 1, kWaitLimitNs / 16);
    }
  }
};

__global__ void __launch_bounds__(flash::kThreads, 1) k_prompt(const __grid_constant__ PromptJob job) {
  extern __shared__ __align__(1024) unsigned char sm[];
  flash::body(job, sm);
}

// The self-test of the failure path: the tile `stalled` (0 K, 1 V, 2 the query rows; of the tile or unit `at`) never comes, and the
// waits that this makes run out have a short limit.
struct StalledJob : PromptJob {
  static constexpr uint64_t kWaitNs = 50000000;
  int stalled, at;
  __device__ __forceinline__ void load_tile(const flash::Unit& x, int j, int kv, int page, uint32_t dst, uint32_t bar,
                                            int lane) const {
    if (kv != stalled || j != at) PromptJob::load_tile(x, j, kv, page, dst, bar, lane);
  }
  __device__ __forceinline__ void load_q(const flash::Unit& x, int g, int r, uint32_t dst, uint32_t bar, const Row& row) const {
    if (stalled != 2 || x.w[1] != at) PromptJob::load_q(x, g, r, dst, bar, row);
  }
};

__global__ void __launch_bounds__(flash::kThreads, 1) k_prompt_stalled(const __grid_constant__ StalledJob job) {
  extern __shared__ __align__(1024) unsigned char sm[];
  flash::body(job, sm);
}

// fp32: a CTA per (unit, KV head).
struct PromptTile {
  const float *qp, *kp, *vp;  // the sequence's first row, this head
  float* op;
  long long q_stride, k_stride, v_stride, out_stride;
  int G, t0, ntok;
  __device__ __forceinline__ int tok(int r) const { return t0 + r / G; }
  __device__ __forceinline__ bool valid(int r) const { return r / G < ntok; }
  __device__ __forceinline__ const float* q(int r) const {
    return valid(r) ? qp + tok(r) * q_stride + (r % G) * kTileD : nullptr;
  }
  __device__ __forceinline__ const float* key(int j) const { return kp + j * k_stride; }
  __device__ __forceinline__ const float* val(int j) const { return vp + j * v_stride; }
  __device__ __forceinline__ TileSees sees(int r) const { return {tok(r) + 1, 0, 0ull}; }
  __device__ __forceinline__ void out(int r, int c, float4 o, float, float l) const {
    if (!valid(r)) return;
    const float inv = 1.f / l;
    *reinterpret_cast<float4*>(op + tok(r) * out_stride + (r % G) * kTileD + c) =
        make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
  }
};

__global__ void __launch_bounds__(kTileThreads, 1) k_prompt_f32(PromptView p, const float* q, const float* k,
                                                             const float* v, float* o) {
  pdl_wait();
  pdl_launch_dependents();
  extern __shared__ __align__(16) unsigned char raw[];
  TileSmem& sm = *reinterpret_cast<TileSmem*>(raw);
  const PromptUnits all(p);
  if (blockIdx.x == 0 && threadIdx.x == 0) PromptUnits::status(p);
  const int total = all.count * p.Hkv;
  for (int id = blockIdx.x; id < total; id += gridDim.x) {
    const PromptUnit e = all(p, id / p.Hkv);
    const int h = id % p.Hkv;
    const long long s0 = e.start;
    const PromptTile src{q + s0 * p.q_stride + h * p.G * kTileD,
                         k + s0 * p.k_stride + h * kTileD,
                         v + s0 * p.v_stride + h * kTileD,
                         o + s0 * p.out_stride + h * p.G * kTileD,
                         p.q_stride, p.k_stride, p.v_stride, p.out_stride, p.G, e.t0, e.ntok};
    tile_attention(sm, src, e.t0 + e.ntok, p.qscale);
    __syncthreads();
  }
}

// The rows of a unit: two tiles of 128 for the tensor cores, or one where few units leave SMs without
// work; 32 for the CUDA cores.
int unit_tokens(int dtype, int G) { return (dtype == GB_BF16 ? 2 * flash::kRows : kTileRows) / G; }

bool shape_ok(int dtype, int D, int Hq, int Hkv) {
  const int G = Hkv > 0 && Hq > 0 && Hq % Hkv == 0 ? Hq / Hkv : 0;
  return (G == 1 || G == 2 || G == 4 || G == 8 || G == 16) &&
         ((dtype == GB_BF16 && D == flash::kD) || (dtype == GB_F32 && D == kTileD));
}

long long max_units(int dtype, int G, int num_tokens, int num_seqs) {
  const int least = dtype == GB_BF16 ? flash::kRows / G : kTileRows / G;
  return (long long)num_tokens / least + num_seqs;
}

}  // namespace
}  // namespace gb

using namespace gb;

extern "C" gb_status gb_prompt_workspace_bytes(int num_tokens, int num_seqs, int num_q_heads, int num_kv_heads,
                                               int head_dim, int dtype, size_t* bytes) {
  if (!bytes || num_tokens < 0 || num_seqs < 0 || num_kv_heads < 1 || num_q_heads < 1 || num_q_heads % num_kv_heads)
    return GB_ERR_INVALID;
  if (dtype != GB_F32 && dtype != GB_BF16) return GB_ERR_INVALID;
  if (!shape_ok(dtype, head_dim, num_q_heads, num_kv_heads)) return GB_ERR_UNSUPPORTED;
  const long long n = max_units(dtype, num_q_heads / num_kv_heads, num_tokens, num_seqs);
  if (n * num_kv_heads >= (1ll << 31)) return GB_ERR_TOO_LARGE;
  *bytes = (size_t)(kPrWords * sizeof(int) + n * sizeof(PromptUnit) + num_seqs * sizeof(int) + 255) & ~(size_t)255;
  return GB_OK;
}

namespace {

bool aligned(const void* p, int64_t stride, int esize) { return !((uintptr_t)p & 15) && !((stride * esize) & 15); }

// [first, last) byte addresses of `rows` rows of `width` elements.
bool meets(const void* a, int64_t as, int aw, const void* b, int64_t bs, int bw, int rows, int esize) {
  const uintptr_t a0 = (uintptr_t)a, b0 = (uintptr_t)b;
  const uintptr_t a1 = a0 + ((uintptr_t)(rows - 1) * as + aw) * esize, b1 = b0 + ((uintptr_t)(rows - 1) * bs + bw) * esize;
  return a0 < b1 && b0 < a1;
}

}  // namespace

// stalled: see StalledJob; -1: the call itself.
static gb_status launch_prompt(const gb_prompt_args* a, int stalled, int at, cudaStream_t s) {
  if (!a) return GB_ERR_INVALID;
  size_t need = 0;
  const gb_status st = gb_prompt_workspace_bytes(a->num_tokens, a->num_seqs, a->num_q_heads, a->num_kv_heads,
                                                 a->head_dim, a->dtype, &need);
  if (st != GB_OK) return st;
  if (!a->workspace || ((uintptr_t)a->workspace & 255) || a->workspace_bytes < need || !a->cu_seqlens ||
      !(a->scale > 0.f) || a->scale > 3e38f)
    return GB_ERR_INVALID;
  if (a->num_tokens == 0) return GB_OK;
  const int es = a->dtype == GB_BF16 ? 2 : 4, D = a->head_dim, qw = a->num_q_heads * D, kw = a->num_kv_heads * D;
  if (!a->q || !a->k || !a->v || !a->out || a->q_stride < qw || a->k_stride < kw || a->v_stride < kw ||
      a->out_stride < qw || !aligned(a->q, a->q_stride, es) || !aligned(a->k, a->k_stride, es) ||
      !aligned(a->v, a->v_stride, es) || !aligned(a->out, a->out_stride, es))
    return GB_ERR_INVALID;
  const int64_t widest = std::max(std::max(a->q_stride, a->k_stride), std::max(a->v_stride, a->out_stride));
  if (widest > (int64_t)1 << 31) return GB_ERR_INVALID;
  if (meets(a->out, a->out_stride, qw, a->q, a->q_stride, qw, a->num_tokens, es) ||
      meets(a->out, a->out_stride, qw, a->k, a->k_stride, kw, a->num_tokens, es) ||
      meets(a->out, a->out_stride, qw, a->v, a->v_stride, kw, a->num_tokens, es))
    return GB_ERR_INVALID;
  int device = 0, sms = 0;
  if (cudaGetDevice(&device) != cudaSuccess ||
      cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device) != cudaSuccess)
    return GB_ERR_CUDA;
  if (a->num_seqs == 0) return GB_OK;
  int* ctl = static_cast<int*>(a->workspace);
  const int G = a->num_q_heads / a->num_kv_heads, tokens = unit_tokens(a->dtype, G);
  // Few units (a short prompt): half the rows each, so that twice as many SMs have work and the longest ends sooner.  Up to
  // one and a half units per SM: 1300 tokens of 8 KV heads 25.5 -> 22.2 us, 1600 tokens 29.9 -> 27.7, but 2000 tokens 34.7 -> 36.1.
  const int few = a->dtype == GB_BF16 ? 3 * sms / (2 * a->num_kv_heads) : 0;
  const long long most = max_units(a->dtype, G, a->num_tokens, a->num_seqs);
  PromptView view{ctl, a->cu_seqlens, (int)most, a->num_seqs, tokens, few ? flash::kRows / G : tokens, few,
                  a->num_kv_heads, G, a->num_tokens, a->scale * 1.4426950408889634f, a->q_stride, a->k_stride, a->v_stride, a->out_stride};
  if (a->dtype == GB_BF16 && (!flash::launches_with(reinterpret_cast<const void*>(k_prompt)) ||
                              (stalled >= 0 && !flash::launches_with(reinterpret_cast<const void*>(k_prompt_stalled)))))
    return GB_ERR_UNSUPPORTED;
  // The tensor maps first: nothing is enqueued when one cannot be made.
  StalledJob job;
  if (a->dtype == GB_BF16) {
    static_cast<PromptView&>(job) = view;
    job.stalled = stalled;
    job.at = at;
    job.q = static_cast<const __nv_bfloat16*>(a->q);
    job.k = static_cast<const __nv_bfloat16*>(a->k);
    job.v = static_cast<const __nv_bfloat16*>(a->v);
    job.o = static_cast<__nv_bfloat16*>(a->out);
    const cuuint64_t n = (cuuint64_t)a->num_tokens;
    const cuuint64_t qd[4] = {64, (cuuint64_t)a->num_q_heads, n, 2}, kd[4] = {64, n, 2, (cuuint64_t)a->num_kv_heads};
    const cuuint64_t qs[3] = {256, (cuuint64_t)a->q_stride * 2, 128};
    const cuuint64_t ks[3] = {(cuuint64_t)a->k_stride * 2, 128, 256}, vs[3] = {(cuuint64_t)a->v_stride * 2, 128, 256};
    const cuuint32_t qb[4] = {64, (cuuint32_t)G, (cuuint32_t)(flash::kRows / G), 2}, kb[4] = {64, flash::kTok, 2, 1};
    if (!encode_tensor_map(&job.tq, a->q, 4, qd, qs, qb) || !encode_tensor_map(&job.tk, a->k, 4, kd, ks, kb) ||
        !encode_tensor_map(&job.tv, a->v, 4, kd, vs, kb))
      return GB_ERR_CUDA;
  }
  if (a->num_seqs != 1 &&
      launch_pdl(k_prompt_plan, 1, kListThreads, 0, s, a->cu_seqlens, a->num_seqs, a->num_tokens, tokens,
                 view.small_tokens, few, (int)most, ctl,
                 reinterpret_cast<int*>(reinterpret_cast<PromptUnit*>(ctl + kPrWords) + most)) != cudaSuccess)
    return GB_ERR_CUDA;
  cudaError_t e;
  if (a->dtype == GB_BF16) {
    const void* kernel = stalled < 0 ? reinterpret_cast<const void*>(k_prompt) : reinterpret_cast<const void*>(k_prompt_stalled);
    const unsigned grid = (unsigned)std::min<long long>(sms, most * a->num_kv_heads);
    e = set_max_dynamic_smem(kernel, flash::kSmem);
    if (e == cudaSuccess)
      e = stalled < 0 ? launch_pdl(k_prompt, grid, flash::kThreads, flash::kSmem, s, job)
                      : launch_pdl(k_prompt_stalled, grid, flash::kThreads, flash::kSmem, s, job);
  } else {
    e = set_max_dynamic_smem(reinterpret_cast<const void*>(k_prompt_f32), (int)sizeof(TileSmem));
    if (e == cudaSuccess)
      e = launch_pdl(k_prompt_f32, (unsigned)std::min<long long>(most * a->num_kv_heads, sms * 16), kTileThreads,
                     sizeof(TileSmem), s, view, static_cast<const float*>(a->q), static_cast<const float*>(a->k),
                     static_cast<const float*>(a->v), static_cast<float*>(a->out));
  }
  return e == cudaSuccess ? GB_OK : GB_ERR_CUDA;
}

extern "C" gb_status gb_prompt_attention(const gb_prompt_args* args, gb_stream_t stream) {
  return launch_prompt(args, -1, 0, reinterpret_cast<cudaStream_t>(stream));
}

extern "C" gb_status gb_prompt_wait_selftest(const gb_prompt_args* args, int stalled, int at, gb_stream_t stream) {
  if (!args || args->dtype != GB_BF16 || stalled < 0 || stalled > 2 || at < 0) return GB_ERR_INVALID;
  return launch_prompt(args, stalled, at, reinterpret_cast<cudaStream_t>(stream));
}

extern "C" gb_status gb_prompt_status(const void* workspace_dev, int* device_status, gb_stream_t stream) {
  if (!workspace_dev || !device_status) return GB_ERR_INVALID;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  int v = GB_OK;
  if (cudaMemcpyAsync(&v, static_cast<const int*>(workspace_dev) + kPrStatus, sizeof(int), cudaMemcpyDeviceToHost, s) !=
          cudaSuccess ||
      cudaStreamSynchronize(s) != cudaSuccess)
    return GB_ERR_CUDA;
  *device_status = v;
  return GB_OK;
}
