// Decode attention over pools held in 8 bits.
//
//   out[b][h] = sum_t softmax_t(scale q . k_t) v_t,   k_t = 2^(e_K) c_t,  v_t = 2^(e_V) d_t
// with one e_K and one e_V for each chunk of 16 tokens of a head (rows.cuh).  A chunk is 4 KiB, K and V, brought by one
// TMA into a CTA's ring; its codes become pairs of fp16 in registers (exact) on their way into m16n8k16 products, 8 query
// rows being the N = 8 columns of a tile:
//   S^T[16 tokens][8] = C Q'^T,   s = scale' 2^(e_K) S     (Q' = q times a power of two that brings a row below 2^15: exact
//                                                           for a bf16 row but for values 2^-39 of its largest)
//   O^T[128][8]      += D^T P^T
// A chunk's e_V goes into the exponent of its weights: with t = s + e_V and a running maximum m of the t,
//   p = 2^(t - m),   O += p d,   L += 2^(-e_V) p
// so that the largest contribution to O has a weight near one whatever the blocks' scales, and out = O / L.  p enters the
// products as two fp16 terms (22 bits): one term would be the largest error of the whole by a factor of 100.
// m is set 7 below the largest t of a step of 32 tokens, and raised only when one exceeds it by more than 15: p stays under
// fp16's 2^16, and the last place of a small p (2^-24) is 2^-31 of the largest.  The products' sums are cut off rather than
// rounded, which adds up over a thousand chunks (to 8e-6 of the output), so each step's are added to O in fp32.
//
// Fragments are chosen so that a lane's operands are 16-byte pieces: the dims (the k of S) and the dims of O^T's rows
// are permuted, which the queries and the output follow.  Lane (r = lane / 4, c = lane % 4) reads dims 32c .. 32c + 31 of
// tokens r, r + 8 of K, and dims 16r .. 16r + 15 of tokens 2c, 2c + 1, 2c + 8, 2c + 9 of V, whose codes are
// interleaved in pairs by byte permutes: 8 loads, 64 conversions, 16 permutes and 24 products a chunk and tile.
//
// Work.  A unit is a run of chunks of one head's pages with the query rows that see them: a beam's own (its G heads), or a
// shared segment's (up to 64 rows of its members; the lists that the grouped path of bf16 pools uses).  A CTA has a warp that
// takes units from the launch's counters, two that stream their chunks through a ring, two chunks a stage, and
// eight warps that share out a unit: row groups of 8 rows, and where those are fewer than eight, groups of stages
// among the warps of a row group, whose softmax states are merged in shared memory when the unit ends.  Units' records are
// merged at the end of the launch (combine.cuh); a beam whose whole context was one unit is written at once.
//
// What bounds it (a launch alone, one layer): unshared caches, memory: 64 x 16384 tokens in 355 us, 6.1 TB/s (without the products
// 339).  Shared ones, the multiplying warps: the same bytes from L2 take 263 us, 8.0 TB/s, without the products 162.  A tile's 32
// tokens are 48 products (384 cycles of a scheduler's) and 540 instructions, for which a warp takes 2200 cycles, two a scheduler; with
// twelve warps, two tiles a warp that share their conversions, or the next stage's K asked for early, the SM does no more.  Small calls, a chain: barriers, plan, page
// ids and exponents, first chunks, merge: 13-15 us cold for 8 or 13 beams, 2.5 of them before the first copy.
#include <float.h>

#include <atomic>

#include "decode_mma.cuh"
#include "rows.cuh"

namespace gb {
namespace {

constexpr int kConsumers8 = 8;                     // warps that multiply
constexpr int kLoaders8 = 2;                       // and that load: each has every second slot of the ring (one issues 34 GB/s an SM)
constexpr int kThreads8 = (kConsumers8 + 4) * 32;  // one that plans, the loaders, and one idle (registers are shared out by fours)
constexpr int kConsumerRegs8 = 216, kLoaderRegs8 = 72;
static_assert((kConsumers8 * kConsumerRegs8 + 4 * kLoaderRegs8) * 32 <= kThreads8 * 168, "shares of the registers at launch");
constexpr int kStages8 = 24;                       // 192 KiB on their way an SM: with 128 the unshared 64 x 16384 tokens take 365 us
// A slot of the ring has the same warps for its stage n and its stage n + kStages8: others could look for the second
// while the first is still on its way, and a barrier cannot tell a phase from the one before the last.
static_assert(kStages8 % kConsumers8 == 0 && kStages8 % kLoaders8 == 0, "groups of stages keep their slots");
constexpr int kChunkBytes8 = 2 * kChunk * 128;     // K and V
constexpr int kStageBytes8 = 2 * kChunkBytes8;     // two chunks
constexpr int kSlots8 = 4;                         // units known ahead
constexpr int kRows8 = 64;                         // query rows of a unit: a tile for each warp
constexpr int kRowFloats8 = 132;                   // of a row in the merge's memory

enum UnitKind : int { kUnitEnd = 0, kUnitBeam = 1, kUnitSegment = 2 };
struct Unit8 {
  int kind, head, tokens, rows;
  int record;    // beam: the record's index
  int direct;    // beam: its only record, so its output
  int source, tok0, again;  // whose table, the first token there, whether others read the pages too
  int members[kRows8];  // the rows' beams
  int records[kRows8];  // segment: their records (of grec, in all heads)
};

struct Smem8 {
  static constexpr int RING = kStages8 * kStageBytes8;
  static constexpr int MERGE = RING;                                                  // float [8 warps][4 rows][132]
  static constexpr int STATE = MERGE + kConsumers8 * 4 * kRowFloats8 * 4;             // float [8 warps][4 rows][m, l]
  static constexpr int EXPS = STATE + kConsumers8 * 4 * 2 * 4;                        // int [stages][K, V of two chunks]
  static constexpr int UNITS = EXPS + kStages8 * 16;
  static constexpr int BARS = UNITS + kSlots8 * (int)sizeof(Unit8);
  static constexpr int STOP = BARS + (2 * kStages8 + 2 * kSlots8) * 8;                // set when a wait ran out
  static constexpr int PLAN = STOP + 8;                                               // offsets, chunk counts
  static constexpr int TOTAL = 1024 + PLAN + 2 * (kMaxBeams + 1) * 4;
  static_assert(BARS % 8 == 0 && EXPS % 16 == 0, "alignment");
  static_assert(TOTAL <= 232448, "shared memory per block");
};

__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                        uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
      "{%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
  uint32_t y;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(y) : "f"(hi), "f"(lo));
  return y;
}

__device__ __forceinline__ uint4 ld_shared16(uint32_t addr) {
  uint4 x;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w) : "r"(addr) : "memory");
  return x;
}

__device__ __forceinline__ void mbar_arrive_n(uint32_t bar, uint32_t n) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(n) : "memory");
}

// The eight multiplying warps.
__device__ __forceinline__ void consumers_sync() { asm volatile("bar.sync 1, %0;" ::"n"(kConsumers8 * 32) : "memory"); }

// The same, and whether any thread says so.
__device__ __forceinline__ bool consumers_any(bool x) {
  int any;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.s32 p, %1, 0;\n\tbarrier.cta.red.or.pred q, 1, %2, p;\n\tselp.s32 %0, 1, 0, q;\n\t}"
      : "=r"(any)
      : "r"((int)x), "n"(kConsumers8 * 32)
      : "memory");
  return any != 0;
}

// A bounded wait that the CTA's other waits end too: the first that runs out stops them all.  The lanes may leave it apart:
// callers bring them together again before an instruction of the whole warp, or one that takes uniform registers.
__device__ __forceinline__ bool wait_or_stop(uint32_t bar, uint32_t parity, volatile int* stop) {
  if (mbar_try_wait(bar, parity)) return true;
  const uint64_t t0 = globaltimer_ns();
  for (uint32_t it = 1;; ++it) {
    if (mbar_try_wait(bar, parity)) return true;
    if ((it & 63) == 0 && (*stop != 0 || globaltimer_ns() - t0 > kWaitLimitNs)) {
      *stop = 1;
      return false;
    }
  }
}

// K and V of one chunk of one head: box {128 bytes, 16 rows, K|V, 1} at row group g.
__device__ __forceinline__ void tma_chunk8(uint32_t dst, const CUtensorMap* tm, int g, uint32_t bar, uint64_t pol) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint"
      " [%0], [%1, {%2, %3, %4, %5}], [%6], %7;" ::"r"(dst),
      "l"(tm), "r"(0), "r"(0), "r"(0), "r"(g), "r"(bar), "l"(pol)
      : "memory");
}

// One tile of 8 query rows in a warp.
struct Tile8 {
  uint32_t q[8][2];  // Q'^T: row r, dims 32c + 4j (+1), (+2, +3)
  float s0, s1;      // scale' of columns 2c, 2c + 1 over their rows' powers of two
  float2 o[8][2];    // O^T: columns 2c, 2c + 1 of dims 16r + 2i, then 16r + 2i + 1
  float m0, m1, l0, l1;
};

// This lane's part of a query row (128 bf16; nullptr: zeros), into the tile's own registers until tile_begin.
__device__ __forceinline__ void tile_load(Tile8& t, const __nv_bfloat16* row, int c) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint4 x = row ? *reinterpret_cast<const uint4*>(row + 32 * c + 8 * i) : make_uint4(0u, 0u, 0u, 0u);
    t.q[2 * i][0] = x.x;
    t.q[2 * i][1] = x.y;
    t.q[2 * i + 1][0] = x.z;
    t.q[2 * i + 1][1] = x.w;
  }
}
__device__ __forceinline__ void tile_begin(Tile8& t, float qscale, int c) {
  uint32_t w[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) w[i] = t.q[i >> 1][i & 1];
  float amax = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const float a = fabsf(__uint_as_float(w[i] << 16)), b = fabsf(__uint_as_float(w[i] & 0xffff0000u));
    amax = fmaxf(amax, a <= 3.4e38f ? a : 0.f);
    amax = fmaxf(amax, b <= 3.4e38f ? b : 0.f);
  }
  amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
  amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
  // 2^sh brings the largest value into [2^14, 2^15).
  const int ex = (int)(__float_as_uint(amax) >> 23) - 127, sh = min(max(14 - ex, -113), 126);
  const float up = pow2i(sh);
#pragma unroll
  for (int i = 0; i < 16; ++i)
    t.q[i >> 1][i & 1] = pack_f16x2(__uint_as_float(w[i] << 16) * up, __uint_as_float(w[i] & 0xffff0000u) * up);
  const float back = qscale * pow2i(-sh);
  t.s0 = __shfl_sync(0xffffffffu, back, 8 * c);      // row 2c's first lane
  t.s1 = __shfl_sync(0xffffffffu, back, 8 * c + 4);
#pragma unroll
  for (int i = 0; i < 8; ++i) t.o[i][0] = t.o[i][1] = make_float2(0.f, 0.f);
  t.m0 = t.m1 = -FLT_MAX;  // not -infinity: a warp whose scores are all NaN has a state, which the merges keep
  t.l0 = t.l1 = 0.f;
}

// K words of a landed stage's two chunks: tokens r, r + 8; dims 32c + 4j .. + 3.
__device__ __forceinline__ void take_k(uint32_t (&w)[2][2][8], uint32_t sb, int r, int c) {
#pragma unroll
  for (int k = 0; k < 2; ++k)
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int z = 0; z < 2; ++z) {
        const uint4 x = ld_shared16(sb + k * kChunkBytes8 + (r + 8 * i) * 128 + (((2 * c + z) ^ r) << 4));
        w[k][i][4 * z] = x.x;
        w[k][i][4 * z + 1] = x.y;
        w[k][i][4 * z + 2] = x.z;
        w[k][i][4 * z + 3] = x.w;
      }
}
// V pieces: tokens 2c, 2c + 1, 2c + 8, 2c + 9; dims 16r .. + 15.
__device__ __forceinline__ void take_v(uint4 (&x)[2][4], uint32_t sb, int nvalid, int r, int c) {
#pragma unroll
  for (int k = 0; k < 2; ++k)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int tok = 2 * c + (i & 1) + 8 * (i >> 1);
      x[k][i] = ld_shared16(sb + k * kChunkBytes8 + kChunk * 128 + tok * 128 + ((r ^ (tok & 7)) << 4));
      if (nvalid < 2 * kChunk && 16 * k + tok >= nvalid) x[k][i] = make_uint4(0u, 0u, 0u, 0u);  // whatever is there
    }
}

// A landed stage (its first nvalid >= 1 tokens) into a tile.  e: K's and V's exponent of each chunk.  leave() gives its slot back: V
// is in registers before it is multiplied.
template <class Leave>
__device__ __forceinline__ void attend(Tile8& u, uint32_t sb, int nvalid, const int (&e)[2][2], int r, int c, Leave leave) {
  uint32_t w[2][2][8];
  uint4 x[2][4];
  take_k(w, sb, r, c);
  take_v(x, sb, nvalid, r, c);
  float y[2][4];
  {
    float s[2][2][4];  // two independent sums a chunk: a product waits for the one before it for as long as four others take
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int z = 0; z < 4; ++z) s[k][0][z] = s[k][1][z] = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int k = 0; k < 2; ++k)
        mma_f16(s[k][j & 1], f16x2_of_e4m3x2(w[k][0][j]), f16x2_of_e4m3x2(w[k][1][j]), f16x2_of_e4m3x2(w[k][0][j] >> 16),
                f16x2_of_e4m3x2(w[k][1][j] >> 16), u.q[j][0], u.q[j][1]);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const float ks = pow2i(e[k][0]), k0 = u.s0 * ks, k1 = u.s1 * ks, add = (float)e[k][1];
#pragma unroll
      for (int z = 0; z < 4; ++z) y[k][z] = fmaf(s[k][0][z] + s[k][1][z], z & 1 ? k1 : k0, add);
      if (nvalid < 2 * kChunk) {
        if (16 * k + r >= nvalid) y[k][0] = y[k][1] = -INFINITY;
        if (16 * k + r + 8 >= nvalid) y[k][2] = y[k][3] = -INFINITY;
      }
    }
  }
  leave();
  float mx0 = fmaxf(fmaxf(y[0][0], y[0][2]), fmaxf(y[1][0], y[1][2]));
  float mx1 = fmaxf(fmaxf(y[0][1], y[0][3]), fmaxf(y[1][1], y[1][3]));
  if (__any_sync(0xffffffffu, mx0 > u.m0 + 15.f || mx1 > u.m1 + 15.f)) {
#pragma unroll
    for (int o = 4; o < 32; o <<= 1) {
      mx0 = fmaxf(mx0, __shfl_xor_sync(0xffffffffu, mx0, o));
      mx1 = fmaxf(mx1, __shfl_xor_sync(0xffffffffu, mx1, o));
    }
    const bool up0 = mx0 > u.m0 + 15.f, up1 = mx1 > u.m1 + 15.f;
    const float n0 = up0 ? mx0 - 7.f : u.m0, n1 = up1 ? mx1 - 7.f : u.m1;
    const float2 f = make_float2(up0 ? ex2_approx(u.m0 - n0) : 1.f, up1 ? ex2_approx(u.m1 - n1) : 1.f);
    u.m0 = n0;
    u.m1 = n1;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      u.o[i][0] = __fmul2_rn(u.o[i][0], f);
      u.o[i][1] = __fmul2_rn(u.o[i][1], f);
    }
    u.l0 *= f.x;
    u.l1 *= f.y;
  }
  uint32_t hi[2][2], lo[2][2];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const float p0 = ex2_approx(y[k][0] - u.m0), p1 = ex2_approx(y[k][1] - u.m1);
    const float p2 = ex2_approx(y[k][2] - u.m0), p3 = ex2_approx(y[k][3] - u.m1);
    const float back = pow2i(-e[k][1]);
    u.l0 = fmaf(p0 + p2, back, u.l0);
    u.l1 = fmaf(p1 + p3, back, u.l1);
    const uint32_t h0 = pack_f16x2(p0, p1), h1 = pack_f16x2(p2, p3);
    const float2 g0 = float2_of_f16x2(h0), g1 = float2_of_f16x2(h1);
    hi[k][0] = movmatrix_t(h0);
    hi[k][1] = movmatrix_t(h1);
    lo[k][0] = movmatrix_t(pack_f16x2(p0 - g0.x, p1 - g0.y));
    lo[k][1] = movmatrix_t(pack_f16x2(p2 - g1.x, p3 - g1.y));
  }
#pragma unroll
  for (int i0 = 0; i0 < 8; i0 += 4) {
    float d[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) d[i][0] = d[i][1] = d[i][2] = d[i][3] = 0.f;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const uint32_t* v0 = &x[k][0].x;
      const uint32_t* v1 = &x[k][1].x;
      const uint32_t* v2 = &x[k][2].x;
      const uint32_t* v3 = &x[k][3].x;
      uint32_t a[4][4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int at = (i0 + i) >> 1;
        const uint32_t sel = i & 1 ? 0x7362 : 0x5140;
        const uint32_t f = __byte_perm(v0[at], v1[at], sel), g = __byte_perm(v2[at], v3[at], sel);
        a[i][0] = f16x2_of_e4m3x2(f);
        a[i][1] = f16x2_of_e4m3x2(f >> 16);
        a[i][2] = f16x2_of_e4m3x2(g);
        a[i][3] = f16x2_of_e4m3x2(g >> 16);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) mma_f16(d[i], a[i][0], a[i][1], a[i][2], a[i][3], lo[k][0], lo[k][1]);
#pragma unroll
      for (int i = 0; i < 4; ++i) mma_f16(d[i], a[i][0], a[i][1], a[i][2], a[i][3], hi[k][0], hi[k][1]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      u.o[i0 + i][0] = __fadd2_rn(u.o[i0 + i][0], make_float2(d[i][0], d[i][1]));
      u.o[i0 + i][1] = __fadd2_rn(u.o[i0 + i][1], make_float2(d[i][2], d[i][3]));
    }
  }
}

__device__ __forceinline__ void tile_finish(Tile8& t) {
#pragma unroll
  for (int o = 4; o < 32; o <<= 1) {
    t.l0 += __shfl_xor_sync(0xffffffffu, t.l0, o);
    t.l1 += __shfl_xor_sync(0xffffffffu, t.l1, o);
  }
}

// Four floats of column 2c + z: dims 16r + 4i ..
__device__ __forceinline__ float4 tile_dims(const Tile8& t, int i, int z) {
  const float2 a = t.o[2 * i][0], b = t.o[2 * i][1], c = t.o[2 * i + 1][0], d = t.o[2 * i + 1][1];
  return z ? make_float4(a.y, b.y, c.y, d.y) : make_float4(a.x, b.x, c.x, d.x);
}

// How a launch takes its beams' own chunks: whole (beam, KV head) pairs, or ranges of the flat list: one of `large` chunks for each
// CTA, and the others of `small` for whoever is done first.
struct Shares {
  bool pairs;
  int large, small, ctas, count;
  __device__ __forceinline__ int begin(int u) const { return u < ctas ? u * large : ctas * large + (u - ctas) * small; }
  __device__ __forceinline__ int of(int x) const {
    if (pairs) return 0;
    return x < ctas * large ? x / large : ctas + (x - ctas * large) / small;
  }
};

__device__ __forceinline__ Shares shares_of(const PoolView& v, int mode, int nact, int total, int ctas) {
  Shares s;
  const int pairs = max(nact, 1) * v.Hkv, even = max(1, (total + ctas - 1) / ctas);
  s.pairs = false;
  s.ctas = ctas;
  // SMs differ, so a tenth of long shares is left for the end.  (In four parts each, a CTA that took a fifth one held up the others
  // for a fifth of the time.  us of 64 x 16384 unshared tokens and 198 x 8000, G = 8, as measured then: four parts 385, 280; four fifths
  // and parts of a twentieth 354, 261; nine tenths and a thirty-second 351, 256; two thirds and a sixteenth 347, 274.)
  s.large = even > 160 ? even * 9 / 10 : even;
  s.small = even > 160 ? max(32, even / 32) : 1;
  const int rest = total - ctas * s.large;
  s.count = rest > 0 ? ctas + (rest + s.small - 1) / s.small : (total + s.large - 1) / s.large;
  if (mode == 1) {  // whoever is done with its segments takes the next one
    s.pairs = total <= 64ll * pairs;
  } else {
    // Chunks that pass a CTA, and a unit's start and merge as so many more.
    const int whole = (pairs + ctas - 1) / ctas * ((total + pairs - 1) / pairs + 16);
    s.pairs = whole <= even + 48;
  }
  if (s.pairs) s.count = v.max_beams * v.Hkv;
  return s;
}

// ---- the loading warps -----------------------------------------------------------------------------

// The stages of every unit whose ring slot is this loader's (number `own` of kLoaders8), but for the CTA's stage `stalled`, which never
// comes (-1: none, but in a self-test).
__device__ void load_stages(const PoolView& v, const CUtensorMap* tm, int layer, int stalled, unsigned char* smem, uint32_t bars, int own,
                            int lane) {
  const uint32_t full = bars, empty = bars + 8 * kStages8, ufull = bars + 16 * kStages8, uempty = ufull + 8 * kSlots8;
  volatile int* stop = reinterpret_cast<volatile int*>(smem + Smem8::STOP);
  const uint64_t once = policy_evict_first(), more = policy_evict_normal();
  const int pg = v.P / kChunk;
  const long long layer_pages = (long long)layer * v.num_pages;
  const size_t gap = (size_t)v.Hkv * pg;  // exponents from K to V
  uint32_t base = 0, top = 0;  // stages of earlier units; past the last that may be on its way
  bool ok = true;
  for (int k = 0; ok; ++k) {
    const int slot = k % kSlots8;
    ok = __all_sync(0xffffffffu, wait_or_stop(ufull + 8 * slot, (k / kSlots8) & 1, stop));
    if (!ok) break;
    const Unit8& u = reinterpret_cast<const Unit8*>(smem + Smem8::UNITS)[slot];
    const int kind = u.kind, h = u.head, tok0 = u.tok0, n = (u.tokens + kChunk - 1) / kChunk, stages = (n + 1) / 2;
    const int* table = v.tables + (size_t)u.source * v.max_pages;
    const uint64_t pol = u.again ? more : once;
    __syncwarp();
    if (lane == 0) mbar_arrive_n(uempty + 8 * slot, 1);
    __syncwarp();
    if (kind == kUnitEnd) return;
    // A chunk a lane: chunk lane % 2 of the loader's stage lane / 2, 16 of its stages at a time.
    const int first = (int)((own - base) & (kLoaders8 - 1));
    auto chunk_at = [&](int i0) { return 2 * (first + kLoaders8 * (i0 + (lane >> 1))) + (lane & 1); };
    auto page_at = [&](int c) { return c < n ? table[(tok0 + c * kChunk) / v.P] : 0; };
    auto group_at = [&](int c, int page) -> long long {  // row group of the chunk's K
      if (page < 0 || page >= v.num_pages) {
        if (c < n) set_status(v.ctl, GB_ERR_INVALID);
        page = 0;
      }
      return ((layer_pages + page) * 2 * v.Hkv + h) * pg + ((tok0 + c * kChunk) & (v.P - 1)) / kChunk;
    };
    int c = chunk_at(0);
    long long g = group_at(c, page_at(c));
    int ek = v.kv_exp[g], ev = v.kv_exp[g + gap];
    for (int i0 = 0; ok && first + kLoaders8 * i0 < stages; i0 += 16) {
      const int next = chunk_at(i0 + 16), page = page_at(next);
      const bool on = first + kLoaders8 * (i0 + 16) < stages;
      long long gn = 0;
      int ekn = 0, evn = 0;
      const int i = c >> 1;  // the unit's stage
      const uint32_t kk = base + i, st = kk % kStages8;
      const bool in = c < n, there = i < stages;
      top = base + min(stages, first + kLoaders8 * (i0 + 16));
#pragma unroll 1
      for (int z = 0; z < 4 && first + kLoaders8 * (i0 + 4 * z) < stages; ++z) {
        if (z == 2 && on) {  // the page ids are there by now
          gn = group_at(next, page);
          ekn = v.kv_exp[gn];
          evn = v.kv_exp[gn + gap];
        }
        // Eight lanes at a time.
        const bool mine = lane >> 3 == z && there;
        const bool good = !(mine && kk >= kStages8) || wait_or_stop(empty + 8 * st, (kk / kStages8 - 1) & 1, stop);
        ok = __all_sync(0xffffffffu, good);
        if (!ok) break;
        if (mine && (int)kk != stalled) {
          *reinterpret_cast<int2*>(smem + Smem8::EXPS + 16 * st + 8 * (lane & 1)) = in ? make_int2(ek, ev) : make_int2(0, 0);
          const uint32_t bar = full + 8 * st;
          if (in) {
            mbar_arrive_expect_tx(bar, kChunkBytes8);
            tma_chunk8(smem_addr(smem) + st * kStageBytes8 + (lane & 1) * kChunkBytes8, tm, (int)g, bar, pol);
          } else {
            mbar_arrive_n(bar, 1);
          }
        }
        __syncwarp();
      }
      if (!ok) break;
      c = next;
      g = gn;
      ek = ekn;
      ev = evn;
    }
    base += stages;
  }
  // A wait ran out: leave no copy in flight.  (What was not issued runs out at once.)
  for (int d = lane; d < 32 + kStages8; d += 32) {
    const uint32_t last = top - 1 - d;
    if ((int)last >= 0) mbar_wait_bounded(full + 8 * (last % kStages8), (last / kStages8) & 1, kWaitLimitNs / 100);
  }
}

// ---- the planning warp -----------------------------------------------------------------------------

struct Planner8 {
  const int lane;
  unsigned char* const smem;
  const uint32_t ufull, uempty;
  volatile int* const stop;
  int units = 0;         // published
  bool ok = true;

  // The next unit's slot, once its last users have read it.
  __device__ Unit8* slot() {
    const int k = units % kSlots8;
    const bool free = units < kSlots8 || wait_or_stop(uempty + 8 * k, (units / kSlots8 - 1) & 1, stop);
    ok = __all_sync(0xffffffffu, free) && ok;
    return reinterpret_cast<Unit8*>(smem + Smem8::UNITS) + k;
  }
  __device__ void publish() {
    __syncwarp();
    if (lane == 0) mbar_arrive_n(ufull + 8 * (units % kSlots8), 1);
    __syncwarp();
    ++units;
  }
};

template <int G>
__device__ void plan_units(const PoolView& v, const Counters& cnt, int mode, const Shares& sh, unsigned char* smem, uint32_t bars, int lane) {
  const int* s_off = reinterpret_cast<const int*>(smem + Smem8::PLAN);
  const int* s_n = s_off + (kMaxBeams + 1);
  Planner8 pl{lane, smem, bars + 16 * kStages8, bars + 16 * kStages8 + 8 * kSlots8, reinterpret_cast<volatile int*>(smem + Smem8::STOP)};
  const bool shared = v.ctl[kCtlSegCount] > 0;
  auto claim = [&](int word) {
    int x = 0;
    if (lane == 0) x = atomicAdd(&cnt.c[word], 1);
    return x;
  };
  if (mode == 1) {
    // The lists' tiles are of 128 rows: two units each, the second one empty where the members end before.
    constexpr int members = kRows8 / G;
    const int tiles = v.ctl[kCtlSegTiles], split = v.ctl[kCtlSegSplit];
    const long long all = 2ll * tiles * v.Hkv;
    int pending = (int)blockIdx.x;
    while (pl.ok) {
      const int u = __shfl_sync(0xffffffffu, pending, 0);
      if (u >= all) break;
      pending = (int)gridDim.x + claim(kCntGrpNext);
      const int tq = u / (2 * v.Hkv), h = u / 2 % v.Hkv;
      const int s = v.seg_tile_seg[tq], t = v.seg_tile_t[tq], sp = v.seg_tile_split[tq];
      const int g = v.seg_g[s], moff = v.seg_mem_off[s], rep = v.seg_rep[s];
      const int tok0 = sp * split, tokens = min(v.seg_len[s] * v.P - tok0, split);
      const int m0 = (2 * t + (u & 1)) * members, have = min(members, g - m0);
      if (have <= 0) continue;
      Unit8* x = pl.slot();
      if (!pl.ok) break;
      for (int m = lane; m < have; m += 32) {
        const int e = v.seg_members[moff + m0 + m], b = e / kMaxSegDepth;
        x->members[m] = b;
        x->records[m] = b * kMaxSegRecords + v.seg_rec_off[e] + sp;
      }
      if (lane == 0) {
        x->kind = kUnitSegment;
        x->head = h;
        x->tokens = tokens;
        x->rows = have * G;
        x->source = rep;
        x->tok0 = v.seg_i0[s] * v.P + tok0;
        x->again = g > members;
      }
      pl.publish();
    }
  }
  // One (beam, head)'s chunks [i, i + n) of its list.
  auto beam_unit = [&](int b, int h, int i, int n, int range) {
    Unit8* x = pl.slot();
    if (!pl.ok) return;
    const int tok0 = plan_start(v, mode)[b] + i * kChunk, tokens = min(n * kChunk, v.seq_len[b] - tok0);
    if (lane == 0) {
      x->kind = kUnitBeam;
      x->head = h;
      x->tokens = tokens;
      x->rows = G;
      x->record = range + b * v.Hkv + h;
      x->direct = n == s_n[b] && (mode == 0 || v.seg_nrec[b] == 0);
      x->members[0] = b;
      x->source = b;
      x->tok0 = tok0;
      x->again = mode == 0 && shared;
    }
    pl.publish();
  };
  // The first share is the CTA's own, the others are whoever's comes first; behind segments, all of them.
  const int own = mode == 1 ? 0 : (int)gridDim.x;
  int pending = own ? (int)blockIdx.x : claim(kCntRange);
  while (pl.ok) {
    const int u = __shfl_sync(0xffffffffu, pending, 0);
    if (u >= sh.count) break;
    if (sh.count > own) pending = own + claim(kCntRange);
    else pending = sh.count;
    if (sh.pairs) {
      const int b = u / v.Hkv;
      if (s_n[b] > 0) beam_unit(b, u - b * v.Hkv, 0, s_n[b], 0);
      continue;
    }
    int x = sh.begin(u);
    const int end = min(s_off[v.max_beams], sh.begin(u + 1));
    int b = 0, hi = v.max_beams;  // s_off[b] <= x < s_off[hi]
    while (hi - b > 1) {
      const int mid = (b + hi) >> 1;
      if (s_off[mid] <= x) b = mid; else hi = mid;
    }
    while (x < end && pl.ok) {
      while (s_off[b + 1] <= x) ++b;
      const int h = (x - s_off[b]) / s_n[b], i = x - s_off[b] - h * s_n[b], n = min(s_n[b] - i, end - x);
      beam_unit(b, h, i, n, u);
      x += n;
    }
  }
  if (pl.ok) {
    Unit8* x = pl.slot();
    if (pl.ok && lane == 0) x->kind = kUnitEnd;
    if (pl.ok) pl.publish();
  }
}

// ---- the multiplying warps --------------------------------------------------------------------------

// Where a unit's row goes: its record, or its output.
template <int G>
__device__ __forceinline__ float* row_record(const PoolView& v, const Unit8& u, int row) {
  if (u.kind == kUnitBeam) return v.partials + (size_t)u.record * v.record_floats;
  return v.grec + ((size_t)u.records[row / G] * v.Hkv + u.head) * v.record_floats;
}

// How the multiplying warps share out a unit: row groups of 8 rows (1, 2, 4 or 8), and in each as many groups of stages as
// there are warps for it.
__device__ __forceinline__ int row_groups(int rows) { return rows <= 8 ? 1 : rows <= 16 ? 2 : rows <= 32 ? 4 : 8; }

// This warp's query rows of a unit, on their way.
template <int G>
__device__ __forceinline__ void load_queries(Tile8& t, const PoolView& v, const Unit8& u, const __nv_bfloat16* q, int warp, int r, int c) {
  if (u.kind == kUnitEnd) return;
  const int row = warp % row_groups(u.rows) * 8 + r;
  tile_load(t, row < u.rows ? q + ((size_t)u.members[row / G] * v.Hq + (size_t)u.head * G + row % G) * 128 : nullptr, c);
}

// One unit by the multiplying warps.  A warp whose wait ran out still keeps step with the others, and none of the unit's outputs is
// written (its records may be: nobody counts them): false.  next(): called when the queries are no longer needed.
template <int G, class Next>
__device__ __forceinline__ bool multiply(Tile8& t, const PoolView& v, const Unit8& u, float qscale, uint32_t base, uint32_t bars,
                                         unsigned char* smem, float* out, Next next) {
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, r = lane >> 2, c = lane & 3;
  const uint32_t full = bars, empty = bars + 8 * kStages8, ring = smem_addr(smem);
  volatile int* stop = reinterpret_cast<volatile int*>(smem + Smem8::STOP);
  const int rgroups = row_groups(u.rows), groups = kConsumers8 / rgroups, rg = warp % rgroups, group = warp / rgroups;
  tile_begin(t, qscale, c);
  const int stages = (u.tokens + 2 * kChunk - 1) / (2 * kChunk);
  const bool any = rg * 8 < u.rows;  // (without rows the stages' slots are only given back)
  bool whole = true;
#pragma unroll 1
  for (int i = group; i < stages; i += groups) {
    const uint32_t k = base + i, s = k % kStages8;
    if (!__all_sync(0xffffffffu, wait_or_stop(full + 8 * s, (k / kStages8) & 1, stop))) {
      whole = false;
      break;
    }
    auto leave = [&] {
      __syncwarp();
      if (lane == 0) mbar_arrive_n(empty + 8 * s, groups);
      __syncwarp();
    };
    if (any) {
      const int4 e = *reinterpret_cast<const int4*>(smem + Smem8::EXPS + 16 * s);
      const int eh[2][2] = {{e.x, e.y}, {e.z, e.w}};
      attend(t, ring + s * kStageBytes8, min(2 * kChunk, u.tokens - i * 2 * kChunk), eh, r, c, leave);
    } else {
      leave();
    }
  }
  next();
  tile_finish(t);
  const uint64_t pol = policy_evict_last();  // the launch's merge reads the records back from L2
  if (groups == 1) {                         // nobody else has these rows
#pragma unroll
    for (int z = 0; z < 2; ++z) {
      const int row = rg * 8 + 2 * c + z;
      if (row >= u.rows) continue;
      float* rec = row_record<G>(v, u, row);
#pragma unroll
      for (int i = 0; i < 4; ++i) st_hint4(rec + row % G * 128 + 16 * r + 4 * i, tile_dims(t, i, z), pol);
      if (r == 0) {
        st_hint(rec + G * 128 + row % G, z ? t.m1 : t.m0, pol);
        st_hint(rec + G * 128 + G + row % G, z ? t.l1 : t.l0, pol);
      }
    }
    return whole;
  }
  // The warps' states of the same rows, merged through shared memory four rows of each at a time.
  float* left = reinterpret_cast<float*>(smem + Smem8::MERGE);
  float2* ml = reinterpret_cast<float2*>(smem + Smem8::STATE);
#pragma unroll 1
  for (int f = 0; f < 2; ++f) {
    if (f > 0 && 4 * f >= u.rows) break;
    if (c >> 1 == f) {
#pragma unroll
      for (int z = 0; z < 2; ++z) {
        const int in = warp * 4 + 2 * (c & 1) + z;
#pragma unroll
        for (int i = 0; i < 4; ++i) *reinterpret_cast<float4*>(left + in * kRowFloats8 + 16 * r + 4 * i) = tile_dims(t, i, z);
        if (r == 0) ml[in] = z ? make_float2(t.m1, t.l1) : make_float2(t.m0, t.l0);
      }
    }
    if (consumers_any(!whole)) return false;
    for (int i = tid; i < rgroups * 4 * 32; i += kConsumers8 * 32) {
      const int g = i >> 7, in = (i >> 5) & 3, row = g * 8 + 4 * f + in, d = 4 * (i & 31);
      if (row >= u.rows) continue;
      float M = -FLT_MAX;
      for (int k = 0; k < groups; ++k) M = fmaxf(M, ml[(g + k * rgroups) * 4 + in].x);
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
      float L = 0.f;
      for (int k = 0; k < groups; ++k) {
        const int w = (g + k * rgroups) * 4 + in;
        const float2 a = ml[w];
        const float f2 = exp2f(a.x - M);  // (a warp without a stage adds zeros)
        const float4 x = *reinterpret_cast<const float4*>(left + w * kRowFloats8 + d);
        acc.x = fmaf(x.x, f2, acc.x);
        acc.y = fmaf(x.y, f2, acc.y);
        acc.z = fmaf(x.z, f2, acc.z);
        acc.w = fmaf(x.w, f2, acc.w);
        L = fmaf(a.y, f2, L);
      }
      if (u.kind == kUnitBeam && u.direct) {
        float* to = out + ((size_t)u.members[0] * v.Hq + (size_t)u.head * G + row) * 128 + d;
        to[0] = acc.x / L;
        to[1] = acc.y / L;
        to[2] = acc.z / L;
        to[3] = acc.w / L;
      } else {
        float* rec = row_record<G>(v, u, row);
        st_hint4(rec + row % G * 128 + d, acc, pol);
        if (d == 0) {
          st_hint(rec + G * 128 + row % G, M, pol);
          st_hint(rec + G * 128 + G + row % G, L, pol);
        }
      }
    }
    consumers_sync();
  }
  return true;
}

// Every unit that the CTA takes; false where a wait ran out.
template <int G>
__device__ bool multiply_units(const PoolView& v, const Counters& cnt, const __nv_bfloat16* q, float qscale, int mode, unsigned char* smem,
                               uint32_t bars, float* out) {
  const int tid = threadIdx.x, lane = tid & 31;
  const uint32_t ufull = bars + 16 * kStages8, uempty = ufull + 8 * kSlots8;
  volatile int* stop = reinterpret_cast<volatile int*>(smem + Smem8::STOP);
  uint32_t base = 0;       // stages of earlier units
  bool segments = mode == 1, there = false;
  const Unit8* units = reinterpret_cast<const Unit8*>(smem + Smem8::UNITS);
  Tile8 t;
  // Unit k's queries, asked for while the unit before it is merged (its slot is filled by then, or soon: kSlots8).
  auto arrive_at = [&](int k) {
    there = __all_sync(0xffffffffu, wait_or_stop(ufull + 8 * (k % kSlots8), (k / kSlots8) & 1, stop));
    if (there) load_queries<G>(t, v, units[k % kSlots8], q, tid >> 5, lane >> 2, lane & 3);
  };
  arrive_at(0);
  for (int k = 0;; ++k) {
    const int slot = k % kSlots8;
    if (consumers_any(!there || *stop != 0)) {  // all leave together
      if (tid == 0) set_status(v.ctl, GB_ERR_TIMEOUT);
      return false;
    }
    const Unit8& u = units[slot];
    if (segments && u.kind != kUnitSegment) {  // this CTA's segment records are written
      if (tid == 0) {
        fence_acq_rel_gpu();
        atomicAdd(&cnt.c[kCntGrpDone], 1);
      }
      segments = false;
    }
    if (u.kind == kUnitEnd) return true;
    const bool done = multiply<G>(t, v, u, qscale, base, bars, smem, out, [&] { arrive_at(k + 1); });
    base += (u.tokens + 2 * kChunk - 1) / (2 * kChunk);
    if (tid == 0 && u.kind == kUnitBeam && done) {  // (a pair written at once is counted for zero_unwritten alone)
      if (!u.direct) fence_acq_rel_gpu();
      atomicAdd(&cnt.pair[u.members[0] * v.Hkv + u.head], 1);
    }
    __syncwarp();
    if (lane == 0) mbar_arrive_n(uempty + 8 * slot, 1);
  }
}

// A CTA gave up, with units that it had taken: zeros for every pair that was to be written at once and has not been.  (The
// others' merges give them zeros.)
template <int G>
__device__ void zero_unwritten(const PoolView& v, const Counters& cnt, int mode, const Shares& sh, float* out) {
  for (int p = threadIdx.x >> 5; p < v.max_beams * v.Hkv; p += kConsumers8) {
    const int b = p / v.Hkv, h = p - b * v.Hkv, n = v.active[b] ? plan_n(v, mode)[b] : 0;
    if (n == 0 || (mode == 1 && v.seg_nrec[b] > 0)) continue;
    const int o0 = plan_off(v, mode)[b] + h * n;
    if (sh.of(o0) == sh.of(o0 + n - 1) && ld_acquire_gpu(&cnt.pair[p]) == 0) zero_pair<G>(v, b, h, out);
  }
}

template <int G>
__global__ void __launch_bounds__(kThreads8, 1)
    k_decode8(PoolView v, const __grid_constant__ CUtensorMap tm, int layer, const __nv_bfloat16* q, float qscale, int mode, int stalled,
              float* __restrict__ out) {
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  unsigned char* smem = smem_raw + ((1024 - (smem_addr(smem_raw) & 1023)) & 1023);
  const int cta = (int)blockIdx.x, nctas = (int)gridDim.x, tid = threadIdx.x;
  const uint32_t bars = smem_addr(smem) + Smem8::BARS;
  if (tid < kStages8) {
    mbar_init(bars + 8 * tid, 2);
    mbar_init(bars + 8 * (kStages8 + tid), kConsumers8);
  }
  if (tid < kSlots8) {
    mbar_init(bars + 8 * (2 * kStages8 + tid), 1);
    mbar_init(bars + 8 * (2 * kStages8 + kSlots8 + tid), kConsumers8 + kLoaders8);
  }
  if (tid == 0) *reinterpret_cast<volatile int*>(smem + Smem8::STOP) = 0;
  if (tid < 32) fence_mbar_init();
  pdl_wait();
  pdl_launch_dependents();
  const int step_ok = v.ctl[kCtlStepOk], steps = v.ctl[kCtlSteps], nact = v.ctl[kCtlActive];
  if (step_ok == 0) {
    zero_all_pairs<G>(v, cta, nctas, out);
    return;
  }
  const int set = counter_set(v, layer, steps);
  const Counters cnt = counters(v, set);
  zero_counters(v, set ^ 1, cta, nctas);
  // mode 1: by segments; mode 2: by segments where that pays.  A segment's pages are read once for all of its members, but a
  // tile's step takes a warp as long for members as for a beam alone, and the records more to merge.  So it pays where beams of up
  // to 4 heads a KV head, two or more of which fill a tile that one would leave half empty, read far more than there is (us, beams
  // alone / segments; MB read alone / there): 99 / 93 (525 / 185, 64 x 4000), 242 / 186 (1600 / 673, 128 x 6100), 173 / 128 (1024 /
  // 369, 200 x 2500, G = 2), 228 / 187 (1660 / 554, 90 x 9000); not 72 / 80 (328 / 109, 40 x 4000), 88 / 93 (410 / 142, 100 x 2000), 132 /
  // 136 (577 / 188, 256 x 1100, on the wrong side), 238 / 280 (1623 / 359, 198 x 8000, G = 8).
  if (v.ctl[kCtlSegTiles] == 0) mode = 0;
  if (mode == 2) {
    const long long all = (long long)plan_off(v, 0)[v.max_beams] * kChunkBytes8;
    const long long there = plan_off(v, 1)[v.max_beams] * (long long)kChunkBytes8 + (long long)v.ctl[kCtlSegTok] * v.Hkv * (kChunkBytes8 / kChunk);
    mode = G <= 4 && all - there > 330000000ll ? 1 : 0;
  }
  {
    int* s_off = reinterpret_cast<int*>(smem + Smem8::PLAN);
    const int* off = plan_off(v, mode);
    const int* nn = plan_n(v, mode);
    for (int i = tid; i <= v.max_beams; i += kThreads8) {
      s_off[i] = off[i];
      s_off[i + kMaxBeams + 1] = i < v.max_beams ? nn[i] : 0;
    }
  }
  __syncthreads();
  const Shares sh = shares_of(v, mode, nact, reinterpret_cast<const int*>(smem + Smem8::PLAN)[v.max_beams], nctas);
  if (tid >> 5 >= kConsumers8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kLoaderRegs8));
    const int w = (tid >> 5) - kConsumers8;
    if (w == 0) plan_units<G>(v, cnt, mode, sh, smem, bars, tid & 31);
    else if (w <= kLoaders8) load_stages(v, &tm, layer, stalled, smem, bars, w - 1, tid & 31);
    return;
  }
  asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kConsumerRegs8));
  if (!multiply_units<G>(v, cnt, q, qscale, mode, smem, bars, out)) zero_unwritten<G>(v, cnt, mode, sh, out);
  // Every CTA is resident with the others (one an SM), and each wait gives up once the status is set.
  combine_shares<G, true>(v, cnt, mode, [sh](int x) { return sh.of(x); }, nctas, false, cta, nctas, kConsumers8, out);
}

template <int G>
cudaError_t launch_decode8_t(gb_pool* pool, int layer, const void* q, float scale, float* out, int mode, int stalled, cudaStream_t s) {
  cudaError_t e = set_max_dynamic_smem(reinterpret_cast<const void*>(k_decode8<G>), Smem8::TOTAL);
  if (e != cudaSuccess) return e;
  // With fewer registers at launch than its warps then share out the kernel would wait for ever.
  static std::atomic<bool> fits{false};
  if (!fits.load(std::memory_order_relaxed)) {
    cudaFuncAttributes a{};
    e = cudaFuncGetAttributes(&a, k_decode8<G>);
    if (e != cudaSuccess) return e;
    if (a.numRegs * kThreads8 < (kConsumers8 * kConsumerRegs8 + 4 * kLoaderRegs8) * 32) return cudaErrorInvalidConfiguration;
    fits.store(true, std::memory_order_relaxed);
  }
  prof_begin(pool, GB_PROF_DECODE, s);
  e = launch_pdl(k_decode8<G>, pool->num_sms, kThreads8, Smem8::TOTAL, s, pool->view,
                 *reinterpret_cast<const CUtensorMap*>(pool->dtmap), layer, static_cast<const __nv_bfloat16*>(q),
                 scale * 1.4426950408889634f, mode, stalled, out);
  prof_end(pool, GB_PROF_DECODE, s);
  pool->launches += 1;
  return e;
}

}  // namespace

cudaError_t launch_decode8(gb_pool* pool, int layer, const void* q, float scale, float* out, int mode, int stalled, cudaStream_t s) {
  switch (pool->view.G) {
    case 1: return launch_decode8_t<1>(pool, layer, q, scale, out, mode, stalled, s);
    case 2: return launch_decode8_t<2>(pool, layer, q, scale, out, mode, stalled, s);
    case 4: return launch_decode8_t<4>(pool, layer, q, scale, out, mode, stalled, s);
    case 8: return launch_decode8_t<8>(pool, layer, q, scale, out, mode, stalled, s);
  }
  return cudaErrorInvalidValue;
}

// The pool as rows of 128 bytes: dims {64 pairs of bytes, 16 rows, K|V, row groups of 16}, strides {128, Hkv P 128 (K slab
// to V slab), 2048} bytes.  The row groups end with the last K slab.
bool make_tensor_map8(gb_pool* pool) {
  const PoolView& v = pool->view;
  const unsigned long long slab = (unsigned long long)v.Hkv * v.P / 16, groups = (unsigned long long)v.layers * v.num_pages * 2 * slab;
  if (groups >= (1ull << 31)) return false;
  const cuuint64_t dims[4] = {64, 16, 2, groups - slab};
  const cuuint64_t strides[3] = {128, (cuuint64_t)v.Hkv * v.P * 128, 2048};
  const cuuint32_t box[4] = {64, 16, 2, 1};
  return pool->have_dtmap = encode_tensor_map(pool->dtmap, v.kv, 4, dims, strides, box);
}

}  // namespace gb
