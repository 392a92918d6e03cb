// Decode attention over pools held in 8 bits.
//
//   out[b][h] = sum_t softmax_t(scale q . k_t) v_t,   k_t = 2^(e_K) c_t,  v_t = 2^(e_V) d_t
// with one e_K and one e_V for each chunk of 16 tokens of a head (rows.cuh).  A chunk is 4 KiB, K and V, brought by one
// TMA into a warp's ring of stages; its codes become pairs of fp16 in registers (exact) on their way into m16n8k16
// products, the G query heads of the KV head being the N = 8 columns:
//   S^T[16 tokens][8] = C Q'^T,   s = scale' 2^(e_K) S     (Q' = q times a power of two that brings a row below 2^15: exact
//                                                           for a bf16 row but for values 2^-39 of its largest)
//   O^T[128][8]      += D^T P^T
// A chunk's e_V goes into the exponent of its weights: with t = s + e_V and a running maximum m of the t,
//   p = 2^(t - m),   O += p d,   L += 2^(-e_V) p
// so that the largest contribution to O has a weight near one whatever the blocks' scales, and out = O / L.  p enters the
// products as two fp16 terms (22 bits): one term would be the largest error of the whole by a factor of 100.
// m is set 7 below the largest t of a chunk, and raised only when a chunk exceeds it by more than 15: p stays under
// fp16's 2^16, and the last place of a small p (2^-24) is 2^-31 of the largest.
//
// Fragments are chosen so that a lane's operands are 16-byte pieces: the dims (the k of S) and the dims of O^T's rows
// are permuted, which the queries and the output follow.  Lane (r = lane / 4, c = lane % 4) reads dims 32c .. 32c + 31 of
// tokens r, r + 8 of K, and dims 16r .. 16r + 15 of tokens 2c, 2c + 1, 2c + 8, 2c + 9 of V, whose codes are
// interleaved in pairs by byte permutes: 8 loads, 64 conversions, 16 permutes, 24 products a chunk.
#include "decode_mma.cuh"
#include "rows.cuh"

namespace gb {
namespace {

constexpr int kWarps8 = 12;
constexpr int kStages8 = 4;
constexpr int kStageBytes8 = 2 * kChunk * 128;
struct Smem8 {
  static constexpr int STAGES = kWarps8 * kStages8 * kStageBytes8;
  static constexpr int BARS = kWarps8 * kStages8 * 8;
  static constexpr int PLAN = 4 * (kMaxBeams + 1) * 4;  // offsets, chunk counts, start tokens, lengths
  static constexpr int TOTAL = 1024 + STAGES + BARS + PLAN;
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
  float o[8][4];     // O^T: dims 16r + 2i of columns 2c, 2c + 1, then dims 16r + 2i + 1
  float m0, m1, l0, l1;
};

// row: this lane's query row (128 bf16), or nullptr for a column without one.
__device__ __forceinline__ void tile_begin(Tile8& t, const __nv_bfloat16* row, float qscale, int c) {
  uint32_t w[16];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint4 x = row ? *reinterpret_cast<const uint4*>(row + 32 * c + 8 * i) : make_uint4(0u, 0u, 0u, 0u);
    w[4 * i] = x.x;
    w[4 * i + 1] = x.y;
    w[4 * i + 2] = x.z;
    w[4 * i + 3] = x.w;
  }
  float amax = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const float a = fabsf(__uint_as_float(w[i] << 16)), b = fabsf(__uint_as_float(w[i] & 0xffff0000u));
    amax = fmaxf(amax, a <= 3.4e38f ? a : 0.f);
    amax = fmaxf(amax, b <= 3.4e38f ? b : 0.f);
  }
  amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
  amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
  // 2^sh brings the largest value into [2^14, 2^15); in two factors, as sh may pass fp32's exponents.
  const int ex = (int)(__float_as_uint(amax) >> 23) - 127, sh = min(max(14 - ex, -113), 126);
  const float up = pow2i(sh);
#pragma unroll
  for (int i = 0; i < 16; ++i)
    t.q[i >> 1][i & 1] = pack_f16x2(__uint_as_float(w[i] << 16) * up, __uint_as_float(w[i] & 0xffff0000u) * up);
  const float back = qscale * pow2i(-sh);
  t.s0 = __shfl_sync(0xffffffffu, back, 8 * c);      // row 2c's first lane
  t.s1 = __shfl_sync(0xffffffffu, back, 8 * c + 4);
#pragma unroll
  for (int i = 0; i < 8; ++i) t.o[i][0] = t.o[i][1] = t.o[i][2] = t.o[i][3] = 0.f;
  t.m0 = t.m1 = -INFINITY;
  t.l0 = t.l1 = 0.f;
}

// A landed chunk (its first nvalid >= 1 tokens) into NT tiles.  ek, ev: its exponents.
template <int NT>
__device__ __forceinline__ void chunk_attend8(Tile8 (&t)[NT], uint32_t sb, int nvalid, int ek, int ev, int r, int c) {
  uint32_t w[2][8];  // K words: tokens r, r + 8; dims 32c + 4j .. + 3
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int z = 0; z < 2; ++z) {
      const uint4 x = ld_shared16(sb + (r + 8 * i) * 128 + (((2 * c + z) ^ r) << 4));
      w[i][4 * z] = x.x;
      w[i][4 * z + 1] = x.y;
      w[i][4 * z + 2] = x.z;
      w[i][4 * z + 3] = x.w;
    }
  float s[NT][2][4];
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int e = 0; e < 4; ++e) s[n][0][e] = s[n][1][e] = 0.f;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const uint32_t a0 = f16x2_of_e4m3x2(w[0][j]), a1 = f16x2_of_e4m3x2(w[1][j]);
    const uint32_t a2 = f16x2_of_e4m3x2(w[0][j] >> 16), a3 = f16x2_of_e4m3x2(w[1][j] >> 16);
#pragma unroll
    for (int n = 0; n < NT; ++n) mma_f16(s[n][j & 1], a0, a1, a2, a3, t[n].q[j][0], t[n].q[j][1]);
  }
  uint4 x[4];  // V pieces of tokens 2c, 2c + 1, 2c + 8, 2c + 9
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int tok = 2 * c + (i & 1) + 8 * (i >> 1);
    x[i] = ld_shared16(sb + kChunk * 128 + tok * 128 + ((r ^ (tok & 7)) << 4));
    if (nvalid < kChunk && tok >= nvalid) x[i] = make_uint4(0u, 0u, 0u, 0u);  // whatever the page holds there
  }
  const float kscale = pow2i(ek), vback = pow2i(-ev), vexp = (float)ev;
  uint32_t hi[NT][2], lo[NT][2];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    Tile8& u = t[n];
    const float k0 = u.s0 * kscale, k1 = u.s1 * kscale;
    float y[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = fmaf(s[n][0][e] + s[n][1][e], e & 1 ? k1 : k0, vexp);
    if (nvalid < kChunk) {
      if (r >= nvalid) y[0] = y[1] = -INFINITY;
      if (r + 8 >= nvalid) y[2] = y[3] = -INFINITY;
    }
    float mx0 = fmaxf(y[0], y[2]), mx1 = fmaxf(y[1], y[3]);
#pragma unroll
    for (int o = 4; o < 32; o <<= 1) {
      mx0 = fmaxf(mx0, __shfl_xor_sync(0xffffffffu, mx0, o));
      mx1 = fmaxf(mx1, __shfl_xor_sync(0xffffffffu, mx1, o));
    }
    const bool up0 = mx0 > u.m0 + 15.f, up1 = mx1 > u.m1 + 15.f;
    if (__any_sync(0xffffffffu, up0 || up1)) {
      const float n0 = up0 ? mx0 - 7.f : u.m0, n1 = up1 ? mx1 - 7.f : u.m1;
      const float f0 = up0 ? ex2_approx(u.m0 - n0) : 1.f, f1 = up1 ? ex2_approx(u.m1 - n1) : 1.f;
      u.m0 = n0;
      u.m1 = n1;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        u.o[i][0] *= f0;
        u.o[i][1] *= f1;
        u.o[i][2] *= f0;
        u.o[i][3] *= f1;
      }
      u.l0 *= f0;
      u.l1 *= f1;
    }
    const float p0 = ex2_approx(y[0] - u.m0), p1 = ex2_approx(y[1] - u.m1);
    const float p2 = ex2_approx(y[2] - u.m0), p3 = ex2_approx(y[3] - u.m1);
    u.l0 = fmaf(p0 + p2, vback, u.l0);
    u.l1 = fmaf(p1 + p3, vback, u.l1);
    const uint32_t h0 = pack_f16x2(p0, p1), h1 = pack_f16x2(p2, p3);
    const float2 g0 = float2_of_f16x2(h0), g1 = float2_of_f16x2(h1);
    hi[n][0] = movmatrix_t(h0);
    hi[n][1] = movmatrix_t(h1);
    lo[n][0] = movmatrix_t(pack_f16x2(p0 - g0.x, p1 - g0.y));
    lo[n][1] = movmatrix_t(pack_f16x2(p2 - g1.x, p3 - g1.y));
  }
  const uint32_t* v0 = &x[0].x;
  const uint32_t* v1 = &x[1].x;
  const uint32_t* v2 = &x[2].x;
  const uint32_t* v3 = &x[3].x;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t sel = i & 1 ? 0x7362 : 0x5140;
    const uint32_t a = __byte_perm(v0[i >> 1], v1[i >> 1], sel), b = __byte_perm(v2[i >> 1], v3[i >> 1], sel);
    const uint32_t a0 = f16x2_of_e4m3x2(a), a1 = f16x2_of_e4m3x2(a >> 16);
    const uint32_t a2 = f16x2_of_e4m3x2(b), a3 = f16x2_of_e4m3x2(b >> 16);
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      mma_f16(t[n].o[i], a0, a1, a2, a3, hi[n][0], hi[n][1]);
      mma_f16(t[n].o[i], a0, a1, a2, a3, lo[n][0], lo[n][1]);
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

// Column 2c + z's record or output: 16 floats at `to` + 16 r.
__device__ __forceinline__ void tile_store(const Tile8& t, float* to, int z, float by, uint64_t pol) {
#pragma unroll
  for (int i = 0; i < 8; i += 2)
    st_hint4(to + 2 * i, make_float4(t.o[i][z] * by, t.o[i][z + 2] * by, t.o[i + 1][z] * by, t.o[i + 1][z + 2] * by), pol);
}

// The flat list of (beam, KV head, chunk) units, an even share for every warp (decode_mma.cuh); records are merged
// in the launch (combine.cuh).
template <int G>
__global__ void __launch_bounds__(kWarps8 * 32, 1)
    k_decode8(PoolView v, const __grid_constant__ CUtensorMap tm, int layer, const __nv_bfloat16* q, float qscale, int mode,
              float* __restrict__ out) {
  pdl_wait();
  pdl_launch_dependents();
  using S = Smem8;
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  unsigned char* smem = smem_raw + ((1024 - (smem_addr(smem_raw) & 1023)) & 1023);
  const int cta = (int)blockIdx.x, nctas = (int)gridDim.x;
  const int step_ok = v.ctl[kCtlStepOk], steps = v.ctl[kCtlSteps];
  if (step_ok == 0) {
    zero_all_pairs<G>(v, cta, nctas, out);
    return;
  }
  const int set = counter_set(v, layer, steps);
  const Counters cnt = counters(v, set);
  zero_counters(v, set ^ 1, cta, nctas);
  int* s_off = reinterpret_cast<int*>(smem + S::STAGES + S::BARS);
  int* s_n = s_off + (kMaxBeams + 1);
  int* s_start = s_n + (kMaxBeams + 1);
  int* s_len = s_start + (kMaxBeams + 1);
  {
    const int* off = plan_off(v, mode);
    const int* nn = plan_n(v, mode);
    const int* st = plan_start(v, mode);
    for (int i = threadIdx.x; i <= v.max_beams; i += blockDim.x) {
      s_off[i] = off[i];
      s_n[i] = i < v.max_beams ? nn[i] : 0;
      s_start[i] = i < v.max_beams ? st[i] : 0;
      s_len[i] = i < v.max_beams ? v.seq_len[i] : 0;
    }
  }
  __syncthreads();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, r = lane >> 2, c = lane & 3;
  const uint32_t stage0 = smem_addr(smem) + warp * kStages8 * kStageBytes8;
  const uint32_t bar0 = smem_addr(smem) + S::STAGES + warp * kStages8 * 8;
  const int W = nctas * kWarps8, w = cta * kWarps8 + warp, Tot = s_off[v.max_beams];
  const int cw = (Tot + W - 1) / W;
  const int x_begin = min(Tot, w * cw), x_end = min(Tot, x_begin + cw);
  if (x_begin < x_end) {
    if (lane == 0) {
      for (int s = 0; s < kStages8; ++s) mbar_init(bar0 + 8 * s, 1);
      fence_mbar_init();
    }
    __syncwarp();
    ChunkIter it;
    {
      int lo = 0, hi = v.max_beams;  // invariant: s_off[lo] <= x < s_off[hi]
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (s_off[mid] <= x_begin) lo = mid; else hi = mid;
      }
      it.b = lo;
      it.n = s_n[lo];
      it.tok0 = s_start[lo];
      const int rr = x_begin - s_off[lo];
      it.h = rr / it.n;
      it.i = rr % it.n;
    }
    const bool reread = mode == 0 && v.ctl[kCtlSegCount] > 0;
    const uint64_t pol = reread || !v.grouped ? policy_evict_normal() : policy_evict_first();
    int pw_b = -1, pw_i0 = 0, pw_lane = 0;
    auto load_page = [&](const ChunkIter& qi) -> int {
      if (qi.b != pw_b || qi.i < pw_i0 || qi.i >= pw_i0 + 32) {
        pw_b = qi.b;
        pw_i0 = qi.i;
        const int i = pw_i0 + lane;
        pw_lane = i >= qi.n ? 0 : v.tables[(size_t)qi.b * v.max_pages + (qi.tok0 + i * kChunk) / v.P];
      }
      return __shfl_sync(0xffffffffu, pw_lane, qi.i - pw_i0);
    };
    const int pg = v.P / kChunk;
    const long long layer_pages = (long long)layer * v.num_pages;
    const size_t kv_gap = (size_t)v.Hkv * pg;  // exponents from K to V
    // Loads of the chunk at `qi` into a stage; lanes 0 and 1 of every warp also fetch its exponents, which wait in
    // registers (`ex`, a slot a stage).
    int ex[kStages8];
    auto issue = [&](const ChunkIter& qi, int page, int stage) -> int {
      if (page < 0 || page >= v.num_pages) {
        if (lane == 0) set_status(v.ctl, GB_ERR_INVALID);
        page = 0;
      }
      const int tok = qi.tok0 + qi.i * kChunk;
      const long long g = ((layer_pages + page) * 2 * v.Hkv + qi.h) * pg + (tok & (v.P - 1)) / kChunk;
      if (lane == 0) {
        mbar_arrive_expect_tx(bar0 + 8 * stage, kStageBytes8);
        tma_chunk8(stage0 + stage * kStageBytes8, &tm, (int)g, bar0 + 8 * stage, pol);
      }
      return lane < 2 ? v.kv_exp[g + lane * (long long)kv_gap] : 0;
    };
    ChunkIter ip = it;
    int ip_x = x_begin, ip_page = load_page(ip);
#pragma unroll
    for (int s = 0; s < kStages8; ++s) {
      ex[s] = 0;
      if (ip_x < x_end) {
        ex[s] = issue(ip, ip_page, s);
        ++ip_x;
        if (ip_x < x_end) {
          iter_advance(ip, s_n, s_start, v.Hkv, v.max_beams);
          ip_page = load_page(ip);
        }
      }
    }
    Tile8 t[1];
    bool fresh = true, alive = true;
    uint32_t parity = 0;
    for (int x0 = x_begin; x0 < x_end && alive; x0 += kStages8, parity ^= 1u) {
#pragma unroll
      for (int s = 0; s < kStages8; ++s) {
        const int x = x0 + s;
        if (x >= x_end || !alive) break;
        if (fresh) {
          tile_begin(t[0], r < G ? q + ((size_t)it.b * v.Hq + it.h * G + r) * 128 : nullptr, qscale, c);
          fresh = false;
        }
        if (!mbar_wait_bounded(bar0 + 8 * s, parity, kWaitLimitNs)) {
          if (lane == 0) set_status(v.ctl, GB_ERR_TIMEOUT);
          for (int z = 1; z < kStages8; ++z)  // a bounded chance for the copies in flight
            if (x + z < ip_x) mbar_wait_bounded(bar0 + 8 * ((s + z) % kStages8), parity ^ (s + z >= kStages8 ? 1u : 0u), kWaitLimitNs / 4);
          alive = false;
          break;
        }
        const int nvalid = min(kChunk, s_len[it.b] - (it.tok0 + it.i * kChunk));
        chunk_attend8<1>(t, stage0 + s * kStageBytes8, nvalid, __shfl_sync(0xffffffffu, ex[s], 0),
                         __shfl_sync(0xffffffffu, ex[s], 1), r, c);
        __syncwarp();
        if (ip_x < x_end) {
          if (lane == 0) fence_proxy_async_smem();
          ex[s] = issue(ip, ip_page, s);
          ++ip_x;
          if (ip_x < x_end) {
            iter_advance(ip, s_n, s_start, v.Hkv, v.max_beams);
            ip_page = load_page(ip);
          }
        }
        if (it.i == it.n - 1 || x + 1 == x_end) {
          tile_finish(t[0]);
          float* rec = v.partials + (size_t)(w + it.b * v.Hkv + it.h) * v.record_floats;
          const uint64_t rpol = policy_evict_last();
#pragma unroll
          for (int z = 0; z < 2; ++z)
            if (2 * c + z < G) {
              tile_store(t[0], rec + (2 * c + z) * 128 + 16 * r, z, 1.f, rpol);
              if (r == 0) {
                st_hint(rec + G * 128 + 2 * c + z, z ? t[0].m1 : t[0].m0, rpol);
                st_hint(rec + G * 128 + G + 2 * c + z, z ? t[0].l1 : t[0].l0, rpol);
              }
            }
          record_arrive(cnt, it.b * v.Hkv + it.h, lane);
          fresh = true;
        }
        if (x + 1 < x_end) iter_advance(it, s_n, s_start, v.Hkv, v.max_beams);
      }
    }
  }
  combine_pairs<G>(v, cnt, mode, W, 0, false, cta, nctas, out);
}

template <int G>
cudaError_t launch_decode8_t(gb_pool* pool, int layer, const void* q, float scale, float* out, int mode, cudaStream_t s) {
  cudaError_t e = set_max_dynamic_smem(reinterpret_cast<const void*>(k_decode8<G>), Smem8::TOTAL);
  if (e != cudaSuccess) return e;
  prof_begin(pool, GB_PROF_DECODE, s);
  e = launch_pdl(k_decode8<G>, pool->num_sms, kWarps8 * 32, Smem8::TOTAL, s, pool->view,
                 *reinterpret_cast<const CUtensorMap*>(pool->dtmap), layer, static_cast<const __nv_bfloat16*>(q),
                 scale * 1.4426950408889634f, mode, out);
  prof_end(pool, GB_PROF_DECODE, s);
  pool->launches += 1;
  return e;
}

}  // namespace

cudaError_t launch_decode8(gb_pool* pool, int layer, const void* q, float scale, float* out, int mode, cudaStream_t s) {
  switch (pool->view.G) {
    case 1: return launch_decode8_t<1>(pool, layer, q, scale, out, mode, s);
    case 2: return launch_decode8_t<2>(pool, layer, q, scale, out, mode, s);
    case 4: return launch_decode8_t<4>(pool, layer, q, scale, out, mode, s);
    case 8: return launch_decode8_t<8>(pool, layer, q, scale, out, mode, s);
  }
  return cudaErrorInvalidValue;
}

// The pool as rows of 128 bytes: dims {64 pairs of bytes, 16 rows, K|V, row groups of 16}, strides {128, Hkv P 128 (K slab
// to V slab), 2048} bytes.  The row groups end with the last K slab.
bool make_tensor_map8(gb_pool* pool) {
  const PoolView& v = pool->view;
  const unsigned long long slab = (unsigned long long)v.Hkv * v.P / 16, groups = (unsigned long long)v.layers * v.num_pages * 2 * slab;
  if (groups >= (1ull << 31) || pool->num_sms * kWarps8 > kMaxDecodeWarps) return false;
  const cuuint64_t dims[4] = {64, 16, 2, groups - slab};
  const cuuint64_t strides[3] = {128, (cuuint64_t)v.Hkv * v.P * 128, 2048};
  const cuuint32_t box[4] = {64, 16, 2, 1};
  return pool->have_dtmap = encode_tensor_map(pool->dtmap, v.kv, 4, dims, strides, box);
}

}  // namespace gb
