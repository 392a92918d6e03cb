// Rows on their way into the cache and out of it: appending with a rotation, appending to and seeding pools of
// 8 bits, turning a step's queries and keys, reading a cache back.
#include <algorithm>

#include "rows.cuh"

namespace gb {
namespace {

// Warps that share a block of 16 positions, half of its rows each: a warp that holds all of them takes 160 registers.
constexpr int kBlockWarps = 2;
constexpr int kMine = kBlockRows / 2 / kBlockWarps;  // rows of a lane, one of each two that its warp takes at a time
constexpr int kCtaWarps = 8, kTeams = kCtaWarps / kBlockWarps;

// The rows t0 .. t0 + cnt - 1 of one block of 16 positions of some heads of K or V by kBlockWarps neighbouring warps: load, turn
// (K), round, store; the next head's rows are loaded meanwhile.  src: the first head's first row, `stride` bytes from one token to
// the next, heads 256 bytes apart; entry, prow: the block's page, read while the rows are on their way, and its first row there.
// 8 bits: a block that has rows before t0 keeps their scale, or has them rounded again where a new row does not fit it; red:
// [2][kCtaWarps] floats of the CTA, used in turn (*turn).
template <int DT, bool E8>
__device__ __forceinline__ void write_block(const PoolView& v, int layer, const int* entry, int kv, int h0, int heads, int prow,
                                            int t0, int cnt, const char* src, size_t stride, const RotationView& rot,
                                            float (*red)[kCtaWarps], int* turn) {
  constexpr int N = RowTraits<DT>::N;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, j = lane & 15, r0 = t0 & (kBlockRows - 1);
  const int mine = 2 * (warp % kBlockWarps), half = lane >> 4;   // this warp's first row, and its lanes' of it and the next
  auto row = [&](int i) { return 2 * kBlockWarps * i + mine + half; };
  uint4 ahead[kMine];
  src += (size_t)(mine + half) * stride + j * 16;
  auto load = [&]() {
#pragma unroll
    for (int i = 0; i < kMine; ++i)
      if (row(i) < cnt) ahead[i] = __ldcs(reinterpret_cast<const uint4*>(src + (size_t)(2 * kBlockWarps * i) * stride));
    src += 256;
  };
  load();
  const int page = *entry;
  if (page < 0 || page >= v.num_pages) {
    if (lane == 0) set_status(v.ctl, GB_ERR_INVALID);
    return;
  }
  const bool turns = kv == 0 && rot.table != nullptr;
  if (turns && t0 + cnt > rot.positions && lane == 0) set_status(v.ctl, GB_ERR_INVALID);
  unsigned char* dst = reinterpret_cast<unsigned char*>(v.kv) + kv_elem_offset(v, layer, page, kv, h0, prow) * (E8 ? 1 : v.esize);
  const size_t head_bytes = (size_t)v.P * (E8 ? 128 : 256);
  signed char* exponent = E8 ? v.kv_exp + exp_offset(v, layer, page, kv, h0, prow) : nullptr;
  const int head_blocks = v.P / kBlockRows;
  for (int h = 0; h < heads; ++h, dst += head_bytes, exponent += E8 ? head_blocks : 0) {
    if constexpr (!E8) {
      uint4 x[kMine];
#pragma unroll
      for (int i = 0; i < kMine; ++i) x[i] = ahead[i];
      if (h + 1 < heads) load();
#pragma unroll
      for (int i = 0; i < kMine; ++i) {
        if (row(i) - half >= cnt) break;
        const bool in = row(i) < cnt;
        if (turns) {
          float f[N];
          row_values<DT>(in ? x[i] : make_uint4(0u, 0u, 0u, 0u), f);
          turn_row<DT>(f, rot, in ? t0 + row(i) : -1);
          x[i] = row_bits<DT>(f);
        }
        if (in) *reinterpret_cast<uint4*>(dst + (r0 + row(i)) * 256 + j * 16) = x[i];
      }
    } else {
      static_assert(DT == GB_BF16, "rows of an 8-bit pool are given in bf16");
      const int was = r0 > 0 ? *exponent : kExpLeast;
      float f[kMine][N];
      float amax = 0.f;
#pragma unroll
      for (int i = 0; i < kMine; ++i) row_values<DT>(row(i) < cnt ? ahead[i] : make_uint4(0u, 0u, 0u, 0u), f[i]);
      if (h + 1 < heads) load();
#pragma unroll
      for (int i = 0; i < kMine; ++i) {
        if (turns && row(i) - half < cnt) turn_row<DT, false>(f[i], rot, row(i) < cnt ? t0 + row(i) : -1);
#pragma unroll
        for (int e = 0; e < N; ++e) amax = fmaxf(amax, fabsf(f[i][e]));  // (passes over NaN)
      }
      if (amax == INFINITY) {                            // e4m3 has no infinity: what is not finite is held as NaN
        amax = 0.f;
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
#pragma unroll
          for (int e = 0; e < N; ++e) {
            if (fabsf(f[i][e]) < INFINITY) amax = fmaxf(amax, fabsf(f[i][e]));
            else f[i][e] = __int_as_float(0x7fffffff);
          }
        }
      }
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
      if (lane == 0) red[*turn][warp] = amax;
      // (Every lane of these warps has read the block's exponent behind it, too.)
      asm volatile("bar.sync %0, %1;" ::"r"(1 + warp / kBlockWarps), "n"(32 * kBlockWarps) : "memory");
#pragma unroll
      for (int w = 0; w < kBlockWarps; ++w) amax = fmaxf(amax, red[*turn][warp / kBlockWarps * kBlockWarps + w]);
      *turn ^= 1;
      const int e = max(was, block_exponent(amax));
      if (r0 > 0 && e != was) {
        const float by = pow2i(was - e);
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
          if (row(i) >= r0) break;
          uint2* at = reinterpret_cast<uint2*>(dst + row(i) * 128 + 8 * j);
          uint2 c = *at;
          const float2 a0 = float2_of_f16x2(f16x2_of_e4m3x2(c.x)), a1 = float2_of_f16x2(f16x2_of_e4m3x2(c.x >> 16));
          const float2 b0 = float2_of_f16x2(f16x2_of_e4m3x2(c.y)), b1 = float2_of_f16x2(f16x2_of_e4m3x2(c.y >> 16));
          c.x = e4m3x4(a0.x * by, a0.y * by, a1.x * by, a1.y * by);
          c.y = e4m3x4(b0.x * by, b0.y * by, b1.x * by, b1.y * by);
          *at = c;
        }
      }
      const float by = pow2i(-e);
#pragma unroll
      for (int i = 0; i < kMine; ++i) {
        if (row(i) >= cnt) break;
        uint2 c;
        c.x = e4m3x4(f[i][0] * by, f[i][1] * by, f[i][2] * by, f[i][3] * by);
        c.y = e4m3x4(f[i][4] * by, f[i][5] * by, f[i][6] * by, f[i][7] * by);
        *reinterpret_cast<uint2*>(dst + (r0 + row(i)) * 128 + 8 * j) = c;
      }
      if (lane == 0 && mine == 0 && (r0 == 0 || e != was)) *exponent = (signed char)e;
    }
  }
}

// Two query rows of slot b (one a half warp) turned to position pos: the heads 2u, 2u + 1.
template <int DT>
__device__ __forceinline__ void turn_queries(const PoolView& v, const RotationView& rot, int b, int u, int pos,
                                             const uint4* q, uint4* qout) {
  const int head = 2 * u + ((threadIdx.x >> 4) & 1), j = threadIdx.x & 15;
  const bool in = head < v.Hq;
  const size_t at = ((size_t)b * v.Hq + head) * 16 + j;
  float f[RowTraits<DT>::N];
  row_values<DT>(in ? q[at] : make_uint4(0u, 0u, 0u, 0u), f);
  turn_row<DT>(f, rot, in ? pos : -1);
  if (in) qout[at] = row_bits<DT>(f);
}

// n_tokens new rows of every active slot at positions [seq_len - n_tokens, seq_len) of one layer, like k_append, but
// turned on the way, or held in 8 bits; and, with q, the slots' queries turned to the last of these positions.
// kin/vin: [n_tokens][max_beams][Hkv] rows of 256 bytes.  Two warps take a block of 16 positions of `heads` heads of
// K or V (heads divides Hkv), one after the other so that the rotation's table comes from L1.  256 slots x 199 tokens x 8 heads
// in 8 bits: 73 us (208 MB in, 104 out, 4.3 TB/s), 115 turned: 13 operations a value, half of the issue slots, 16 warps an SM.
template <int DT, bool E8>
__global__ void __launch_bounds__(32 * kCtaWarps, 2) k_append_rows(PoolView v, int layer, int n_tokens, int heads, RotationView rot, const char* kin,
                                                     const char* vin, const uint4* q, uint4* qout) {
  pdl_wait();
  pdl_launch_dependents();
  // Both counter sets of the attention launches: as in k_append.  (An attention launch of this layer may follow.)
  if (blockIdx.x == 0 && blockIdx.y == 0) {
    zero_counters(v, 0, 0, 1);
    zero_counters(v, 1, 0, 1);
  }
  if (v.ctl[kCtlStepOk] == 0) return;
  // Tail pages copied on write, as in k_append.  In 8 bits the copies are made by a launch before (k_cow_rows, all layers at
  // layer 0): the slot that keeps the page may round its rows again here.
  const int ncow = E8 ? 0 : v.ctl[kCtlCowJobs];
  const long long per_job = 2LL * v.Hkv * v.P * 16;
  const long long nthreads = (long long)gridDim.x * gridDim.y * blockDim.x;
  for (long long i = ((long long)blockIdx.y * gridDim.x + blockIdx.x) * blockDim.x + threadIdx.x; i < per_job * ncow;
       i += nthreads) {
    const int job = (int)(i / per_job);
    long long r = i % per_job;
    const int c = (int)(r & 15); r >>= 4;
    const int row = (int)(r % v.P); r /= v.P;
    const int head = (int)(r % v.Hkv), kv = (int)(r / v.Hkv);
    const int old = v.cow[3 * job], page = v.cow[3 * job + 1], have = v.cow[3 * job + 2];
    if (row >= have) continue;
    reinterpret_cast<uint4*>(v.kv + kv_elem_offset(v, layer, page, kv, head, row) * v.esize)[c] =
        reinterpret_cast<const uint4*>(v.kv + kv_elem_offset(v, layer, old, kv, head, row) * v.esize)[c];
  }
  __shared__ float red[2][kCtaWarps];
  const int warp = threadIdx.x >> 5, team = warp / kBlockWarps, parts = v.Hkv / heads;
  const int qunits = q != nullptr ? (v.Hq + 2 * kBlockWarps - 1) / (2 * kBlockWarps) : 0;
  int turn = 0;
  for (int b = blockIdx.x; b < v.max_beams; b += gridDim.x) {
    if (!v.active[b]) continue;
    const int L = v.seq_len[b], pos0 = L - n_tokens;
    if (pos0 < 0) continue;
    const int blk0 = pos0 / kBlockRows, blks = (L - 1) / kBlockRows - blk0 + 1;
    for (int u = (int)blockIdx.y * kTeams + team; u < blks * 2 * parts + qunits; u += (int)gridDim.y * kTeams) {
      if (u >= blks * 2 * parts) {
        turn_queries<DT>(v, rot, b, (u - blks * 2 * parts) * kBlockWarps + warp % kBlockWarps, L - 1, q, qout);
        continue;
      }
      const int kv = u >= blks * parts, w = u - (kv ? blks * parts : 0);  // (K first: it takes longer where it is turned)
      const int blk = blk0 + w / parts, h0 = w % parts * heads;
      const int t0 = max(pos0, blk * kBlockRows), cnt = min(L, (blk + 1) * kBlockRows) - t0;
      const int pi = blk * kBlockRows / v.P;
      const size_t stride = (size_t)v.max_beams * v.Hkv * 256;
      const char* src = (kv ? vin : kin) + (size_t)(t0 - pos0) * stride + ((size_t)b * v.Hkv + h0) * 256;
      write_block<DT, E8>(v, layer, v.tables + (size_t)b * v.max_pages + pi, kv, h0, heads, blk * kBlockRows - pi * v.P, t0, cnt,
                          src, stride, rot, red, &turn);
    }
  }
}

// A step's queries and keys turned to the step's position, into the pool's scratch (pools of bf16 and fp32, whose
// attention launch reads them there and writes the keys to the cache itself).  A warp takes two rows.
template <int DT>
__global__ void __launch_bounds__(256) k_turn(PoolView v, RotationView rot, const uint4* q, uint4* qout, const uint4* k, uint4* kout) {
  pdl_wait();
  pdl_launch_dependents();
  if (v.ctl[kCtlStepOk] == 0) return;
  const int qunits = (v.Hq + 1) / 2, units = qunits + (v.Hkv + 1) / 2;
  for (int i = (int)(blockIdx.x * blockDim.x + threadIdx.x) >> 5; i < v.max_beams * units; i += (int)(gridDim.x * blockDim.x) >> 5) {
    const int b = i / units, u = i - b * units;
    if (!v.active[b]) continue;
    const int pos = v.seq_len[b] - 1;
    if (pos >= rot.positions && (threadIdx.x & 31) == 0) set_status(v.ctl, GB_ERR_INVALID);
    if (u < qunits) {
      turn_queries<DT>(v, rot, b, u, pos, q, qout);
    } else {
      PoolView w = v;
      w.Hq = v.Hkv;
      turn_queries<DT>(w, rot, b, u - qunits, pos, k, kout);
    }
  }
}

// The prompt's K/V ([layer][T][Hkv] rows of 256 bytes) into the 8-bit pages of slot 0's table.
__global__ void __launch_bounds__(32 * kCtaWarps, 2) k_seed_rows8(PoolView v, int T, const char* kp, const char* vp) {
  pdl_wait();
  pdl_launch_dependents();
  __shared__ float red[2][kCtaWarps];
  int turn = 0;
  const int blks = (T + kBlockRows - 1) / kBlockRows;
  const long long units = (long long)v.layers * blks * 2;
  for (long long u = (long long)blockIdx.x * kTeams + (threadIdx.x >> 5) / kBlockWarps; u < units; u += (long long)gridDim.x * kTeams) {
    const int layer = (int)(u / (2 * blks)), r = (int)(u % (2 * blks));
    const int kv = r & 1, t0 = (r >> 1) * kBlockRows;
    const size_t stride = (size_t)v.Hkv * 256;
    write_block<GB_BF16, true>(v, layer, v.tables + t0 / v.P, kv, 0, v.Hkv, t0 % v.P, t0, min(kBlockRows, T - t0),
                               (kv ? vp : kp) + ((size_t)layer * T + t0) * stride, stride, RotationView{}, red, &turn);
  }
}

// Tokens first[b] .. first[b] + n - 1 of every slot as the cache holds them, in the type that rows are given in;
// zeros where a slot has no such token.  A warp takes a block of 16 positions of a (K|V, head), two rows at a time: memory, 256
// slots x 199 tokens x 8 heads of 8 bits in 52 us (6.0 TB/s; 16 bytes a thread, with a page lookup each, took 165).
template <bool E8>
__global__ void __launch_bounds__(256) k_read_kv(PoolView v, int layer, const int* first, int n, uint4* kout, uint4* vout) {
  pdl_wait();
  pdl_launch_dependents();
  const int warp = threadIdx.x >> 5, nw = (int)blockDim.x >> 5, pairs = 2 * v.Hkv, half = (threadIdx.x >> 4) & 1, j = threadIdx.x & 15;
  for (int b = blockIdx.x; b < v.max_beams; b += gridDim.x) {
    const int L = v.active[b] ? v.seq_len[b] : 0;
    const long long from = first[b], end = from + n;
    const long long blk0 = from >> 4;                  // (from < 0: rounded down)
    const int blks = (int)(((end - 1) >> 4) - blk0 + 1);
    for (long long u = blockIdx.y * nw + warp; u < (long long)blks * pairs; u += gridDim.y * nw) {
      const long long blk = blk0 + u / pairs;
      const int kv = (int)(u % pairs) / v.Hkv, h = (int)(u % pairs) % v.Hkv;
      const long long t0 = max(from, blk * kBlockRows);
      const int cnt = (int)(min(end, (blk + 1) * kBlockRows) - t0);
      int have = 0, page = 0, prow = 0;                // rows of the block that the cache has
      if (t0 >= 0 && t0 < L) {
        page = v.tables[(size_t)b * v.max_pages + t0 / v.P];
        prow = (int)(t0 % v.P);
        have = min(cnt, L - (int)t0);
        if (page < 0 || page >= v.num_pages) {
          have = 0;
          if ((threadIdx.x & 31) == 0) set_status(v.ctl, GB_ERR_INVALID);
        }
      }
      const size_t stride = (size_t)v.max_beams * v.Hkv * 16;
      uint4* dst = (kv ? vout : kout) + (size_t)(t0 - from) * stride + ((size_t)b * v.Hkv + h) * 16 + j;
      const char* src = v.kv + kv_elem_offset(v, layer, page, kv, h, prow) * v.esize;
      if constexpr (E8) {
        uint2 c[kBlockRows / 2];
#pragma unroll
        for (int i = 0; i < kBlockRows / 2; ++i)
          c[i] = 2 * i + half < have ? *reinterpret_cast<const uint2*>(src + (2 * i + half) * 128 + 8 * j) : make_uint2(0u, 0u);
        const float by = have > 0 ? pow2i(v.kv_exp[exp_offset(v, layer, page, kv, h, prow)]) : 0.f;
#pragma unroll
        for (int i = 0; i < kBlockRows / 2; ++i) {
          const uint32_t w[4] = {c[i].x & 0xffffu, c[i].x >> 16, c[i].y & 0xffffu, c[i].y >> 16};
          float f[8];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float2 g = float2_of_f16x2(f16x2_of_e4m3x2(w[e]));
            f[2 * e] = g.x * by;
            f[2 * e + 1] = g.y * by;
          }
          if (2 * i + half < cnt) __stcs(dst + (2 * i + half) * stride, row_bits<GB_BF16>(f));
        }
      } else {
        uint4 x[kBlockRows / 2];
#pragma unroll
        for (int i = 0; i < kBlockRows / 2; ++i)
          x[i] = 2 * i + half < have ? *(reinterpret_cast<const uint4*>(src + (2 * i + half) * 256) + j) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
        for (int i = 0; i < kBlockRows / 2; ++i)
          if (2 * i + half < cnt) __stcs(dst + (2 * i + half) * stride, x[i]);
      }
    }
  }
}

}  // namespace

// Appends n_tokens rows of a layer through k_append_rows; q, qout: the queries to turn, or nullptr.
cudaError_t launch_append_rows(gb_pool* pool, int layer, int n_tokens, const RotationView& rot, const void* k, const void* vv,
                               const void* q, void* qout, cudaStream_t s) {
  const PoolView& v = pool->view;
  const int blks = (n_tokens + 2 * kBlockRows - 2) / kBlockRows;  // at most, of a slot
  // Heads one after the other where there are blocks enough without (two CTAs an SM), else side by side.
  int heads = v.Hkv;
  while (heads % 2 == 0 && (long long)blks * v.max_beams * 2 * (v.Hkv / heads) < (long long)kTeams * 2 * pool->num_sms) heads /= 2;
  if ((long long)blks * v.max_beams * 2 * (v.Hkv / heads) < (long long)kTeams * 2 * pool->num_sms) heads = 1;
  const long long units = (long long)blks * 2 * (v.Hkv / heads) + (q ? (v.Hq + 2 * kBlockWarps - 1) / (2 * kBlockWarps) : 0);
  const dim3 grid(v.max_beams, (unsigned)std::min((units + kTeams - 1) / kTeams, 65535ll));
  pool->launches += 1;
  const char *kc = static_cast<const char*>(k), *vc = static_cast<const char*>(vv);
  const uint4* qc = static_cast<const uint4*>(q);
  uint4* qo = static_cast<uint4*>(qout);
  switch (v.dtype) {
    case GB_FP8: return launch_pdl(k_append_rows<GB_BF16, true>, grid, 32 * kCtaWarps, 0, s, v, layer, n_tokens, heads, rot, kc, vc, qc, qo);
    case GB_BF16: return launch_pdl(k_append_rows<GB_BF16, false>, grid, 32 * kCtaWarps, 0, s, v, layer, n_tokens, heads, rot, kc, vc, qc, qo);
    default: return launch_pdl(k_append_rows<GB_F32, false>, grid, 32 * kCtaWarps, 0, s, v, layer, n_tokens, heads, rot, kc, vc, qc, qo);
  }
}

cudaError_t launch_turn(gb_pool* pool, const RotationView& rot, const void* q, void* qout, const void* k, void* kout, cudaStream_t s) {
  const PoolView& v = pool->view;
  const int units = v.max_beams * ((v.Hq + 1) / 2 + (v.Hkv + 1) / 2);
  const int grid = std::min((units + 7) / 8, 8 * pool->num_sms);
  pool->launches += 1;
  return launch_pdl(v.dtype == GB_F32 ? k_turn<GB_F32> : k_turn<GB_BF16>, grid, 256, 0, s, v, rot, static_cast<const uint4*>(q),
                    static_cast<uint4*>(qout), static_cast<const uint4*>(k), static_cast<uint4*>(kout));
}

cudaError_t launch_seed_rows8(gb_pool* pool, int prompt_len, const void* k, const void* vv, cudaStream_t s) {
  const PoolView& v = pool->view;
  const long long units = (long long)v.layers * ((prompt_len + kBlockRows - 1) / kBlockRows) * 2;
  const int grid = (int)std::min((units + kTeams - 1) / kTeams, 8ll * pool->num_sms);
  k_seed_rows8<<<grid, 32 * kCtaWarps, 0, s>>>(v, prompt_len, static_cast<const char*>(k), static_cast<const char*>(vv));
  return cudaGetLastError();
}

}  // namespace gb

using namespace gb;

extern "C" gb_status gb_read_kv(gb_pool* pool, int layer, const int32_t* first_dev, int n_tokens, void* k_out_dev,
                                void* v_out_dev, gb_stream_t stream) {
  if (!pool) return GB_ERR_INVALID;
  if (layer < 0 || layer >= pool->cfg.num_layers || n_tokens < 0 || !first_dev || !k_out_dev || !v_out_dev ||
      (((uintptr_t)k_out_dev | (uintptr_t)v_out_dev) & 15))
    return fail(pool, GB_ERR_INVALID, "read_kv: bad arguments");
  if (!on_device(pool)) return fail(pool, GB_ERR_STATE, "read_kv: the pool is on another device than the current one");
  if (!pool->seeded) return fail(pool, GB_ERR_STATE, "pool not seeded");
  if (pool->next_layer != 0) return fail(pool, GB_ERR_STATE, "read_kv inside an open step");
  if (n_tokens == 0) return GB_OK;
  const PoolView& v = pool->view;
  const long long units = 2ll * ((n_tokens + 2ll * kBlockRows - 2) / kBlockRows) * v.Hkv;   // at most, of a slot
  const long long most = std::max(1ll, (8ll * pool->num_sms + v.max_beams - 1) / v.max_beams);
  const dim3 grid(v.max_beams, (unsigned)std::min(std::min((units + 7) / 8, most), 65535ll));
  launch_pdl(v.dtype == GB_FP8 ? k_read_kv<true> : k_read_kv<false>, grid, 256, 0, reinterpret_cast<cudaStream_t>(stream), v, layer,
             first_dev, n_tokens, static_cast<uint4*>(k_out_dev), static_cast<uint4*>(v_out_dev));
  pool->launches += 1;
  return check_launch(pool, "read_kv");
}
