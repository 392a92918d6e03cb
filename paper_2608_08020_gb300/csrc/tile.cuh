// Attention of one tile of 32 query rows over a run of keys on the CUDA cores, for 32-bit inputs of 64 dims: the
// tensor cores have no product of that precision.  One pass over the keys with the running maximum and
// sum of each row's softmax, 64 keys at a time:
//   S = scale' Q K^T,  m' = max(m, rowmax S),  P = 2^(S - m'),  l = l 2^(m - m') + rowsum P,
//   O = O 2^(m - m') + P V          (scale' = scale log2 e; all of it in fp32)
// Four teams of 128 threads take every fourth tile of keys, each with its own tiles and barriers, and are joined at the
// end: a tile is a chain of dependent steps (some 2000 instructions a warp), which sixteen warps cover for each other, and
// a long run of keys is four times shorter.  1100 keys by one team took 69 us, by two 64 us.
// A team's threads are 8 x 16; thread (y, x) owns rows 4y..4y+3, keys x, x + 16, x + 32, x + 48 of S and columns
// 4x..4x+3 of O, two fp32 operations to an instruction.  All tiles lie row by row in shared memory, 16 bytes
// apart in the banks, so a step of four dims (or keys) reads eight 16-byte pieces for 64 multiply-adds.  K's
// next tile comes while P V runs and V's while S does (cp.async).
#pragma once
#include "internal.cuh"
#include "ptx.cuh"

namespace gb {

constexpr int kTileRows = 32, kTileKeys = 64, kTileD = 64, kTileTeam = 128, kTileTeams = 4, kTileThreads = kTileTeams * kTileTeam;
constexpr int kTileLd = kTileD + 4;
struct TileTeam {
  float q[kTileRows][kTileLd];
  float k[kTileKeys][kTileLd];
  float v[kTileKeys][kTileLd];
  float p[kTileRows][kTileLd];  // [row][key]; at the end O
  float2 ml[kTileRows];
};
struct TileSmem {
  TileTeam team[kTileTeams];
};

// The keys a row sees: those below `limit`, and from `base` on those whose bit is set.
struct TileSees {
  int limit, base;
  unsigned long long bits;
  __device__ __forceinline__ bool operator()(int j) const {
    return j < limit || (j >= base && j - base < 64 && ((bits >> (j - base)) & 1));
  }
};

__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  unsigned long long r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;"
      : "=l"(r)
      : "l"(*reinterpret_cast<unsigned long long*>(&a)), "l"(*reinterpret_cast<unsigned long long*>(&b)),
        "l"(*reinterpret_cast<unsigned long long*>(&c)));
  return *reinterpret_cast<float2*>(&r);
}

// Src: q(r) the row's query or nullptr, key(j) and val(j) its rows or nullptr, sees(r), out(r, c, o, m, l): columns
// c..c+3 of the unnormalised sum with the row's maximum (base 2) and sum.
template <class Src>
__device__ __forceinline__ void tile_attention(TileSmem& both, const Src& src, int nkeys, float qscale) {
  const int team = threadIdx.x / kTileTeam, tid = threadIdx.x % kTileTeam, ty = tid >> 4, tx = tid & 15;
  TileTeam& sm = both.team[team];
  auto sync = [&]() { asm volatile("bar.sync %0, %1;" ::"r"(team + 1), "n"(kTileTeam) : "memory"); };
  // Two threads to a key's row, eight 16-byte pieces each; a row that is not there is zeros.
  auto load = [&](float (*to)[kTileLd], int j0, bool val) {
    const int j = tid >> 1, h = (tid & 1) * 32;
    const float* p = j0 + j < nkeys ? (val ? src.val(j0 + j) : src.key(j0 + j)) : nullptr;
    const uint32_t dst = static_cast<uint32_t>(__cvta_generic_to_shared(&to[j][h]));
    if (p) {
#pragma unroll
      for (int c = 0; c < 8; ++c)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst + 16 * c), "l"(p + h + 4 * c) : "memory");
    } else {
#pragma unroll
      for (int c = 0; c < 8; ++c) *reinterpret_cast<float4*>(&to[j][h + 4 * c]) = make_float4(0.f, 0.f, 0.f, 0.f);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  load(sm.k, team * kTileKeys, false);
  load(sm.v, team * kTileKeys, true);
  for (int i = tid; i < kTileRows * (kTileD / 4); i += kTileTeam) {
    const int r = i >> 4, c = (i & 15) * 4;
    const float* p = src.q(r);
    const float4 x = p ? *reinterpret_cast<const float4*>(p + c) : make_float4(0.f, 0.f, 0.f, 0.f);
    *reinterpret_cast<float4*>(&sm.q[r][c]) = make_float4(x.x * qscale, x.y * qscale, x.z * qscale, x.w * qscale);
  }
  TileSees sees[4];
  float2 o[4][2] = {};
  float m[4], l[4] = {};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    sees[i] = src.sees(4 * ty + i);
    m[i] = -INFINITY;
  }
  for (int j0 = team * kTileKeys; j0 < nkeys; j0 += kTileTeams * kTileKeys) {
    asm volatile("cp.async.wait_group 1;" ::: "memory");  // K of this tile
    sync();
    float2 acc[4][4] = {};  // even and odd dims
#pragma unroll 4
    for (int d = 0; d < kTileD; d += 4) {
      float4 a[4], b[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) a[i] = *reinterpret_cast<const float4*>(&sm.q[4 * ty + i][d]);
#pragma unroll
      for (int j = 0; j < 4; ++j) b[j] = *reinterpret_cast<const float4*>(&sm.k[tx + 16 * j][d]);
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          acc[i][j] = fma2(make_float2(a[i].x, a[i].y), make_float2(b[j].x, b[j].y), acc[i][j]);
          acc[i][j] = fma2(make_float2(a[i].z, a[i].w), make_float2(b[j].z, b[j].w), acc[i][j]);
        }
    }
    sync();  // K has been read
    if (j0 + kTileTeams * kTileKeys < nkeys) load(sm.k, j0 + kTileTeams * kTileKeys, false);
    else asm volatile("cp.async.commit_group;" ::: "memory");
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float s[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) s[j] = acc[i][j].x + acc[i][j].y;
      if (j0 + kTileKeys > min(nkeys, sees[i].limit)) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int key = j0 + tx + 16 * j;
          if (key >= nkeys || !sees[i](key)) s[j] = -INFINITY;
        }
      }
      float mt = fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]));
#pragma unroll
      for (int w = 8; w > 0; w >>= 1) mt = fmaxf(mt, __shfl_xor_sync(0xffffffffu, mt, w));
      const float mn = fmaxf(m[i], mt);
      const float ref = mn == -INFINITY ? 0.f : mn;  // no key seen yet: every p is 0
      const float alpha = exp2f(m[i] - ref);
      m[i] = mn;
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float p = ex2_approx(s[j] - ref);  // (2 ulp)
        sm.p[4 * ty + i][tx + 16 * j] = p;
        sum += p;
      }
      l[i] = l[i] * alpha + sum;  // this thread's keys; added over x at the end
#pragma unroll
      for (int c = 0; c < 2; ++c) o[i][c] = make_float2(o[i][c].x * alpha, o[i][c].y * alpha);
    }
    asm volatile("cp.async.wait_group 1;" ::: "memory");  // V of this tile
    sync();
#pragma unroll 4
    for (int j = 0; j < kTileKeys; j += 4) {
      float4 a[4], b[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) a[i] = *reinterpret_cast<const float4*>(&sm.p[4 * ty + i][j]);
#pragma unroll
      for (int e = 0; e < 4; ++e) b[e] = *reinterpret_cast<const float4*>(&sm.v[j + e][4 * tx]);
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float p = e == 0 ? a[i].x : e == 1 ? a[i].y : e == 2 ? a[i].z : a[i].w;
          o[i][0] = fma2(make_float2(p, p), make_float2(b[e].x, b[e].y), o[i][0]);
          o[i][1] = fma2(make_float2(p, p), make_float2(b[e].z, b[e].w), o[i][1]);
        }
    }
    sync();  // V and P have been read
    if (j0 + kTileTeams * kTileKeys < nkeys) load(sm.v, j0 + kTileTeams * kTileKeys, true);
    else asm volatile("cp.async.commit_group;" ::: "memory");
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
#pragma unroll
  for (int i = 0; i < 4; ++i) {
#pragma unroll
    for (int w = 8; w > 0; w >>= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], w);
    if (team > 0) {
      *reinterpret_cast<float4*>(&sm.p[4 * ty + i][4 * tx]) = make_float4(o[i][0].x, o[i][0].y, o[i][1].x, o[i][1].y);
      if (tx == 0) sm.ml[4 * ty + i] = make_float2(m[i], l[i]);
    }
  }
  __syncthreads();
  if (team > 0) return;
#pragma unroll 1
  for (int i = 0; i < 4; ++i) {
    const int row = 4 * ty + i, c = 4 * tx;
    float mm = m[0], ll = l[0];
    float2 x0 = o[0][0], x1 = o[0][1];
    TileSees see = sees[0];
#pragma unroll
    for (int e = 1; e < 4; ++e)  // (registers are not indexed)
      if (i == e) {
        mm = m[e];
        ll = l[e];
        x0 = o[e][0];
        x1 = o[e][1];
        see = sees[e];
      }
    float4 x = make_float4(x0.x, x0.y, x1.x, x1.y);
    for (int t = 1; t < kTileTeams; ++t) {
      const float2 ml = both.team[t].ml[row];
      const float4 y = *reinterpret_cast<const float4*>(&both.team[t].p[row][c]);
      const float mn = fmaxf(mm, ml.x), ref = mn == -INFINITY ? 0.f : mn, f0 = exp2f(mm - ref), f1 = exp2f(ml.x - ref);
      // (a team that saw no key of the row has summed 0 x V)
      auto join = [&](float p, float q) { return (f0 == 0.f ? 0.f : p * f0) + (f1 == 0.f ? 0.f : q * f1); };
      x = make_float4(join(x.x, y.x), join(x.y, y.y), join(x.z, y.z), join(x.w, y.w));
      ll = ll * f0 + ml.y * f1;
      mm = mn;
    }
    const float* qr = src.q(row);
    // P V takes every key of a tile, with p = 0 for those the row does not see, and 0 x inf is NaN: columns that are
    // not finite although the row's sum is, are summed again over the keys it sees.
    if (qr && isfinite(mm) && isfinite(ll) && !(isfinite(x.x) && isfinite(x.y) && isfinite(x.z) && isfinite(x.w))) {
      float again[4] = {};
      for (int j = 0; j < nkeys; ++j) {
        const float *k = see(j) ? src.key(j) : nullptr, *v = k ? src.val(j) : nullptr;
        if (!v) continue;
        float sc = 0.f;
        for (int d = 0; d < kTileD; ++d) sc = fmaf(qr[d] * qscale, k[d], sc);
        const float p = exp2f(sc - mm);
        for (int e = 0; e < 4; ++e) again[e] = fmaf(p, v[c + e], again[e]);
      }
      x = make_float4(again[0], again[1], again[2], again[3]);
    }
    src.out(row, c, x, mm, ll);
  }
}

}  // namespace gb
