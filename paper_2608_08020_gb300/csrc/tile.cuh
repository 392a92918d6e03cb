// Attention of one tile of 64 query rows over a run of keys on the CUDA cores, for 32-bit inputs: the
// tensor cores have no product of that precision.  One pass over the keys with the running maximum and
// sum of each row's softmax, 64 keys at a time:
//   S = scale' Q K^T,  m' = max(m, rowmax S),  P = 2^(S - m'),  l = l 2^(m - m') + rowsum P,
//   O = O 2^(m - m') + P V          (scale' = scale log2 e; all of it in fp32)
// 256 threads as 16 x 16; thread (y, x) owns rows 4y..4y+3, keys 4x..4x+3 of S and columns 4x..4x+3 of O.
// Q and K lie transposed in shared memory, so a step of either product reads two 16-byte pieces
// for 16 multiply-adds.
#pragma once
#include "internal.cuh"

namespace gb {

constexpr int kTileRows = 64, kTileKeys = 64, kTileD = 64, kTileThreads = 256;
constexpr int kTileLd = kTileKeys + 4;  // row length of the transposed tiles: 16-byte pieces, spread over the banks
struct TileSmem {
  float q[kTileD][kTileLd];   // [dim][row]
  float k[kTileD][kTileLd];   // [dim][key]
  float v[kTileKeys][kTileLd];  // [key][dim]
  float p[kTileKeys][kTileLd];  // [key][row]
};

// Src: q(r) the row's query or nullptr, key(j) and val(j) its rows or nullptr, on(r, j) whether row r sees key j,
// out(r, c, o, m, l): columns c..c+3 of the unnormalised sum with the row's maximum (base 2) and sum.
template <class Src>
__device__ __forceinline__ void tile_attention(TileSmem& sm, const Src& src, int nkeys, float qscale) {
  const int tid = threadIdx.x, ty = tid >> 4, tx = tid & 15;
  for (int i = tid; i < kTileRows * (kTileD / 4); i += kTileThreads) {
    const int r = i & (kTileRows - 1), c = i / kTileRows * 4;
    const float* p = src.q(r);
    const float4 x = p ? *reinterpret_cast<const float4*>(p + c) : make_float4(0.f, 0.f, 0.f, 0.f);
    sm.q[c][r] = x.x * qscale;
    sm.q[c + 1][r] = x.y * qscale;
    sm.q[c + 2][r] = x.z * qscale;
    sm.q[c + 3][r] = x.w * qscale;
  }
  float o[4][4] = {}, m[4], l[4] = {};
#pragma unroll
  for (int i = 0; i < 4; ++i) m[i] = -INFINITY;
  for (int j0 = 0; j0 < nkeys; j0 += kTileKeys) {
    __syncthreads();  // the previous tile has been read
    for (int i = tid; i < kTileKeys * (kTileD / 4); i += kTileThreads) {
      const int j = i & (kTileKeys - 1), c = i / kTileKeys * 4;
      const float* p = j0 + j < nkeys ? src.key(j0 + j) : nullptr;
      const float4 x = p ? *reinterpret_cast<const float4*>(p + c) : make_float4(0.f, 0.f, 0.f, 0.f);
      sm.k[c][j] = x.x;
      sm.k[c + 1][j] = x.y;
      sm.k[c + 2][j] = x.z;
      sm.k[c + 3][j] = x.w;
    }
    for (int i = tid; i < kTileKeys * (kTileD / 4); i += kTileThreads) {
      const int c = (i & 15) * 4, j = i >> 4;
      const float* p = j0 + j < nkeys ? src.val(j0 + j) : nullptr;
      *reinterpret_cast<float4*>(&sm.v[j][c]) =
          p ? *reinterpret_cast<const float4*>(p + c) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
    __syncthreads();
    float s[4][4] = {};
#pragma unroll 8
    for (int d = 0; d < kTileD; ++d) {
      const float4 a = *reinterpret_cast<const float4*>(&sm.q[d][4 * ty]);
      const float4 b = *reinterpret_cast<const float4*>(&sm.k[d][4 * tx]);
      const float av[4] = {a.x, a.y, a.z, a.w}, bv[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) s[i][j] = fmaf(av[i], bv[j], s[i][j]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float mt = -INFINITY;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int key = j0 + 4 * tx + j;
        if (key >= nkeys || !src.on(4 * ty + i, key)) s[i][j] = -INFINITY;
        mt = fmaxf(mt, s[i][j]);
      }
#pragma unroll
      for (int w = 8; w > 0; w >>= 1) mt = fmaxf(mt, __shfl_xor_sync(0xffffffffu, mt, w));
      const float mn = fmaxf(m[i], mt);
      const float ref = mn == -INFINITY ? 0.f : mn;  // no key seen yet: every p is 0
      const float alpha = exp2f(m[i] - ref);
      m[i] = mn;
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float p = exp2f(s[i][j] - ref);
        sm.p[4 * tx + j][4 * ty + i] = p;
        sum += p;
      }
      l[i] = l[i] * alpha + sum;  // this thread's keys; added over x at the end
#pragma unroll
      for (int c = 0; c < 4; ++c) o[i][c] *= alpha;
    }
    __syncwarp();  // rows 4y..4y+3 of P are written and read by the same half warp
#pragma unroll 8
    for (int j = 0; j < kTileKeys; ++j) {
      const float4 a = *reinterpret_cast<const float4*>(&sm.p[j][4 * ty]);
      const float4 b = *reinterpret_cast<const float4*>(&sm.v[j][4 * tx]);
      const float av[4] = {a.x, a.y, a.z, a.w}, bv[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int c = 0; c < 4; ++c) o[i][c] = fmaf(av[i], bv[c], o[i][c]);
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
#pragma unroll
    for (int w = 8; w > 0; w >>= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], w);
    const int row = 4 * ty + i, c = 4 * tx;
    const float* qr = src.q(row);
    // P V takes every key of a tile, with p = 0 for those the row does not see, and 0 x inf is NaN: columns that are
    // not finite although the row's sum is, are summed again over the keys it sees.
    if (qr && isfinite(m[i]) && isfinite(l[i]) &&
        !(isfinite(o[i][0]) && isfinite(o[i][1]) && isfinite(o[i][2]) && isfinite(o[i][3]))) {
      float acc[4] = {};
      for (int j = 0; j < nkeys; ++j) {
        const float *k = src.on(row, j) ? src.key(j) : nullptr, *v = k ? src.val(j) : nullptr;
        if (!v) continue;
        float sc = 0.f;
        for (int d = 0; d < kTileD; ++d) sc = fmaf(qr[d] * qscale, k[d], sc);
        const float p = exp2f(sc - m[i]);
        for (int e = 0; e < 4; ++e) acc[e] = fmaf(p, v[c + e], acc[e]);
      }
      for (int e = 0; e < 4; ++e) o[i][e] = acc[e];
    }
    src.out(row, c, make_float4(o[i][0], o[i][1], o[i][2], o[i][3]), m[i], l[i]);
  }
}

}  // namespace gb
