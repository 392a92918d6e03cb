// Rows of a head on their way into the cache: 16 bytes of 16 lanes each (128 bf16 or 64 fp32 values), turned to
// their position where a rotation is given, and held in 8 bits where the pool is of that type.
#pragma once
#include <cuda_bf16.h>
#include <math.h>

#include "internal.cuh"

namespace gb {

// ---- 8-bit blocks ----------------------------------------------------------------------------
//
// A block is 16 tokens (by position) of one head's K or V: e4m3 codes and one exponent e, a code c standing for
// c 2^e.  e is the least in [kExpLeast, kExpMost] with every row of the block within 448 2^e.  A power of two
// makes both directions exact but for the one rounding of x 2^-e, and a block whose e rises afterwards keeps its
// values where they stay above e4m3's subnormals (2^-15 of the block's largest); a free scale would round them all again.
// The range keeps 2^-e and its products with the attention's weights inside fp32.
constexpr int kBlockRows = 16;
constexpr int kExpLeast = -60, kExpMost = 60;
static_assert(kBlockRows == kChunk, "a chunk of the attention kernels is a block");

__device__ __forceinline__ float pow2i(int e) { return __int_as_float((e + 127) << 23); }  // |e| < 127

// The least e in range with amax <= 448 2^e = 1.75 2^(8 + e).
__device__ __forceinline__ int block_exponent(float amax) {
  const int b = __float_as_int(amax);
  const int e = (b >> 23) - 127 - 8 + ((b & 0x7fffff) > 0x600000 ? 1 : 0);
  return min(max(e, kExpLeast), kExpMost);
}

// Four values to e4m3 codes, ties to even; values past 448 to 448, NaN to NaN.
__device__ __forceinline__ uint32_t e4m3x4(float a, float b, float c, float d) {
  uint16_t lo, hi;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
  return (uint32_t)lo | ((uint32_t)hi << 16);
}

// Two codes as a pair of fp16 (exact).
__device__ __forceinline__ uint32_t f16x2_of_e4m3x2(uint32_t two) {
  uint32_t y;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(y) : "h"((uint16_t)two));
  return y;
}
__device__ __forceinline__ float2 float2_of_f16x2(uint32_t x) {
  float2 f;
  asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.f32.f16 %0, a;\n\tcvt.f32.f16 %1, b;\n\t}" : "=f"(f.x), "=f"(f.y) : "r"(x));
  return f;
}

// Exponent of the block of row `row` of (layer, page, K|V, head).
__device__ __forceinline__ long long exp_offset(const PoolView& v, int layer, long long page, int kv, int head, int row) {
  return ((((long long)layer * v.num_pages + page) * 2 + kv) * v.Hkv + head) * (v.P / kBlockRows) + row / kBlockRows;
}

// ---- rotation ----------------------------------------------------------------------------------

// By value to kernels: the table [positions][4][half] of cos, its rounding errors, sin, its rounding errors.  Each apart, so that
// a half warp's lanes read neighbouring values: with the four side by side a row took 32 lines of L1 a load instead of eight.
struct RotationView {
  const float* table;   // nullptr: none
  int positions, half, interleaved;
};

// a cos + g sin (g: minus the pair's other value, or it), rounded once: the products' and the sum's rounding errors are carried
// along.  What follows rounds to 16 or 8 bits, and a result that is off in its last place can end on the other side of a tie
// there.  Where the plain sum is infinite the errors are no numbers, and it stays (Inf; 8 bits hold neither).
template <bool Inf>
__device__ __forceinline__ float turn(float a, float c, float ce, float g, float s, float se) {
  const float p = __fmul_rn(a, c), q = __fmul_rn(g, s);
  const float pe = __fmaf_rn(a, ce, __fmaf_rn(a, c, -p)), qe = __fmaf_rn(g, se, __fmaf_rn(g, s, -q));
  const float d = __fadd_rn(p, q), t = __fsub_rn(d, p);
  const float err = __fadd_rn(__fsub_rn(p, __fsub_rn(d, t)), __fsub_rn(q, t));
  const float r = __fadd_rn(d, __fadd_rn(err, __fadd_rn(pe, qe)));
  return Inf && r != r ? d : r;
}

template <int DT>
struct RowTraits {                                    // DT: the type of the rows that a caller gives
  static constexpr int N = DT == GB_F32 ? 4 : 8;      // values of a lane's 16 bytes
};

template <int DT>
__device__ __forceinline__ void row_values(const uint4& x, float (&f)[RowTraits<DT>::N]) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (DT == GB_F32) {
      f[i] = __uint_as_float(w[i]);
    } else {
      f[2 * i] = __uint_as_float(w[i] << 16);
      f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
}

template <int DT>
__device__ __forceinline__ uint4 row_bits(const float (&f)[RowTraits<DT>::N]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (DT == GB_F32) {
      w[i] = __float_as_uint(f[i]);
    } else {
      const __nv_bfloat162 t = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&t);
    }
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// The M angles from i0 on of a position (i0: a multiple of M).
template <int M>
__device__ __forceinline__ void angles(const RotationView& rot, int pos, int i0, float (&c)[4][M]) {
  const float* t = rot.table + (size_t)pos * 4 * rot.half + i0;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if constexpr (M == 2) {
      const float2 x = __ldg(reinterpret_cast<const float2*>(t + k * rot.half));
      c[k][0] = x.x;
      c[k][1] = x.y;
    } else {
#pragma unroll
      for (int i = 0; i < M; i += 4) {
        const float4 x = __ldg(reinterpret_cast<const float4*>(t + k * rot.half + i));
        c[k][i] = x.x;
        c[k][i + 1] = x.y;
        c[k][i + 2] = x.z;
        c[k][i + 3] = x.w;
      }
    }
  }
}

// Turn the row that lanes 16h .. 16h + 15 hold (h: this lane's half of the warp) to position pos.  Every lane of
// the warp calls it; pos may differ between the halves.  A position past the table leaves the row as it is.
template <int DT, bool Inf = true>
__device__ __forceinline__ void turn_row(float (&f)[RowTraits<DT>::N], const RotationView& rot, int pos) {
  constexpr int N = RowTraits<DT>::N;
  const int j = threadIdx.x & 15;
  const bool in = pos >= 0 && pos < rot.positions;
  if (rot.interleaved) {
    const int i0 = N / 2 * j;                        // this lane's first pair
    if (in && i0 < rot.half) {
      float c[4][N / 2];
      angles(rot, pos, i0, c);
#pragma unroll
      for (int i = 0; i < N / 2; ++i) {
        const float a = f[2 * i], b = f[2 * i + 1];
        f[2 * i] = turn<Inf>(a, c[0][i], c[1][i], -b, c[2][i], c[3][i]);
        f[2 * i + 1] = turn<Inf>(b, c[0][i], c[1][i], a, c[2][i], c[3][i]);
      }
    }
    return;
  }
  const int away = rot.half / N;                     // lanes between a pair's values (half is a multiple of 8)
  const bool low = j < away, turns = j < 2 * away;
  const int from = (threadIdx.x & 16) + (low ? j + away : turns ? j - away : j);
  float g[N];
#pragma unroll
  for (int i = 0; i < N; ++i) g[i] = __shfl_sync(0xffffffffu, f[i], from);
  if (in && turns) {
    float c[4][N];
    angles(rot, pos, N * (low ? j : j - away), c);
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = turn<Inf>(f[i], c[0][i], c[1][i], low ? -g[i] : g[i], c[2][i], c[3][i]);
  }
}

}  // namespace gb
