// What the fp32 attention kernels share: products on the fp32 matrix instruction
// (v_mfma_f32_16x16x4_f32) of 16 queries (keys) with blocks of 32 keys (queries), and the merge
// of a workgroup's four waves.
//
// Fragments (lane l, group g = l / 16): a score product takes A[row l % 16][k
// slot g] and B[k slot g][column l % 16]. Its k slots may stand for any features
// as long as both operands agree: product (j, c) uses feature 16 j + 4 g + c, so
// that a lane's values are 16-byte runs. The scores come out with the column
// (query in forward and dQ, key in dK/dV) on the lane and rows 4 g + r in
// register r, which is the B operand of the second product with k slot g standing
// for row 4 g + r: no data moves between the two. Its rows stand for features NI
// (l % 16) + i of product i, so that a lane's loads and its outputs (features 4 NI
// g + NI r + i) are runs too.
//
// A masked pair has weight 0, but 0 times an infinite or NaN value would be NaN:
// in blocks that hold masked pairs the values are looked at, and if one is not
// finite the block's second product is formed pair by pair instead.
#pragma once

#include "common.hpp"

#include <math.h>

namespace lc {
namespace {

constexpr int QR = 16;  // queries (keys) per workgroup
constexpr int KB = 32;  // keys (queries) per block
constexpr int NW = 4;   // waves
constexpr int NTF = 64 * NW;

__device__ __forceinline__ f32x4_v mfma4(float a, float b, f32x4_v c) {
  return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
}

// x[i] = row[e0 + i], 0 at or past hd (i < n, n a power of two, e0 a multiple of n)
template <int N>
__device__ __forceinline__ void load_run(const float *row, int e0, int hd, bool vec, float (&x)[N]) {
  if constexpr (N >= 4) {
    if (vec) {  // hd, e0 multiples of 4: a run of four is inside the row or past it
#pragma unroll
      for (int i = 0; i < N; i += 4) {
        float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (e0 + i < hd) v = *reinterpret_cast<const float4 *>(row + e0 + i);
        x[i] = v.x; x[i + 1] = v.y; x[i + 2] = v.z; x[i + 3] = v.w;
      }
      return;
    }
  }
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = e0 + i < hd ? row[e0 + i] : 0.0f;
}

// the lane's score-product fragment of a row: features 16 j + 4 g + c
template <int NI>
__device__ __forceinline__ void load_frag(const float *row, int g, int hd, bool vec, float (&x)[NI][4]) {
#pragma unroll
  for (int j = 0; j < NI; ++j) load_run<4>(row, 16 * j + 4 * g, hd, vec, x[j]);
}

template <int NI>
__device__ __forceinline__ f32x4_v score(const float (&a)[NI][4], const float (&b)[NI][4]) {
  f32x4_v s = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int j = 0; j < NI; ++j)
#pragma unroll
    for (int c = 0; c < 4; ++c) s = mfma4(a[j][c], b[j][c], s);
  return s;
}

// sum (max) over the four lanes of a column
__device__ __forceinline__ float col_sum(float x) {
  x += __shfl_xor(x, 16, 64);
  return x + __shfl_xor(x, 32, 64);
}
__device__ __forceinline__ float col_max(float x) {
  x = fmaxf(x, __shfl_xor(x, 16, 64));
  return fmaxf(x, __shfl_xor(x, 32, 64));
}

// acc[e][column] += sum over the block's rows of w[row][column] X[row][e], the
// rows at r0 .. r0 + 31 (X rows x0 + row, at most last). `masked`: some pair of
// the block is masked; vis(row) says whether this lane's column sees a row.
template <int NI, typename F>
__device__ __forceinline__ void accumulate(f32x4_v (&acc)[NI], const f32x4_v (&w)[2], const float *x0,
                                           int64_t ld, int r0, int last, int hd, bool vec, int lane,
                                           bool masked, F vis) {
  const int g = lane >> 4, c = lane & 15;
  float x[2][4][NI];
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r)
      load_run<NI>(x0 + (int64_t)min(r0 + 16 * t + 4 * g + r, last) * ld, NI * c, hd, vec, x[t][r]);
  if (masked) {
    bool bad = false;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int i = 0; i < NI; ++i) bad |= !(fabsf(x[t][r][i]) < INFINITY);
    if (__any(bad)) {
#pragma unroll 1
      for (int n = 0; n < 32; ++n) {
        const int row = r0 + n, t = n >> 4, r = n & 3;
        float mine = 0.0f;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (u == t && e == r) mine = w[u][e];
        const float wv = __shfl(mine, c + 16 * ((n >> 2) & 3), 64);
        if (row > last || !vis(row)) continue;
#pragma unroll
        for (int i = 0; i < NI; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int f = NI * (4 * g + e) + i;
            if (f < hd) acc[i][e] += wv * x0[(int64_t)row * ld + f];
          }
      }
      return;
    }
  }
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int i = 0; i < NI; ++i) acc[i] = mfma4(x[t][r][i], w[t][r], acc[i]);
}

// The waves' accumulators in LDS: feature e of column c of wave w at (w 16 + c) LD + e
template <int NI, int W = NW>
struct Merge {
  static constexpr int LD = 16 * NI + 4;
  static constexpr int FLOATS = W * QR * LD;
  __device__ __forceinline__ static void put(float *s, const f32x4_v (&acc)[NI], int w, int lane) {
    float *row = s + (w * QR + (lane & 15)) * LD + 4 * NI * (lane >> 4);
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int i = 0; i < NI; ++i) row[NI * e + i] = acc[i][e];
  }
  __device__ __forceinline__ static float sum(const float *s, int c, int e) {
    float t = s[c * LD + e];
#pragma unroll
    for (int w = 1; w < W; ++w) t += s[(w * QR + c) * LD + e];
    return t;
  }
};

}  // namespace
}  // namespace lc
