// Shared by the kernels of 8-bit products with block scales: launch parameters, tile
// lookup, fragments and epilogue.
#pragma once

#include "common.hpp"
#include "lds_dma.hpp"

namespace lc {

struct Fp8P {
  const uint8_t *A, *B, *sa, *sb;
  void *C;
  const void *R;
  const int32_t *goff;
  int64_t lda, ldb, ldsa, ldsb, ldc, ldr;
  int64_t gstride_b, gstride_sb, gstride_c;
  int M, N, K;
  int tiles_m, tiles_n;
  int ash, bsh;        // rows of a block of scales: 1 << ash, 1 << bsh
  int gmode, ngroups;
  int epi, c_dt, r_dt;
  int vec;             // four columns of C and R from a multiple of 4 on are aligned
};

namespace {

typedef __attribute__((ext_vector_type(8))) int i32x8_v;  // 32 8-bit values of a lane

constexpr int KB = 128;  // k of a block

// A workgroup's tile: rows m0 .. m_lim - 1, columns n0 .., k blocks kb0 .. kb1 - 1 of
// values below kend.
struct Fp8Tile {
  int m0, m_lim, n0;
  int kb0, kb1, kend;
  const uint8_t *B, *sb;
  int64_t c_off;
};

// Tile of workgroup wg; false where it has none (uniform in the workgroup). Group
// offsets are read with a lane per group (at most 64). Grouped rows: the row tiles of
// the groups one after the other, all columns of one first.
template <int BM, int BN>
__device__ __forceinline__ bool fp8_tile(const Fp8P &p, uint32_t wg, Fp8Tile &t) {
  const int lane = threadIdx.x & 63;
  t.m_lim = p.M;
  t.kb0 = 0;
  t.kend = p.K;
  t.B = p.B;
  t.sb = p.sb;
  t.c_off = 0;
  if (p.gmode == LC_GROUP_NONE) {
    t.m0 = (int)(wg / (uint32_t)p.tiles_n) * BM;
    t.n0 = (int)(wg % (uint32_t)p.tiles_n) * BN;
  } else {
    const int most = p.gmode == LC_GROUP_ROWS ? p.M : p.K;
    const int unit = p.gmode == LC_GROUP_ROWS ? BM : KB;
    int lo = 0, hi = 0;
    if (lane < p.ngroups) {
      lo = min(max(p.goff[lane], 0), most);
      hi = max(lo, min(p.goff[lane + 1], most));
    }
    const int nt = (hi - lo + unit - 1) / unit;
    int end = nt;
#pragma unroll
    for (int s = 1; s < 64; s *= 2) {
      const int e = __shfl_up(end, s);
      end += lane >= s ? e : 0;
    }
    if (p.gmode == LC_GROUP_ROWS) {
      const int slot = (int)(wg / (uint32_t)p.tiles_n);
      if (slot >= __builtin_amdgcn_readlane(end, 63)) return false;
      const int g = __builtin_ctzll(__ballot(end > slot));
      t.m0 = __builtin_amdgcn_readlane(lo, g) + (slot - __builtin_amdgcn_readlane(end - nt, g)) * BM;
      t.m_lim = __builtin_amdgcn_readlane(hi, g);
      t.n0 = (int)(wg % (uint32_t)p.tiles_n) * BN;
      t.B = p.B + g * p.gstride_b;
      t.sb = p.sb + g * p.gstride_sb;
    } else {
      const uint32_t per = (uint32_t)p.tiles_m * (uint32_t)p.tiles_n;
      const int g = (int)(wg / per);
      wg -= (uint32_t)g * per;
      t.m0 = (int)(wg / (uint32_t)p.tiles_n) * BM;
      t.n0 = (int)(wg % (uint32_t)p.tiles_n) * BN;
      const int blocks = (p.K + KB - 1) / KB;  // (offsets out of order may ask for more)
      t.kb0 = min(__builtin_amdgcn_readlane(end - nt, g), blocks);
      t.kb1 = min(__builtin_amdgcn_readlane(end, g), blocks);
      t.kend = min(t.kb1 * KB, p.K);
      t.c_off = g * p.gstride_c;
      return true;
    }
  }
  t.kb1 = (t.kend + KB - 1) / KB;
  return true;
}

// acc += the 16 x 16 x 128 product of fragments b (columns) and a (rows): lane l then
// holds row l % 16, columns 4 (l / 16) .. + 3. A lane's 32 values are any 32 of its
// row's 128, the same ones in both operands.
// The blocks' scales (bytes sa of the lane's row, sb of its column) are applied by the
// instruction.
template <int FA, int FB>
__device__ __forceinline__ f32x4_v fp8_mul(const i32x8_v &a, const i32x8_v &b, int sa, int sb, f32x4_v acc) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b, a, acc, FB, FA, 0, sb, 0, sa);
}

// For results of fp32: the values times their scales as bf16 (exact: at most 4
// significant bits), for four bf16 instructions.
// The scale byte s as the float that the conversions take (they read its exponent)
__device__ __forceinline__ float fp8_scale(int s) { return __uint_as_float((uint32_t)s << 23); }
// 8 values (two words) of format F times the scale 2^(s - 127) given as a float
template <int F>
__device__ __forceinline__ bf16x8_v fp8_to_bf16(int lo, int hi, float scale) {
  typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_v;
  bf16x2_v v[4];
  if constexpr (F == 0) {
    v[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false);
    v[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
    v[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false);
    v[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
  } else {
    v[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(lo, scale, false);
    v[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(lo, scale, true);
    v[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(hi, scale, false);
    v[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(hi, scale, true);
  }
  return __builtin_bit_cast(bf16x8_v, v);
}

// C(m, n .. n + 3) = v by the epilogue; m and n in range, columns from N on left out
__device__ __forceinline__ void fp8_store4(const Fp8P &p, int64_t c_off, int64_t m, int n, f32x4_v v) {
  const int64_t at = c_off + m * p.ldc + n;
  const bool whole = p.vec && n + 4 <= p.N;
  if (whole) {
    if (p.epi == LC_EPI_ACCUM_F32) {
      const float4 o = load4_dt(p.C, at, LC_FP32);
      v = f32x4_v{o.x + v[0], o.y + v[1], o.z + v[2], o.w + v[3]};
    } else if (p.epi == LC_EPI_RESIDUAL) {
      const float4 o = load4_dt(p.R, m * p.ldr + n, p.r_dt);
      v = f32x4_v{o.x + v[0], o.y + v[1], o.z + v[2], o.w + v[3]};
    }
    store4_dt(p.C, at, p.c_dt, v[0], v[1], v[2], v[3]);
    return;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if (n + e >= p.N) continue;
    float x = v[e];
    if (p.epi == LC_EPI_ACCUM_F32) x += static_cast<const float *>(p.C)[at + e];
    if (p.epi == LC_EPI_RESIDUAL) {
      const int64_t r = m * p.ldr + n + e;
      x += p.r_dt == LC_FP32 ? static_cast<const float *>(p.R)[r]
           : p.r_dt == LC_BF16 ? bf2f(static_cast<const bf16_t *>(p.R)[r])
                               : (float)static_cast<const _Float16 *>(p.R)[r];
    }
    if (p.c_dt == LC_FP32) static_cast<float *>(p.C)[at + e] = x;
    else if (p.c_dt == LC_BF16) static_cast<__bf16 *>(p.C)[at + e] = (__bf16)x;
    else static_cast<_Float16 *>(p.C)[at + e] = (_Float16)x;
  }
}

}  // namespace
}  // namespace lc
