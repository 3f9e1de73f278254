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
  int goff_max;        // offsets end there: M (grouped rows) or K
  int epi, c_dt, r_dt;
  int store16;         // STORE of 16-bit values
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
  // values of a row from kb0 on; a group without blocks may begin behind the last value
  __device__ __forceinline__ int span() const { return max(kend - kb0 * KB, 0); }
};

// Tile of workgroup wg; false where it has none (uniform in the workgroup). Group
// offsets are read with a lane per group (at most 64). Grouped rows: the row tiles of
// the groups one after the other, all columns of one first. MAP: workgroups are dealt
// to the 8 XCDs in turn, so XCD x takes the x-th eighth of the tiles, walked in groups
// of WALK tile rows: neighbours share rows of A and columns of B in its L2. (Selects
// instead of branches throughout: behind divergent branches the kernels' loops are
// compiled with vector registers for what is uniform, and the 256 tile spills: 4096 x
// 11008 x 4096 605 us, without spills 145.)
__device__ __forceinline__ uint32_t fp8_xcd_tile(uint32_t wg, uint32_t n) {
  const uint32_t x = wg & 7u;
  return x * (n >> 3) + min(x, n & 7u) + (wg >> 3);
}
// Of 1 to 6 and 8 tile rows 4 is within 1% of the fastest, at odd and even numbers of tile
// columns (2048 x 2176 x 4096 alone 4%: 25.6 us by 1, 26.6). us by 1, 3, 4, 8: 4096 x 11008 x 4096
// (43 columns of 256) 152, 145, 144, 144; 4096 x 11264 x 4096 (44) 154, 146, 143, 144; 4096 x 4352 x
// 4096 (17) 100, 86, 85, 85; 8192 x 8192 x 1024 (32) 77, 71, 70, 80; in fp32 4096 x 4224 x 4096 (33
// of 128) 134, 128, 127, 127.
__device__ __forceinline__ void fp8_walk(const Fp8P &p, uint32_t wg, uint32_t &tm, uint32_t &tn) {
  constexpr uint32_t WALK = 4;
  const uint32_t per = WALK * (uint32_t)p.tiles_n, first = wg / per * WALK;
  const uint32_t rows = min((uint32_t)p.tiles_m - first, WALK);
  tm = first + wg % per % rows;
  tn = wg % per / rows;
}
template <int BM, int BN, bool MAP>
__device__ __forceinline__ bool fp8_find_tile(const Fp8P &p, uint32_t wg, Fp8Tile &t) {
  t.m_lim = p.M;
  t.kb0 = 0;
  t.kb1 = (p.K + KB - 1) / KB;
  t.kend = p.K;
  t.B = p.B;
  t.sb = p.sb;
  t.c_off = 0;
  uint32_t n = (uint32_t)p.tiles_m * (uint32_t)p.tiles_n, tm, tn;
  bool there = true;
  if (p.gmode == LC_GROUP_NONE) {
    if constexpr (MAP) {
      wg = fp8_xcd_tile(wg, n);
      fp8_walk(p, wg, tm, tn);
    } else {
      tm = wg / (uint32_t)p.tiles_n;
      tn = wg % (uint32_t)p.tiles_n;
    }
    t.m0 = (int)tm * BM;
  } else {
    // a lane per group, without a branch
    const int lane = threadIdx.x & 63, at = min(lane, p.ngroups - 1);
    const int unit = p.gmode == LC_GROUP_ROWS ? BM : KB;
    const int lo = min(max(p.goff[at], 0), p.goff_max), hi = max(lo, min(p.goff[at + 1], p.goff_max));
    const int nt = lane < p.ngroups ? (hi - lo + unit - 1) / unit : 0;
    int end = nt;
#pragma unroll
    for (int s = 1; s < 64; s *= 2) {
      const int e = __shfl_up(end, s);
      end += lane >= s ? e : 0;
    }
    if (p.gmode == LC_GROUP_ROWS) {
      n = (uint32_t)__builtin_amdgcn_readlane(end, 63) * (uint32_t)p.tiles_n;
      there = wg < n;
      wg = there ? wg : 0;
      if constexpr (MAP) wg = fp8_xcd_tile(wg, n);
      const int slot = (int)(wg / (uint32_t)p.tiles_n);
      const uint64_t later = __ballot(end > slot);
      const int g = later ? __builtin_ctzll(later) : 0;
      there = there && later != 0;
      t.m0 = __builtin_amdgcn_readlane(lo, g) + (slot - __builtin_amdgcn_readlane(end - nt, g)) * BM;
      t.m_lim = __builtin_amdgcn_readlane(hi, g);
      tn = wg % (uint32_t)p.tiles_n;
      t.B = p.B + g * p.gstride_b;
      t.sb = p.sb + g * p.gstride_sb;
    } else {
      // Groups of very different lengths: the longest first, and each group's tiles over all
      // XCDs (an XCD's eighth of all tiles could be one long group's).
      const uint32_t per = (n + 7) & ~7u;
      int before = 0;  // groups that come before this lane's
      for (int i = 0; i < p.ngroups; ++i) {
        const int other = __builtin_amdgcn_readlane(nt, i);
        before += other > nt || (other == nt && i < lane) ? 1 : 0;
      }
      const uint64_t mine = __ballot(lane < p.ngroups && before == (int)(wg / per));
      const int g = mine ? __builtin_ctzll(mine) : 0;
      wg %= per;
      if constexpr (MAP) {
        const uint32_t x = wg & 7u, share = (n >> 3) + (x < (n & 7u) ? 1u : 0u);
        there = (wg >> 3) < share;
        wg = there ? fp8_xcd_tile(wg, n) : 0;
        fp8_walk(p, wg, tm, tn);
      } else {
        there = wg < n;
        tm = wg / (uint32_t)p.tiles_n;
        tn = wg % (uint32_t)p.tiles_n;
      }
      t.m0 = (int)tm * BM;
      // (offsets out of order may ask for more blocks than there are)
      t.kb0 = min(__builtin_amdgcn_readlane(end - nt, g), t.kb1);
      t.kb1 = min(__builtin_amdgcn_readlane(end, g), t.kb1);
      t.kend = min(t.kb1 * KB, p.K);
      t.c_off = g * p.gstride_c;
    }
  }
  t.n0 = (int)tn * BN;
  return there;
}

// A wave-uniform 64-bit value in scalar registers
__device__ __forceinline__ uint64_t fp8_uniform(uint64_t v) {
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v), hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
  return (uint64_t)hi << 32 | lo;
}
// The same in scalar registers, whatever way it was found (the 256 tile spills otherwise:
// 165 us)
template <int BM, int BN, bool MAP = false>
__device__ __forceinline__ bool fp8_tile(const Fp8P &p, uint32_t wg, Fp8Tile &t) {
  const bool there = fp8_find_tile<BM, BN, MAP>(p, wg, t);
  t.m0 = __builtin_amdgcn_readfirstlane(t.m0);
  t.m_lim = __builtin_amdgcn_readfirstlane(t.m_lim);
  t.n0 = __builtin_amdgcn_readfirstlane(t.n0);
  t.kb0 = __builtin_amdgcn_readfirstlane(t.kb0);
  t.kb1 = __builtin_amdgcn_readfirstlane(t.kb1);
  t.kend = __builtin_amdgcn_readfirstlane(t.kend);
  t.B = reinterpret_cast<const uint8_t *>(fp8_uniform(reinterpret_cast<uint64_t>(t.B)));
  t.sb = reinterpret_cast<const uint8_t *>(fp8_uniform(reinterpret_cast<uint64_t>(t.sb)));
  t.c_off = (int64_t)fp8_uniform((uint64_t)t.c_off);
  return there;
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

// For results of fp16 and fp32: the values times their scales as bf16 (exact: at most 4
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

// One value of C or R
__device__ __forceinline__ float fp8_load1(const void *base, int64_t at, int dt) {
  if (dt == LC_FP32) return static_cast<const float *>(base)[at];
  if (dt == LC_BF16) return bf2f(static_cast<const bf16_t *>(base)[at]);
  return (float)static_cast<const _Float16 *>(base)[at];
}

// Four consecutive values at any alignment of their type (the hardware's wide accesses
// take any address; rows of an odd number of values start anywhere)
__device__ __forceinline__ float4 fp8_load4(const void *base, int64_t at, int dt) {
  if (dt == LC_FP32) {
    float4 v;
    __builtin_memcpy(&v, static_cast<const float *>(base) + at, 16);
    return v;
  }
  if (dt == LC_BF16) {
    bf16x4_v v;
    __builtin_memcpy(&v, static_cast<const __bf16 *>(base) + at, 8);
    return make_float4((float)v[0], (float)v[1], (float)v[2], (float)v[3]);
  }
  f16x4_v v;
  __builtin_memcpy(&v, static_cast<const _Float16 *>(base) + at, 8);
  return make_float4((float)v[0], (float)v[1], (float)v[2], (float)v[3]);
}

// Results are stored past the caches, at any alignment of their type: kept there, they push
// the operands out, and written back later, they stand in the way. 4096 x 2816 x 2048 24.2
// us, kept 26.2, and with a kernel that reads C next 33.5 and 34.2; weight gradients of 8
// experts (92 MB) 57 and 93.
template <typename V>
__device__ __forceinline__ void fp8_stream_store(void *to, const V &v) {
  typedef V any __attribute__((aligned(2)));
  __builtin_nontemporal_store(v, static_cast<any *>(to));
}

// C(m, n .. n + 3) = x by the epilogue; m and n in range, columns from N on left out
__device__ __forceinline__ void fp8_store4(const Fp8P &p, int64_t c_off, int64_t m, int n, float x0, float x1,
                                           float x2, float x3) {
  const int64_t at = c_off + m * p.ldc + n;
  if (n + 4 <= p.N) {
    if (p.epi != LC_EPI_STORE && p.epi != LC_EPI_STORE_F32) {
      const bool acc = p.epi == LC_EPI_ACCUM_F32;
      const float4 o = fp8_load4(acc ? p.C : p.R, acc ? at : m * p.ldr + n, acc ? (int)LC_FP32 : p.r_dt);
      x0 += o.x; x1 += o.y; x2 += o.z; x3 += o.w;
    }
    if (p.c_dt == LC_FP32) {
      fp8_stream_store(static_cast<float *>(p.C) + at, f32x4_v{x0, x1, x2, x3});
    } else if (p.c_dt == LC_BF16) {
      fp8_stream_store(static_cast<__bf16 *>(p.C) + at, bf16x4_v{(__bf16)x0, (__bf16)x1, (__bf16)x2, (__bf16)x3});
    } else {
      fp8_stream_store(static_cast<_Float16 *>(p.C) + at, f16x4_v{(_Float16)x0, (_Float16)x1, (_Float16)x2, (_Float16)x3});
    }
    return;
  }
  const float x[4] = {x0, x1, x2, x3};
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (n + e < p.N) {
      float y = x[e];
      if (p.epi == LC_EPI_ACCUM_F32) y += static_cast<const float *>(p.C)[at + e];
      if (p.epi == LC_EPI_RESIDUAL) y += fp8_load1(p.R, m * p.ldr + n + e, p.r_dt);
      if (p.c_dt == LC_FP32) static_cast<float *>(p.C)[at + e] = y;
      else if (p.c_dt == LC_BF16) static_cast<__bf16 *>(p.C)[at + e] = (__bf16)y;
      else static_cast<_Float16 *>(p.C)[at + e] = (_Float16)y;
    }
}

// Calls f with the operands' formats (0: e4m3, 1: e5m2) as constants
template <typename F>
void fp8_with_formats(const lc_gemm_fp8_args &a, F f) {
  auto fb = [&](auto x) {
    if (a.b_dtype == LC_FP8_E4M3) f(x, std::integral_constant<int, 0>{});
    else f(x, std::integral_constant<int, 1>{});
  };
  if (a.a_dtype == LC_FP8_E4M3) fb(std::integral_constant<int, 0>{});
  else fb(std::integral_constant<int, 1>{});
}

// The grid of BM x BN tiles: p's tile counts, and workgroups in *grid
template <int BM, int BN>
lc_status fp8_grid(Fp8P &p, uint32_t *grid) {
  p.tiles_m = (p.M + BM - 1) / BM;
  p.tiles_n = (p.N + BN - 1) / BN;
  // grouped rows: each group may add a partial tile
  const int64_t rows = (int64_t)p.tiles_m + (p.gmode == LC_GROUP_ROWS ? p.ngroups : 0);
  int64_t n = rows * p.tiles_n;
  if (p.gmode == LC_GROUP_K) n = (n + 7) / 8 * 8 * p.ngroups;
  if (n > (int64_t)INT32_MAX) return fail(LC_ERR_UNSUPPORTED, "gemm fp8: too many outputs");
  *grid = (uint32_t)n;
  return LC_OK;
}

}  // namespace

// k_gemm_fp8_tile.hip: tiles of 32, 64, 128 or 256 (256: results of bf16); deep: four
// stages in LDS instead of two (128); f32: summed by the bf16 instructions
lc_status gemm_fp8_tile_launch(Fp8P p, const lc_gemm_fp8_args &a, int tile, bool deep, bool f32, hipStream_t s);

}  // namespace lc
