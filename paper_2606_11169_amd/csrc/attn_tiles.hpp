// What the matrix-core attention kernels share: operand types and the 32 x 32 x 16
// matrix instruction, the reads of row tiles in LDS in an accumulator's order, and lane
// pair reductions.
#pragma once

#include "lds_dma.hpp"

#include <type_traits>

namespace lc {
namespace {

constexpr float LOG2E = 1.4426950408889634f;

// 2^x by the hardware instruction (v_exp_f32): no range reduction for results
// below the normal range, which only ever go into softmax weights that are
// rounded to 16 bits (where they are zero anyway); 2^-inf = 0.
__device__ __forceinline__ float ex2(float x) { return __builtin_amdgcn_exp2f(x); }
constexpr float LN2 = 0.6931471805599453f;

// row tiles consist of load runs of 1 KiB (one 16-byte chunk per lane), 16 bytes apart
constexpr int RUNB = 1024 + 16;

template <typename E> struct V8;
template <> struct V8<__bf16> { typedef bf16x8_v type; };
template <> struct V8<_Float16> { typedef f16x8_v type; };

__device__ __forceinline__ f32x16_v mfma(bf16x8_v a, bf16x8_v b, f32x16_v c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16_v mfma(f16x8_v a, f16x8_v b, f32x16_v c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}

__device__ __forceinline__ void wait_vm0() { __builtin_amdgcn_s_waitcnt(0x0F70); }

// The transposing reads of frag_cols (k_attn.hip) from the byte address `a` of the lane's
// first row: 32 columns from 32 i on, rows kbase + .. in an accumulator's order; rows 8
// further sit two runs further
template <typename VT>
__device__ __forceinline__ VT frag_cols_x(uint32_t a, int i, int kbase) {
  typedef __attribute__((address_space(3))) s16x4_v lds_v4;
  const uint32_t lo = a + 64u * i + 16u * kbase;
  const s16x4_v v[2] = {__builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4 *)(uintptr_t)lo),
                        __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4 *)(uintptr_t)(lo + 2 * RUNB))};
  return __builtin_bit_cast(VT, v);
}

// max / sum of a lane's value and lane (l ^ 32)'s, in every lane
// (v_permlane32_swap: the upper half of one register trades places with the
// lower half of the other; with both registers holding x, the results hold the
// lower and the upper half of x in both halves)
__device__ __forceinline__ float max_with_partner(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_with_partner(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

template <typename E>
__device__ __forceinline__ typename V8<E>::type pack8(const f32x16_v &a, int base) {
  typename V8<E>::type r;
#pragma unroll
  for (int e = 0; e < 8; ++e) r[e] = (E)a[base + e];
  return r;
}

// row index inside a 32-row MFMA output block held by register r of a lane in half hf
__device__ __forceinline__ int out_row(int r, int hf) { return (r & 3) + 8 * (r >> 2) + 4 * hf; }

__device__ __forceinline__ f32x16_v zero16() {
  f32x16_v z;
#pragma unroll
  for (int r = 0; r < 16; ++r) z[r] = 0.0f;
  return z;
}

// 8 elements of type E (16 bytes) as 8 bf16
template <typename E>
__device__ __forceinline__ bf16x8_v to_bf16x8(uint4 v) {
  if constexpr (std::is_same<E, __bf16>::value) {
    return __builtin_bit_cast(bf16x8_v, v);
  } else {
    const f16x8_v h = __builtin_bit_cast(f16x8_v, v);
    bf16x8_v b;
#pragma unroll
    for (int e = 0; e < 8; ++e) b[e] = (__bf16)(float)h[e];
    return b;
  }
}

}  // namespace
}  // namespace lc
