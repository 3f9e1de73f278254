// Quantisation to 8-bit floating point in blocks of 128 with power-of-two scales
// (gfx950): the operands of the products in k_gemm_fp8.hip.
//
//   a = largest finite |x| of a block, s = ceil(log2(a / max)) + 127 >= 0,
//   q = round(x 2^(127 - s))            (max 448 or 57344 = 1.75 * 2^8 or 2^15)
//
// From a's bits, a = 1.f * 2^(e - 127): s = e - 8 (15), one more where f > 0.75. The
// scaling by a power of two is exact, so the only rounding is the conversion's.
//
// A workgroup of 512 threads takes a tile of 128 x 128 values: thread (tx, ty) of 16 x
// 32 holds 4 rows (4 ty ..) of 8 columns (8 tx ..) in registers, read once for both
// layouts. A row block's 128 values sit in the 16 lanes of a DPP row (largest value in
// four DPP steps); a column block's in the 32 thread rows (through LDS). Row layout: 8
// bytes per lane and row, 128-byte lines. Column layout: a thread's 4 rows of a column
// are a word in LDS, read back as whole 128-byte lines. 16-bit inputs find their
// largest values two at a time on the bit patterns (v_pk_max_u16: magnitudes order as
// integers, and unlike a floating maximum a signalling NaN does not swallow the rest).
//
// Bound: HBM. 4096 x 4096 of bf16 into both layouts 13.3 us (5.0 TB/s), rows alone 10.3, columns
// 9.6, of fp16 the same within 2%, of fp32 18.0, 14.4 and 14.5 (5.6 to 5.8 TB/s); 11008 x 4096 in
// blocks of 128 x 128 32 us (5.6).
// The column layout goes past the caches, as it is read by a product over the rows, mostly
// not the next one; the row layout stays for the product that reads it next, but that of
// blocks of 128 rows (weights, read by products much later). Quantised rows and columns of
// 4096 x 4096, then the product with 4096 columns, us: 65.4; all kept 68.1, nothing 69.5;
// of 8192 x 8192, with 1024 columns: 108, 133, 130. 11008 x 4096 by itself: 32, kept 39.
#include "common.hpp"

namespace lc {
namespace {

struct QuantP {
  const void *x;
  const int32_t *index;
  const float *weight;
  const int32_t *goff;
  uint8_t *q, *scale, *qt, *scale_t;
  int64_t ld_x, ld_q, ld_s, ld_qt, ld_st;
  int64_t T, x_rows;
  int d, ngroups;
  int nct;         // column tiles
  int col_blocks;  // column layout: blocks of 128 that qt has room for
};

typedef __attribute__((ext_vector_type(2))) uint16_t u16x2_v;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2_v;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4_v;

__device__ __forceinline__ uint32_t max_pair(uint32_t a, uint32_t b) {
  const u16x2_v r = __builtin_elementwise_max(__builtin_bit_cast(u16x2_v, a), __builtin_bit_cast(u16x2_v, b));
  return __builtin_bit_cast(uint32_t, r);
}

// the largest of a DPP row's 16 lanes, in all of them
__device__ __forceinline__ uint32_t row_max(uint32_t v) {
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, true));   // lane ^ 1
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, true));   // lane ^ 2
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xF, 0xF, true));  // mirrored in 8
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x140, 0xF, 0xF, true));  // mirrored in 16
  return v;
}

// scale byte of a block whose largest magnitude has the fp32 bits a
template <bool E5>
__device__ __forceinline__ uint32_t scale_byte(uint32_t a) {
  const int s = (int)(a >> 23) - (E5 ? 15 : 8) + ((a & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return (uint32_t)max(s, 0);
}
// 2^(127 - s), s <= 247
__device__ __forceinline__ float scale_up(uint32_t s) { return __uint_as_float((254u - s) << 23); }

template <bool E5>
__device__ __forceinline__ uint32_t pack4(float a, float b, float c, float d) {
  int r;
  if constexpr (E5) {
    r = __builtin_amdgcn_cvt_pk_bf8_f32(a, b, 0, false);
    r = __builtin_amdgcn_cvt_pk_bf8_f32(c, d, r, true);
  } else {
    r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    r = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
  }
  return (uint32_t)r;
}

template <int XD>
__device__ __forceinline__ float half_value(uint32_t bits16) {
  if constexpr (XD == LC_BF16) return __uint_as_float(bits16 << 16);
  else return (float)__builtin_bit_cast(_Float16, (uint16_t)bits16);
}

constexpr int kColRow = 144;  // bytes of a column's 128 in LDS, with padding
constexpr int R = 4;           // rows of a thread

// XD: type of x; W: rows are weighted; E5: e5m2, else e4m3; SQ: blocks of 128 x 128
template <int XD, bool W, bool E5, bool SQ>
__global__ __launch_bounds__(512) void fp8_quantize_kernel(QuantP p, uint32_t first) {
  constexpr bool H = XD != LC_FP32;  // values stay pairs of 16 bits in registers
  constexpr bool P = H && !W;        // and their magnitudes are compared as such
  constexpr int NW = H ? 4 : 8;      // words of 8 values
  constexpr int NM = P ? 4 : 8;      // words of 8 magnitudes
  constexpr uint32_t INF = !P ? 0x7F800000u : XD == LC_BF16 ? 0x7F80u : 0x7C00u;
  __shared__ __align__(16) uint8_t tile8[128 * kColRow];
  __shared__ __align__(16) uint8_t cexp[128];
  // (the thread rows' maxima are read before the tile's bytes are written)
  auto cmax = reinterpret_cast<uint32_t(*)[16 * NM]>(tile8);
  static_assert(sizeof(tile8) >= 32 * 16 * NM * 4, "maxima of 32 thread rows");

  const int tid = threadIdx.x, lane = tid & 63, tx = tid & 15, ty = tid >> 4;
  const uint32_t wg = first + blockIdx.x;
  const int ct = (int)(wg % (uint32_t)p.nct);
  const int slot = (int)(wg / (uint32_t)p.nct);
  // rows r0 .. rlim - 1 (at most 128), column block cb (-1: no column layout)
  int64_t r0 = (int64_t)slot * 128, rlim = min(p.T, r0 + 128);
  int cb = slot;
  if (p.ngroups > 0) {
    // a lane per group; then the rows behind the groups, then those before them
    int lo = 0, hi = 0;
    if (lane < p.ngroups) {
      lo = (int)min((int64_t)max(p.goff[lane], 0), p.T);
      hi = (int)max((int64_t)lo, min((int64_t)p.goff[lane + 1], p.T));
    }
    const int nb = (int)(((int64_t)hi - lo + 127) / 128);
    int end = nb;
#pragma unroll
    for (int s = 1; s < 64; s *= 2) {
      const int e = __shfl_up(end, s);
      end += lane >= s ? e : 0;
    }
    const int total = __builtin_amdgcn_readlane(end, 63);
    if (slot < total) {
      const int g = __builtin_ctzll(__ballot(end > slot));
      const int before = __builtin_amdgcn_readlane(end - nb, g);
      r0 = __builtin_amdgcn_readlane(lo, g) + (int64_t)(slot - before) * 128;
      rlim = min((int64_t)__builtin_amdgcn_readlane(hi, g), r0 + 128);
      if (slot >= p.col_blocks) cb = -1;
    } else {
      cb = -1;
      const int64_t head = __builtin_amdgcn_readlane(lo, 0);
      const int64_t tail = __builtin_amdgcn_readlane(hi, p.ngroups - 1);
      const int64_t tail_blocks = (p.T - tail + 127) / 128;
      const int64_t j = slot - total;
      if (j < tail_blocks) {
        r0 = tail + j * 128;
        rlim = min(p.T, r0 + 128);
      } else {
        r0 = (j - tail_blocks) * 128;
        rlim = min(head, r0 + 128);
      }
      if (r0 >= rlim || !p.q) return;  // uniform, before any barrier
    }
  }
  const bool rows = p.q != nullptr, cols = p.qt != nullptr && cb >= 0;
  const int c0 = ct * 128 + tx * 8;

  // ---- the thread's 8 x 8 values
  uint32_t w[R][NW];
  float wt[R];  // the rows' weights
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int64_t r = r0 + R * ty + i;
    int64_t src = r;
    bool ok = r < rlim && c0 < p.d;
    if (ok && p.index) {
      src = p.index[r];
      ok = src >= 0 && src < p.x_rows;
    }
    if constexpr (W) wt[i] = ok ? p.weight[r] : 1.0f;
    constexpr int XS = XD == LC_FP32 ? 4 : 2;
    const char *row = static_cast<const char *>(p.x) + (ok ? src * p.ld_x + c0 : 0) * XS;
    uint32_t v[XD == LC_FP32 ? 8 : 4];
#pragma unroll
    for (int k = 0; k < (int)(sizeof(v) / 4); ++k) v[k] = 0;
    if (ok) {
      if (c0 + 8 <= p.d) {  // (rows may start anywhere: wide loads take any address)
        __builtin_memcpy(v, row, sizeof(v));
      } else {
#pragma unroll
        for (int c = 0; c < 8; ++c)
          if (c0 + c < p.d) {
            if constexpr (XD == LC_FP32) v[c] = reinterpret_cast<const uint32_t *>(row)[c];
            else v[c >> 1] |= (uint32_t)reinterpret_cast<const uint16_t *>(row)[c] << (16 * (c & 1));
          }
      }
    }
#pragma unroll
    for (int k = 0; k < NW; ++k) w[i][k] = v[k];
  }
  auto value = [&](int i, int c) -> float {
    float x;
    if constexpr (H) x = half_value<XD>(c & 1 ? w[i][c >> 1] >> 16 : w[i][c >> 1] & 0xFFFFu);
    else x = __uint_as_float(w[i][c]);
    return W ? x * wt[i] : x;
  };

  // ---- largest magnitudes: of the thread's 8 values of each row, of each column
  uint32_t rm[R], cm[NM];
  auto magnitude = [&](uint32_t u, bool finite) -> uint32_t {
    if constexpr (P) {
      u &= 0x7FFF7FFFu;
      if (finite) {
        if ((u & 0xFFFFu) >= INF) u &= 0xFFFF0000u;
        if ((u >> 16) >= INF) u &= 0xFFFFu;
      }
    } else {
      u &= 0x7FFFFFFFu;
      if (finite && u >= INF) u = 0;
    }
    return u;
  };
  auto largest = [&](uint32_t a, uint32_t b) -> uint32_t {
    if constexpr (P) return max_pair(a, b);
    else return max(a, b);
  };
  auto local_max = [&](bool finite) {
#pragma unroll
    for (int k = 0; k < NM; ++k) cm[k] = 0;
#pragma unroll
    for (int i = 0; i < R; ++i) {
      uint32_t m = 0;
#pragma unroll
      for (int k = 0; k < NM; ++k) {
        uint32_t u;
        if constexpr (P) u = magnitude(w[i][k], finite);
        else u = magnitude(__float_as_uint(value(i, k)), finite);
        m = largest(m, u);
        cm[k] = largest(cm[k], u);
      }
      if constexpr (P) m = max(m & 0xFFFFu, m >> 16);
      rm[i] = m;
    }
  };
  // 16-bit values are widened and weighted anew for each use: kept as products they take
  // twice the registers
  auto forget = [&]() {
    if constexpr (H) {
#pragma unroll
      for (int i = 0; i < R; ++i)
#pragma unroll
        for (int k = 0; k < NW; ++k) asm volatile("" : "+v"(w[i][k]));
    }
  };
  local_max(false);
  forget();
  uint32_t any = 0;
#pragma unroll
  for (int i = 0; i < R; ++i) any = max(any, rm[i]);
  if (__syncthreads_or(any >= INF)) local_max(true);  // an infinity or NaN in the tile: without them
  // fp32 bits of a magnitude
  auto bits32 = [&](uint32_t m) -> uint32_t {
    if constexpr (P) return __float_as_uint(half_value<XD>(m));
    else return m;
  };

  uint32_t sq = 0;  // the tile's one scale (SQ)
  if constexpr (SQ) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < R; ++i) m = max(m, rm[i]);
    m = row_max(m);
    if (tx == 0) cmax[ty][0] = m;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 32; ++i) m = max(m, cmax[i][0]);
    __syncthreads();
    sq = scale_byte<E5>(bits32(m));
    if (tid == 0) {
      if (rows) p.scale[(int64_t)ct * p.ld_s + slot] = (uint8_t)sq;
      if (cols) p.scale_t[(int64_t)slot * p.ld_st + ct] = (uint8_t)sq;
    }
  }

  // ---- row layout
  if (rows) {
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int64_t r = r0 + R * ty + i;
      uint32_t s = sq;
      if constexpr (!SQ) s = scale_byte<E5>(bits32(row_max(rm[i])));
      const float up = scale_up(s);
      if (r < rlim) {
        if (c0 < ((p.d + 15) & ~15)) {
          uint2 o;
          o.x = pack4<E5>(value(i, 0) * up, value(i, 1) * up, value(i, 2) * up, value(i, 3) * up);
          o.y = pack4<E5>(value(i, 4) * up, value(i, 5) * up, value(i, 6) * up, value(i, 7) * up);
          if (W && c0 + 8 > p.d) {  // zeros behind d, whatever 0 times the row's weight is
            const int have = max(p.d - c0, 0);
            const uint64_t keep = ((uint64_t)1 << (8 * have)) - 1;  // (have < 8)
            o.x &= (uint32_t)keep;
            o.y &= (uint32_t)(keep >> 32);
          }
          if constexpr (SQ) __builtin_nontemporal_store(u32x2_v{o.x, o.y}, reinterpret_cast<u32x2_v *>(p.q + r * p.ld_q + c0));
          else *reinterpret_cast<uint2 *>(p.q + r * p.ld_q + c0) = o;
        }
        if (!SQ && tx == i) p.scale[(int64_t)ct * p.ld_s + r] = (uint8_t)s;
      }
    }
  }

  // ---- column layout
  if (!cols) return;  // uniform
  forget();
  float up[8];
  if constexpr (SQ) {
#pragma unroll
    for (int c = 0; c < 8; ++c) up[c] = scale_up(sq);
  } else {
#pragma unroll
    for (int k = 0; k < NM; ++k) cmax[ty][tx * NM + k] = cm[k];
    __syncthreads();
    if (tid < 16 * NM) {
      uint32_t m = 0;
#pragma unroll
      for (int i = 0; i < 32; ++i) m = largest(m, cmax[i][tid]);
      const int c = ct * 128 + (P ? 2 * tid : tid);
      uint8_t *const to = p.scale_t + (int64_t)cb * p.ld_st + c;
      if constexpr (P) {
        const uint32_t a = scale_byte<E5>(bits32(m & 0xFFFFu)), b = scale_byte<E5>(bits32(m >> 16));
        cexp[2 * tid] = (uint8_t)a;
        cexp[2 * tid + 1] = (uint8_t)b;
        if (c < p.d) to[0] = (uint8_t)a;
        if (c + 1 < p.d) to[1] = (uint8_t)b;
      } else {
        const uint32_t a = scale_byte<E5>(bits32(m));
        cexp[tid] = (uint8_t)a;
        if (c < p.d) to[0] = (uint8_t)a;
      }
    }
    __syncthreads();
    const uint2 e = *reinterpret_cast<const uint2 *>(cexp + tx * 8);
#pragma unroll
    for (int c = 0; c < 8; ++c) up[c] = scale_up(((c < 4 ? e.x : e.y) >> (8 * (c & 3))) & 0xFFu);
  }
  // column 8 tx + c of the tile is line 16 c + tx: lines of neighbouring lanes are 36
  // banks apart
#pragma unroll
  for (int c = 0; c < 8; ++c) {
    *reinterpret_cast<uint32_t *>(tile8 + (16 * c + tx) * kColRow + R * ty) =
        pack4<E5>(value(0, c) * up[c], value(1, c) * up[c], value(2, c) * up[c], value(3, c) * up[c]);
  }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int j = u * 512 + tid, line = j >> 3, ch = j & 7;  // line 16 c + tx
    const int col = ct * 128 + 8 * (line & 15) + (line >> 4);
    if (col < p.d)
      __builtin_nontemporal_store(*reinterpret_cast<const u32x4_v *>(tile8 + line * kColRow + 16 * ch),
                                  reinterpret_cast<u32x4_v *>(p.qt + (int64_t)col * p.ld_qt + (int64_t)cb * 128 + 16 * ch));
  }
}

}  // namespace

static int64_t padded_rows(int64_t T, int n_groups) {
  const int64_t g = n_groups > 0 ? n_groups : 1;
  return (T + 127 * g) / 128 * 128;
}

static lc_status quantize_launch(const lc_fp8_quantize_args &a, hipStream_t s) {
  if (a.T < 0 || a.d < 1) return fail(LC_ERR_INVALID_ARG, "fp8 quantize: need T >= 0 and d >= 1");
  if (a.T > INT32_MAX || a.d > (1 << 24)) return fail(LC_ERR_UNSUPPORTED, "fp8 quantize: T or d too large");
  if (!valid_dtype(a.x_dtype)) return fail(LC_ERR_INVALID_ARG, "fp8 quantize: unknown x_dtype");
  if (a.q_dtype != LC_FP8_E4M3 && a.q_dtype != LC_FP8_E5M2)
    return fail(LC_ERR_INVALID_ARG, "fp8 quantize: q_dtype must be e4m3 or e5m2");
  if (a.block_rows != 1 && a.block_rows != 128)
    return fail(LC_ERR_INVALID_ARG, "fp8 quantize: block_rows must be 1 or 128");
  if (a.n_groups < 0 || a.n_groups > 64) return fail(LC_ERR_INVALID_ARG, "fp8 quantize: n_groups must be 0..64");
  if (a.n_groups > 0 && a.block_rows != 1)
    return fail(LC_ERR_UNSUPPORTED, "fp8 quantize: groups need block_rows 1");
  if (a.n_groups > 0 && (!a.group_offsets || (reinterpret_cast<uintptr_t>(a.group_offsets) & 3)))
    return fail(LC_ERR_INVALID_ARG, "fp8 quantize: group offsets must be a 4-byte aligned device array");
  if ((a.row_index && (a.x_rows < 0 || (reinterpret_cast<uintptr_t>(a.row_index) & 3))) ||
      (reinterpret_cast<uintptr_t>(a.row_weight) & 3))
    return fail(LC_ERR_INVALID_ARG, "fp8 quantize: bad row_index, x_rows or row_weight");
  const int64_t ld_x = a.ld_x ? a.ld_x : a.d, br = a.block_rows;
  if (ld_x < a.d || ld_x > ((int64_t)1 << 40)) return fail(LC_ERR_INVALID_ARG, "fp8 quantize: bad ld_x");
  if (!a.q && !a.qt) return fail(LC_ERR_INVALID_ARG, "fp8 quantize: neither layout asked for");
  if (!a.q != !a.scale || !a.qt != !a.scale_t)
    return fail(LC_ERR_INVALID_ARG, "fp8 quantize: values and scales come together");
  if (a.T > 0 && (!a.x || !aligned16(a.x) || !aligned16(a.q) || !aligned16(a.scale) || !aligned16(a.qt) || !aligned16(a.scale_t)))
    return fail(LC_ERR_INVALID_ARG, "fp8 quantize: null or unaligned pointer");
  if (a.q && (a.ld_q % 16 || a.ld_q < a.d || a.ld_q > ((int64_t)1 << 40) || a.ld_scale % 4 ||
              a.ld_scale < (a.T + br - 1) / br || a.ld_scale > ((int64_t)1 << 40)))
    return fail(LC_ERR_INVALID_ARG, "fp8 quantize: bad ld_q or ld_scale");
  const int64_t cols = padded_rows(a.T, a.n_groups);
  if (a.qt && (a.ld_qt % 16 || a.ld_qt < cols || a.ld_qt > ((int64_t)1 << 40) || a.ld_scale_t % 4 ||
               a.ld_scale_t < (a.d + br - 1) / br || a.ld_scale_t > ((int64_t)1 << 40)))
    return fail(LC_ERR_INVALID_ARG, "fp8 quantize: bad ld_qt or ld_scale_t");
  if (a.T == 0) return LC_OK;

  QuantP p{};
  p.x = a.x;
  p.index = a.row_index;
  p.weight = a.row_weight;
  p.goff = a.group_offsets;
  p.q = static_cast<uint8_t *>(a.q);
  p.scale = a.scale;
  p.qt = static_cast<uint8_t *>(a.qt);
  p.scale_t = a.scale_t;
  p.ld_x = ld_x;
  p.ld_q = a.ld_q;
  p.ld_s = a.ld_scale;
  p.ld_qt = a.ld_qt;
  p.ld_st = a.ld_scale_t;
  p.T = a.T;
  p.x_rows = a.row_index ? a.x_rows : a.T;
  p.d = (int)a.d;
  p.ngroups = a.n_groups;
  p.nct = (int)((a.d + 127) / 128);
  p.col_blocks = (int)(cols / 128);
  // groups: one partial block each, and one each for the rows before and behind them
  const int64_t slots = a.n_groups > 0 ? (a.T + 127 * (int64_t)(a.n_groups + 2)) / 128 : (a.T + 127) / 128;
  if (slots * p.nct > (int64_t)UINT32_MAX) return fail(LC_ERR_UNSUPPORTED, "fp8 quantize: too many values");
  const bool w = a.row_weight != nullptr, e5 = a.q_dtype == LC_FP8_E5M2, sq = a.block_rows == 128;
  launch_parts((uint32_t)(slots * p.nct), [&](uint32_t first, uint32_t count) {
    with_dtype(a.x_dtype, [&](auto xd) {
      constexpr int XD = decltype(xd)::value;
      auto go = [&](auto w_, auto e_, auto s_) {
        hipLaunchKernelGGL((fp8_quantize_kernel<XD, decltype(w_)::value, decltype(e_)::value, decltype(s_)::value>),
                           dim3(count), dim3(512), 0, s, p, first);
      };
      using T_ = std::true_type;
      using F_ = std::false_type;
      if (sq) {
        if (w) e5 ? go(T_{}, T_{}, T_{}) : go(T_{}, F_{}, T_{});
        else e5 ? go(F_{}, T_{}, T_{}) : go(F_{}, F_{}, T_{});
      } else {
        if (w) e5 ? go(T_{}, T_{}, F_{}) : go(T_{}, F_{}, F_{});
        else e5 ? go(F_{}, T_{}, F_{}) : go(F_{}, F_{}, F_{});
      }
    });
  });
  return check_launch("fp8_quantize_kernel");
}

}  // namespace lc

extern "C" {

lc_status lc_fp8_quantize(const lc_fp8_quantize_args *args, void *stream) {
  if (!args) return lc::fail(LC_ERR_INVALID_ARG, "fp8 quantize: null args");
  return lc::quantize_launch(*args, static_cast<hipStream_t>(stream));
}

int64_t lc_fp8_padded_rows(int64_t T, int32_t n_groups) {
  if (T < 0 || T > INT32_MAX || n_groups < 0 || n_groups > 64) return 0;
  return lc::padded_rows(T, n_groups);
}

}  // extern "C"
