// Balance and z loss of a top-2 router, per-expert counts, and the gradients of both
// through the router's product (gfx950).
//
//   l = n Wr^T, p = softmax(l), f_e = counts[e] / (2N), P_e = sum_t p[t, e] / N
//   loss = (E sum_e f_e P_e, sum_t lse[t]^2 / N)
//   dl[t, e] = coef E / N p (f_e - sum f p) + 2 z_coef / N lse p + the pair's gate gradient
//   dn = dres + dl Wr, dWr = dl^T n
//
// The three products run on the bf16 matrix cores for every type: a value is cut into
// bf16 pieces of 8 bits (fp16 into 2, fp32 into 3, exactly), and the pieces' products
// above 2^-24 of the whole are added in fp32, so a bf16 router pays one instruction
// where fp32 ones would take sixteen times as long. dl is fp32 and takes three pieces.
//
// Bound: HBM, by n (forward), and n, dres and dn (backward).
#include "common.hpp"
#include "lds_dma.hpp"

namespace lc {
namespace {

struct BalanceP {
  const void *n, *wr, *dres;
  const int32_t *sel;
  const uint8_t *mask;
  float *probs, *lse, *loss;
  int32_t *counts;
  const float *w, *dw;
  void *dn;
  float *dwr, *part;
  int64_t T;
  int d, E;
  int dn_dt, dres_dt;
  int splits;      // backward: parts of the tokens
  int64_t tiles;   // token tiles
  float coef, z_coef;
  int store;
};

template <int DT> constexpr int kPieces = DT == LC_FP32 ? 3 : DT == LC_FP16 ? 2 : 1;

// x as P bf16 pieces, largest first: each takes the next 8 bits
template <int P>
__device__ __forceinline__ void split_bf16(float x, uint16_t (&out)[P]) {
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const uint32_t u = __float_as_uint(x);
    out[i] = (uint16_t)(u >> 16);
    x = (u & 0x7F800000u) == 0x7F800000u ? 0.0f : x - __uint_as_float(u & 0xFFFF0000u);
  }
}

// 8 values at base[idx] as P MFMA fragments
template <int DT>
__device__ __forceinline__ void load_pieces(const void *base, int64_t idx, bool ok, bf16x8_v (&out)[kPieces<DT>]) {
  constexpr int P = kPieces<DT>;
  if constexpr (P == 1) {
    typedef __attribute__((ext_vector_type(4))) uint32_t u32x4_v;
    u32x4_v v = u32x4_v{0, 0, 0, 0};
    if (ok) v = *reinterpret_cast<const u32x4_v *>(static_cast<const bf16_t *>(base) + idx);
    out[0] = __builtin_bit_cast(bf16x8_v, v);
  } else {
    float x[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
    if (ok) load8_dt(base, idx, DT, x);
    typedef __attribute__((ext_vector_type(8))) uint16_t u16x8_v;
    u16x8_v v[P];
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      uint16_t s[P];
      split_bf16<P>(x[c], s);
#pragma unroll
      for (int i = 0; i < P; ++i) v[i][c] = s[i];
    }
#pragma unroll
    for (int i = 0; i < P; ++i) out[i] = __builtin_bit_cast(bf16x8_v, v[i]);
  }
}

// acc += a b over the pieces, smallest products first
template <int PA, int PB>
__device__ __forceinline__ f32x4_v mul_pieces(const bf16x8_v (&a)[PA], const bf16x8_v (&b)[PB], f32x4_v acc) {
#pragma unroll
  for (int s = 2; s >= 0; --s)
#pragma unroll
    for (int i = 0; i < PA; ++i) {
      const int j = s - i;
      if (j >= 0 && j < PB) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[i], b[j], acc, 0, 0, 0);
    }
  return acc;
}

constexpr int kFwdTokens = 32;   // tokens per tile
constexpr int kFwdBlocks = 256;  // partial sums at most

// Sums of the partial sums part[nblk][2 E + 2] (P_e, counts, sum of lse^2, N), the loss
// and the counts; by one workgroup of 256 threads.
__device__ void balance_finish(const BalanceP &p, int nblk, float *sp, int *sc) {
  const int tid = threadIdx.x, ld = 2 * p.E + 2;
  const int col = tid & 63, sl = tid >> 6;
  __syncthreads();
  // thread (col, sl): its quarter of the blocks, in order; then the quarters in order
  double ps = 0.0, zs = 0.0;
  int cs = 0, ns = 0;
  const int b0 = (int)((int64_t)nblk * sl / 4), b1 = (int)((int64_t)nblk * (sl + 1) / 4);
  for (int b = b0; b < b1; ++b) {
    const float *q = p.part + (int64_t)b * ld;
    if (col < p.E) {
      ps += q[col];
      cs += __float_as_int(q[p.E + col]);
    }
    if (col == 0) {
      zs += q[2 * p.E];
      ns += __float_as_int(q[2 * p.E + 1]);
    }
  }
  double *const dp = reinterpret_cast<double *>(sp);  // [4][64], then 4 of z
  dp[tid] = ps;
  sc[tid] = cs;
  if (col == 0) {
    dp[256 + sl] = zs;
    sc[256 + sl] = ns;
  }
  __syncthreads();
  if (tid < 64) {
    double a = dp[tid], z = dp[256];
    int c = sc[tid], N = sc[256];
    for (int s = 1; s < 4; ++s) {
      a += dp[64 * s + tid];
      c += sc[64 * s + tid];
      z += dp[256 + s];
      N += sc[256 + s];
    }
    double l = tid < p.E ? a * c : 0.0;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) l += __shfl_xor(l, o, 64);
    if (tid < p.E) p.counts[tid] = c;
    if (tid == 0) {
      p.counts[p.E] = N;
      const double n = N;
      p.loss[0] = N > 0 ? (float)(p.E * l / (2.0 * n * n)) : 0.0f;
      p.loss[1] = N > 0 ? (float)(z / n) : 0.0f;
    }
  }
}

__global__ __launch_bounds__(256) void balance_finish_kernel(BalanceP p, int nblk) {
  __shared__ __align__(16) float sp[2 * 260];
  __shared__ int sc[260];
  balance_finish(p, nblk, sp, sc);
}

// A workgroup takes tiles of 32 tokens: its four waves split d (64 values in turn), and
// the waves' logits are added in LDS in wave order. EF: experts / 16, rounded up.
template <int ND, int WD, int EF>
__global__ __launch_bounds__(256) void balance_fwd_kernel(BalanceP p) {
  constexpr int LD = 16 * EF + 4;  // a token's logits in LDS
  __shared__ __align__(16) float sl[4][kFwdTokens * LD];
  __shared__ float sz[kFwdTokens];
  __shared__ int scnt[65];
  static_assert(sizeof(sl) >= 5200, "balance_finish's sums");
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int i16 = lane & 15, g = lane >> 4;
  if (tid < 65) scnt[tid] = 0;
  float psum = 0.0f, zsum = 0.0f;  // thread e: the workgroup's sum of probs; thread 0: of lse^2
  for (int64_t tile = blockIdx.x; tile < p.tiles; tile += gridDim.x) {
    const int64_t t0 = tile * kFwdTokens;
    f32x4_v acc[2][EF];
#pragma unroll
    for (int a = 0; a < 2; ++a)
#pragma unroll
      for (int b = 0; b < EF; ++b) acc[a][b] = f32x4_v{0.0f, 0.0f, 0.0f, 0.0f};
    for (int k0 = wave * 64; k0 < p.d; k0 += 256) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int k = k0 + 32 * h + 8 * g;
        bf16x8_v fa[2][kPieces<ND>], fb[EF][kPieces<WD>];
#pragma unroll
        for (int a = 0; a < 2; ++a) {
          const int64_t t = t0 + 16 * a + i16;
          const bool ok = t < p.T && k < p.d;
          load_pieces<ND>(p.n, ok ? t * p.d + k : 0, ok, fa[a]);
        }
#pragma unroll
        for (int b = 0; b < EF; ++b) {
          const int e = 16 * b + i16;
          const bool ok = e < p.E && k < p.d;
          load_pieces<WD>(p.wr, ok ? (int64_t)e * p.d + k : 0, ok, fb[b]);
        }
#pragma unroll
        for (int a = 0; a < 2; ++a)
#pragma unroll
          for (int b = 0; b < EF; ++b) acc[a][b] = mul_pieces(fb[b], fa[a], acc[a][b]);
      }
    }
    // lane: token 16 a + i16, experts 16 b + 4 g ..
    __syncthreads();  // the last tile's readers are done
#pragma unroll
    for (int a = 0; a < 2; ++a)
#pragma unroll
      for (int b = 0; b < EF; ++b)
        *reinterpret_cast<f32x4_v *>(&sl[wave][(16 * a + i16) * LD + 16 * b + 4 * g]) = acc[a][b];
    __syncthreads();
    // 8 lanes per token, experts j, j + 8, ...
    const int tl = tid >> 3, j = tid & 7;
    const int64_t t = t0 + tl;
    const bool live = t < p.T && (!p.mask || p.mask[t] != 0);
    float l[2 * EF], m = -INFINITY, sum = 0.0f;
#pragma unroll
    for (int i = 0; i < 2 * EF; ++i) {
      const int e = j + 8 * i;
      float v = sl[0][tl * LD + e];
#pragma unroll
      for (int u = 1; u < 4; ++u) v += sl[u][tl * LD + e];
      l[i] = v;
      if (e < p.E) m = v > m || v != v ? v : m;  // (a NaN stays)
    }
#pragma unroll
    for (int o = 1; o < 8; o *= 2) {
      const float v = __shfl_xor(m, o, 64);
      m = v > m || v != v ? v : m;
    }
#pragma unroll
    for (int i = 0; i < 2 * EF; ++i) {
      l[i] = j + 8 * i < p.E ? expf(l[i] - m) : 0.0f;
      sum += l[i];
    }
#pragma unroll
    for (int o = 1; o < 8; o *= 2) sum += __shfl_xor(sum, o, 64);
    const float inv = 1.0f / sum, lse = live ? m + logf(sum) : 0.0f;
    __syncthreads();  // logits read
#pragma unroll
    for (int i = 0; i < 2 * EF; ++i) {
      const int e = j + 8 * i;
      const float v = live ? l[i] * inv : 0.0f;
      sl[0][tl * LD + e] = v;
      if (t < p.T && e < p.E) p.probs[t * p.E + e] = v;
    }
    if (j == 0) {
      sz[tl] = lse * lse;
      if (t < p.T) p.lse[t] = lse;
      if (live) {  // (integer counts: any order gives the same)
        const int a = p.sel[2 * t], b = p.sel[2 * t + 1];
        if (a >= 0 && a < p.E) atomicAdd(&scnt[a], 1);
        if (b >= 0 && b < p.E && b != a) atomicAdd(&scnt[b], 1);
        atomicAdd(&scnt[64], 1);
      }
    }
    __syncthreads();
    if (tid < p.E) {
      float s = 0.0f;
      for (int i = 0; i < kFwdTokens; ++i) s += sl[0][i * LD + tid];
      psum += s;
    }
    if (tid == 0) {
      float s = 0.0f;
      for (int i = 0; i < kFwdTokens; ++i) s += sz[i];
      zsum += s;
    }
  }
  __syncthreads();  // counts
  float *const q = p.part + (int64_t)blockIdx.x * (2 * p.E + 2);
  if (tid < p.E) {
    q[tid] = psum;
    q[p.E + tid] = __int_as_float(scnt[tid]);
  }
  if (tid == 0) {
    q[2 * p.E] = zsum;
    q[2 * p.E + 1] = __int_as_float(scnt[64]);
  }
  if (gridDim.x == 1) {  // a single workgroup finishes by itself
    __threadfence_block();
    balance_finish(p, 1, &sl[0][0], reinterpret_cast<int *>(&sl[0][0]) + 1040);
  }
}

constexpr int kBwdTokens = 32;
constexpr int kBwdCols = 128;

// A workgroup takes kBwdCols columns and a split's tokens, 32 at a time. dl of a tile is
// formed in LDS in three bf16 pieces, [token][expert] for dn = dl Wr and [expert][token]
// for dWr = dl^T n; Wr's fragments stay in registers for all tiles, dWr's sums too. n's
// fragments (tokens along k) are transposing LDS reads of the rows.
template <int ND, int WD, int EF>
__global__ __launch_bounds__(256) void balance_bwd_kernel(BalanceP p) {
  constexpr int PN = kPieces<ND>, PW = kPieces<WD>, KE = (EF + 1) / 2;
  constexpr int LE = 32 * KE + 8;  // [token][expert] row
  constexpr int LT = kBwdTokens + 8;
  constexpr int LN = kBwdCols + 16;
  __shared__ __align__(16) uint16_t s_te[3][kBwdTokens * LE];
  __shared__ __align__(16) uint16_t s_et[3][16 * EF * LT];
  __shared__ __align__(16) uint16_t s_n[PN][kBwdTokens * LN];
  __shared__ float s_f[64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int i16 = lane & 15, g = lane >> 4;
  const int nchunk = (p.d + kBwdCols - 1) / kBwdCols;
  const int chunk = blockIdx.x % nchunk, split = blockIdx.x / nchunk;
  const int c0 = chunk * kBwdCols, cw = c0 + 32 * wave;  // the wave's 32 columns
  const int64_t tile0 = p.tiles * split / p.splits, tile1 = p.tiles * (split + 1) / p.splits;
  const int N = p.counts[p.E];
  const float rn = N > 0 ? 1.0f / (float)N : 0.0f;
  const float cb = p.coef * p.E * rn, cz = 2.0f * p.z_coef * rn;
  if (tid < 64) s_f[tid] = tid < p.E ? (float)p.counts[tid] * 0.5f * rn : 0.0f;
  for (int i = tid; i < kBwdTokens * LE; i += 256) s_te[0][i] = s_te[1][i] = s_te[2][i] = 0;
  for (int i = tid; i < 16 * EF * LT; i += 256) s_et[0][i] = s_et[1][i] = s_et[2][i] = 0;

  // Wr fragments: rows columns cw + 16 b + i16, k experts 32 k + 8 g ..
  bf16x8_v fw[2][KE][PW];
#pragma unroll
  for (int b = 0; b < 2; ++b)
#pragma unroll
    for (int k = 0; k < KE; ++k) {
      typedef __attribute__((ext_vector_type(8))) uint16_t u16x8_v;
      u16x8_v v[PW];
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        const int e = 32 * k + 8 * g + c, col = cw + 16 * b + i16;
        float x = 0.0f;
        if (e < p.E && col < p.d) {
          const int64_t at = (int64_t)e * p.d + col;
          if constexpr (WD == LC_FP32) x = static_cast<const float *>(p.wr)[at];
          else if constexpr (WD == LC_BF16) x = bf2f(static_cast<const bf16_t *>(p.wr)[at]);
          else x = (float)static_cast<const _Float16 *>(p.wr)[at];
        }
        uint16_t s[PW];
        split_bf16<PW>(x, s);
#pragma unroll
        for (int i = 0; i < PW; ++i) v[i][c] = s[i];
      }
#pragma unroll
      for (int i = 0; i < PW; ++i) fw[b][k][i] = __builtin_bit_cast(bf16x8_v, v[i]);
    }
  f32x4_v aw[EF][2];  // dWr: experts 16 a + i16, columns 16 b + 4 g ..
#pragma unroll
  for (int a = 0; a < EF; ++a)
#pragma unroll
    for (int b = 0; b < 2; ++b) aw[a][b] = f32x4_v{0.0f, 0.0f, 0.0f, 0.0f};

  for (int64_t tile = tile0; tile < tile1; ++tile) {
    const int64_t t0 = tile * kBwdTokens;
    __syncthreads();  // the last tile's fragments are read
    {  // dl: 8 lanes per token, experts 8 j .. 8 j + 7
      const int tl = tid >> 3, j = tid & 7;
      const int64_t t = t0 + tl;
      const bool live = t < p.T && (!p.mask || p.mask[t] != 0);
      float pr[8], dot = 0.0f;
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        const int e = 8 * j + c;
        pr[c] = live && e < p.E ? p.probs[t * p.E + e] : 0.0f;
        dot += pr[c] * s_f[e];
      }
#pragma unroll
      for (int o = 1; o < 8; o *= 2) dot += __shfl_xor(dot, o, 64);
      const float z = live ? cz * p.lse[t] : 0.0f;
      int e0 = -1, e1 = -1;
      float g0 = 0.0f, g1 = 0.0f;
      if (live && p.dw) {
        e0 = p.sel[2 * t];
        e1 = p.sel[2 * t + 1];
        if (e0 < 0 || e0 >= p.E) e0 = -1;
        if (e1 < 0 || e1 >= p.E || e1 == p.sel[2 * t]) e1 = -1;
        const float w0 = e0 >= 0 ? p.w[2 * t] : 0.0f, w1 = e1 >= 0 ? p.w[2 * t + 1] : 0.0f;
        const float d0 = e0 >= 0 ? p.dw[2 * t] : 0.0f, d1 = e1 >= 0 ? p.dw[2 * t + 1] : 0.0f;
        const float inner = w0 * d0 + w1 * d1;
        g0 = w0 * (d0 - inner);
        g1 = w1 * (d1 - inner);
      }
      if (8 * j < 16 * EF) {
#pragma unroll
        for (int c = 0; c < 8; ++c) {
          const int e = 8 * j + c;
          float v = pr[c] * (cb * (s_f[e] - dot) + z);
          v += e == e0 ? g0 : e == e1 ? g1 : 0.0f;
          if (!live || e >= p.E) v = 0.0f;
          uint16_t s[3];
          split_bf16<3>(v, s);
#pragma unroll
          for (int i = 0; i < 3; ++i) {
            s_te[i][tl * LE + e] = s[i];
            s_et[i][e * LT + tl] = s[i];
          }
        }
      }
    }
    if (p.dwr) {  // n: 16 lanes per token, 8 columns each
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int tl = 16 * u + (tid >> 4), c = 8 * (tid & 15);
        const int64_t t = t0 + tl;
        const bool ok = t < p.T && c0 + c < p.d && (!p.mask || p.mask[t] != 0);
        bf16x8_v f[PN];
        load_pieces<ND>(p.n, ok ? t * p.d + c0 + c : 0, ok, f);
#pragma unroll
        for (int i = 0; i < PN; ++i) *reinterpret_cast<bf16x8_v *>(&s_n[i][tl * LN + c]) = f[i];
      }
    }
    __syncthreads();
    if (p.dwr) {
      bf16x8_v fn[2][PN];  // columns 16 b + i16, tokens 8 g ..
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < PN; ++i) {
          // each 16 lanes: rows 8 g + i16 / 4 (and + 4), columns 4 (i16 % 4) ..
          lds_t *q = LDS_AS(char, &s_n[i][(8 * g + (i16 >> 2)) * LN + 32 * wave + 16 * b + 4 * (i16 & 3)]);
          typedef __attribute__((address_space(3))) s16x4_v lds_v4;
          const s16x4_v v[2] = {__builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4 *)q),
                                __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4 *)(q + 4 * LN * 2))};
          fn[b][i] = __builtin_bit_cast(bf16x8_v, v);
        }
#pragma unroll
      for (int a = 0; a < EF; ++a) {
        bf16x8_v fd[3];
#pragma unroll
        for (int i = 0; i < 3; ++i)
          fd[i] = *reinterpret_cast<const bf16x8_v *>(&s_et[i][(16 * a + i16) * LT + 8 * g]);
#pragma unroll
        for (int b = 0; b < 2; ++b) aw[a][b] = mul_pieces(fn[b], fd, aw[a][b]);
      }
    }
    if (p.dn) {
#pragma unroll
      for (int a = 0; a < 2; ++a) {  // tokens 16 a + i16
        bf16x8_v fd[KE][3];
#pragma unroll
        for (int k = 0; k < KE; ++k)
#pragma unroll
          for (int i = 0; i < 3; ++i)
            fd[k][i] = *reinterpret_cast<const bf16x8_v *>(&s_te[i][(16 * a + i16) * LE + 32 * k + 8 * g]);
        const int64_t t = t0 + 16 * a + i16;
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          const int col = cw + 16 * b + 4 * g;
          const bool ok = t < p.T && col < p.d;
          const int64_t at = ok ? t * p.d + col : 0;
          float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
          if (ok && p.dres) x = load4_dt(p.dres, at, p.dres_dt);
          f32x4_v s = f32x4_v{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
          for (int k = 0; k < KE; ++k) s = mul_pieces(fw[b][k], fd[k], s);
          if (ok) store4_dt(p.dn, at, p.dn_dt, x.x + s[0], x.y + s[1], x.z + s[2], x.w + s[3]);
        }
      }
    }
  }
  if (p.dwr) {
    float *const out = p.splits > 1 ? p.part + (int64_t)split * p.E * p.d : p.dwr;
    const bool add = p.splits == 1 && !p.store;
#pragma unroll
    for (int a = 0; a < EF; ++a)
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const int e = 16 * a + i16, col = cw + 16 * b + 4 * g;
        if (e >= p.E || col >= p.d) continue;
        float4 *q = reinterpret_cast<float4 *>(out + (int64_t)e * p.d + col);
        float4 v = make_float4(aw[a][b][0], aw[a][b][1], aw[a][b][2], aw[a][b][3]);
        if (add) {
          const float4 o = *q;
          v = make_float4(o.x + v.x, o.y + v.y, o.z + v.z, o.w + v.w);
        }
        *q = v;
      }
  }
}

// dWr: the splits' sums, added in order
__global__ __launch_bounds__(256) void balance_dwr_kernel(BalanceP p) {
  const int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x, n4 = (int64_t)p.E * p.d / 4;
  if (q >= n4) return;
  const float4 *src = reinterpret_cast<const float4 *>(p.part) + q;
  float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  int b = 0;
  for (; b + 8 <= p.splits; b += 8) {  // (eight loads in flight)
    float4 v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = src[(b + i) * n4];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      s.x += v[i].x; s.y += v[i].y; s.z += v[i].z; s.w += v[i].w;
    }
  }
  for (; b < p.splits; ++b) {
    const float4 v = src[b * n4];
    s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
  }
  float4 *out = reinterpret_cast<float4 *>(p.dwr) + q;
  if (!p.store) {
    const float4 o = *out;
    s.x += o.x; s.y += o.y; s.z += o.z; s.w += o.w;
  }
  *out = s;
}

// Parts of the tokens in the backward: enough workgroups to fill the chip twice
int bwd_splits(int64_t T, int64_t d) {
  const int64_t chunks = (d + kBwdCols - 1) / kBwdCols, tiles = (T + kBwdTokens - 1) / kBwdTokens;
  const int64_t want = (512 + chunks - 1) / chunks;
  return (int)(tiles < 1 ? 1 : tiles < want ? tiles : want);
}

size_t balance_scratch(int64_t T, int64_t d, int64_t E) {
  const size_t f = (size_t)kFwdBlocks * (2 * E + 2) * 4;
  const int s = bwd_splits(T, d);
  const size_t b = s > 1 ? (size_t)s * E * d * 4 : 0;
  return f > b ? f : b;
}

template <typename F>
void with_experts(int E, F f) {
  if (E <= 16) f(std::integral_constant<int, 1>{});
  else if (E <= 32) f(std::integral_constant<int, 2>{});
  else if (E <= 48) f(std::integral_constant<int, 3>{});
  else f(std::integral_constant<int, 4>{});
}

}  // namespace

static lc_status check_balance(const lc_moe_balance_args &a, bool backward) {
  if (a.T < 0 || a.d <= 0 || a.E < 2 || a.E > 64)
    return fail(LC_ERR_INVALID_ARG, "moe balance: need T >= 0, d > 0 and 2 <= E <= 64");
  if (a.T >= ((int64_t)1 << 30)) return fail(LC_ERR_UNSUPPORTED, "moe balance: too many tokens");
  if (a.d % 8) return fail(LC_ERR_UNSUPPORTED, "moe balance: d %% 8 != 0");
  if (!valid_dtype(a.n_dtype) || !valid_dtype(a.w_dtype))
    return fail(LC_ERR_INVALID_ARG, "moe balance: unknown dtype");
  if (!a.counts || !aligned16(a.counts) || (!backward && (!a.loss || !aligned16(a.loss))))
    return fail(LC_ERR_INVALID_ARG, "moe balance: null or unaligned counts or loss");
  if (a.T > 0) {
    if (!a.n || !a.wr || !a.sel || !a.probs || !a.lse || !aligned16(a.n) || !aligned16(a.wr) ||
        !aligned16(a.sel) || !aligned16(a.probs) || !aligned16(a.lse))
      return fail(LC_ERR_INVALID_ARG, "moe balance: null or unaligned pointer");
  }
  if (backward) {
    if (!a.w != !a.dw) return fail(LC_ERR_INVALID_ARG, "moe balance: w and dw come together");
    if (!aligned16(a.w) || !aligned16(a.dw) || !aligned16(a.dn) || !aligned16(a.dres) || !aligned16(a.dwr_accum))
      return fail(LC_ERR_INVALID_ARG, "moe balance: unaligned pointer");
    if ((a.dn && !valid_dtype(a.dn_dtype)) || (a.dres && !valid_dtype(a.dres_dtype)))
      return fail(LC_ERR_INVALID_ARG, "moe balance: unknown dn or dres dtype");
    if (!(a.coef == a.coef) || !(a.z_coef == a.z_coef))
      return fail(LC_ERR_INVALID_ARG, "moe balance: coefficients must be numbers");
  }
  const bool need = !backward || (a.dwr_accum && bwd_splits(a.T, a.d) > 1);
  if (need && (!a.scratch || !aligned16(a.scratch)))
    return fail(LC_ERR_INVALID_ARG, "moe balance: null or unaligned scratch");
  if (need && a.scratch_bytes < balance_scratch(a.T, a.d, a.E))
    return fail(LC_ERR_WORKSPACE, "moe balance: scratch too small");
  return LC_OK;
}

static BalanceP balance_params(const lc_moe_balance_args &a) {
  BalanceP p{};
  p.n = a.n;
  p.wr = a.wr;
  p.dres = a.dres;
  p.sel = a.sel;
  p.mask = a.mask;
  p.probs = a.probs;
  p.lse = a.lse;
  p.loss = a.loss;
  p.counts = a.counts;
  p.w = a.w;
  p.dw = a.dw;
  p.dn = a.dn;
  p.dwr = a.dwr_accum;
  p.part = static_cast<float *>(a.scratch);
  p.T = a.T;
  p.d = a.d;
  p.E = a.E;
  p.dn_dt = a.dn_dtype;
  p.dres_dt = a.dres_dtype;
  p.coef = a.coef;
  p.z_coef = a.z_coef;
  p.store = a.store_dwr == 1;
  return p;
}

static lc_status balance_forward(const lc_moe_balance_args &a, hipStream_t s) {
  LC_TRY(check_balance(a, false));
  BalanceP p = balance_params(a);
  p.tiles = (a.T + kFwdTokens - 1) / kFwdTokens;
  const int nblk = (int)(p.tiles < kFwdBlocks ? p.tiles : kFwdBlocks);
  if (nblk > 0) {
    with_dtype(a.n_dtype, [&](auto nd) {
      with_dtype(a.w_dtype, [&](auto wd) {
        with_experts(a.E, [&](auto ef) {
          hipLaunchKernelGGL((balance_fwd_kernel<decltype(nd)::value, decltype(wd)::value, decltype(ef)::value>),
                             dim3((unsigned)nblk), dim3(256), 0, s, p);
        });
      });
    });
    LC_TRY(check_launch("balance_fwd_kernel"));
  }
  if (nblk == 1) return LC_OK;
  hipLaunchKernelGGL(balance_finish_kernel, dim3(1), dim3(256), 0, s, p, nblk);
  return check_launch("balance_finish_kernel");
}

static lc_status balance_backward(const lc_moe_balance_args &a, hipStream_t s) {
  LC_TRY(check_balance(a, true));
  if (!a.dn && !a.dwr_accum) return LC_OK;
  BalanceP p = balance_params(a);
  p.tiles = (a.T + kBwdTokens - 1) / kBwdTokens;
  p.splits = bwd_splits(a.T, a.d);
  if (a.T == 0) {
    if (a.dwr_accum && p.store) return zero_fill_launch(a.dwr_accum, (size_t)a.E * a.d, s);
    return LC_OK;
  }
  const unsigned grid = (unsigned)p.splits * (unsigned)((a.d + kBwdCols - 1) / kBwdCols);
  with_dtype(a.n_dtype, [&](auto nd) {
    with_dtype(a.w_dtype, [&](auto wd) {
      with_experts(a.E, [&](auto ef) {
        hipLaunchKernelGGL((balance_bwd_kernel<decltype(nd)::value, decltype(wd)::value, decltype(ef)::value>),
                           dim3(grid), dim3(256), 0, s, p);
      });
    });
  });
  LC_TRY(check_launch("balance_bwd_kernel"));
  if (!a.dwr_accum || p.splits == 1) return LC_OK;
  hipLaunchKernelGGL(balance_dwr_kernel, dim3(ceil_div((size_t)a.E * a.d / 4, 256)), dim3(256), 0, s, p);
  return check_launch("balance_dwr_kernel");
}

}  // namespace lc

extern "C" {

lc_status lc_moe_balance_forward(const lc_moe_balance_args *args, void *stream) {
  if (!args) return lc::fail(LC_ERR_INVALID_ARG, "moe balance: null args");
  return lc::balance_forward(*args, static_cast<hipStream_t>(stream));
}

lc_status lc_moe_balance_backward(const lc_moe_balance_args *args, void *stream) {
  if (!args) return lc::fail(LC_ERR_INVALID_ARG, "moe balance: null args");
  return lc::balance_backward(*args, static_cast<hipStream_t>(stream));
}

size_t lc_moe_balance_scratch_bytes(int64_t T, int32_t d, int32_t E) {
  if (T < 0 || T >= ((int64_t)1 << 30) || d <= 0 || E < 2 || E > 64) return 0;
  return lc::balance_scratch(T, d, E);
}

}  // extern "C"
