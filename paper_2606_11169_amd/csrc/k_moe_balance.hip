// Balance and z loss of a top-2 router, per-expert counts, and the gradients of both
// through the router's product (gfx950).
//
//   l = n Wr^T, p = softmax(l), f_e = counts[e] / (2N), P_e = sum_t p[t, e] / N
//   loss = (E sum_e f_e P_e, sum_t lse[t]^2 / N)
//   dl[t, e] = coef E / N p (f_e - sum f p) + 2 z_coef / N lse p + the pair's gate gradient
//   dn = dres + dl Wr, dWr = dl^T n
//
// The three products run on the bf16 matrix cores for every type: a value is split into
// bf16 pieces of 8 bits (fp16 into 2, fp32 into 3, exactly), and the pieces' products are added
// in fp32, but for second by third ones: two of at most 2^-25 of the values' powers of two
// (fp16 by fp32: one of 2^-24). So a bf16 router pays one instruction where fp32 ones would
// take sixteen times as long. dl is fp32 and takes three pieces.
//
// Bound: HBM, by n (forward), and n, dres and dn (backward). bf16, us: 4096 tokens x 2048, 8
// experts, forward 7.1 + 3.0 (sums), backward 21.9 + 4.2 (dWr's parts); 16411 x 4096, 64 experts,
// 52.3 + 5.3 (n at 2.6 TB/s) and 100.8 + 6.3 (reads and writes past L2, each column chunk's
// probs among them, at 4.8 TB/s, a copy's rate; of 4096 x 2048 at 4.1). 8192 tokens x 4096, 64
// experts, forward and backward with fp32 n and Wr 68, 114, fp16 36, 106, bf16 33, 93.
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

// a and b as P bf16 pieces each, largest first, in pairs (a low). Three, of fp32 values: each
// is what is left rounded to nearest, at most 2^-8, then 2^-17 of the value's power of two;
// exact down to 2^-109, as the last one's step is 2^-133 at least. (The first is clamped: what
// rounds to infinity is cut.) Two, of fp16 values: the upper 8 bits and the rest, at most 2^-7.
// A NaN of any payload, and in two or three pieces an infinity, leaves a NaN among the pieces.
template <int P>
__device__ __forceinline__ void split_bf16(float a, float b, uint32_t (&out)[P]) {
  typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_v;
  constexpr float MOST = 3.3895313892515355e38f;  // bf16's largest
#pragma unroll
  for (int i = 0; i < P; ++i) {
    if constexpr (P == 3) {
      const float u = i == 0 ? __builtin_amdgcn_fmed3f(a, -MOST, MOST) : a, v = i == 0 ? __builtin_amdgcn_fmed3f(b, -MOST, MOST) : b;
      out[i] = __builtin_bit_cast(uint32_t, bf16x2_v{(__bf16)u, (__bf16)v});
    } else {
      out[i] = (__float_as_uint(a) >> 16) | (__float_as_uint(b) & 0xFFFF0000u);
    }
    a -= __uint_as_float(out[i] << 16);
    b -= __uint_as_float(out[i] & 0xFFFF0000u);
  }
}

// 8 values of type DT as they lie in memory
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4_v;
template <int DT>
struct Raw8 {
  static constexpr int W = DT == LC_FP32 ? 2 : 1;
  u32x4_v w[W];
  // byte offset `off` of a buffer; zeros past its end
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t rs, uint32_t off) {
#pragma unroll
    for (int i = 0; i < W; ++i)
      w[i] = __builtin_bit_cast(u32x4_v, __builtin_amdgcn_raw_buffer_load_b128(rs, (int)(off + 16 * i), 0, 0));
  }
  __device__ __forceinline__ float value(int c) const {
    if constexpr (DT == LC_FP32) return __uint_as_float(w[c >> 2][c & 3]);
    else if constexpr (DT == LC_BF16) return __uint_as_float(w[0][c >> 1] << 16 * (1 - (c & 1)) & 0xFFFF0000u);
    else return (float)__builtin_bit_cast(_Float16, (uint16_t)(w[0][c >> 1] >> 16 * (c & 1)));
  }
  // as bf16 pieces
  __device__ __forceinline__ void pieces(bf16x8_v (&out)[kPieces<DT>]) const {
    constexpr int P = kPieces<DT>;
    if constexpr (P == 1) {
      out[0] = __builtin_bit_cast(bf16x8_v, w[0]);
    } else {
      u32x4_v v[P];
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        uint32_t s[P];
        split_bf16<P>(value(2 * c), value(2 * c + 1), s);
#pragma unroll
        for (int i = 0; i < P; ++i) v[i][c] = s[i];
      }
#pragma unroll
      for (int i = 0; i < P; ++i) out[i] = __builtin_bit_cast(bf16x8_v, v[i]);
    }
  }
};

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

constexpr int kFwdBlocks = 512;  // workgroups of the forward, and partial sums, at most

// Sums of the partial sums part[2 E + 2][kFwdBlocks] (sums of probs, counts, sum of lse^2,
// N), the loss and the counts; by one workgroup, 8 lanes for each entry, every one of them
// reading whole lines of blocks in turn. In 64 bits: once per call.
__global__ __launch_bounds__(1024) void balance_finish_kernel(BalanceP p, int nblk) {
  __shared__ double sums[136];
  const int lane = threadIdx.x & 63, j = threadIdx.x & 7, n = 2 * p.E + 2;
  for (int e = threadIdx.x >> 3; e < n; e += 128) {
    const bool whole = (e >= p.E && e < 2 * p.E) || e == n - 1;  // a count: an integer's bits
    double s = 0.0;
    for (int b0 = 0; b0 < nblk; b0 += 256) {
      float4 v[8];
#pragma unroll
      for (int u = 0; u < 8; ++u)
        v[u] = *reinterpret_cast<const float4 *>(p.part + e * kFwdBlocks + b0 + 32 * u + 4 * j);
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const float w[4] = {v[u].x, v[u].y, v[u].z, v[u].w};
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (b0 + 32 * u + 4 * j + i < nblk) s += whole ? (double)__float_as_int(w[i]) : (double)w[i];
      }
    }
#pragma unroll
    for (int o = 1; o < 8; o *= 2) s += __shfl_xor(s, o, 64);
    if (j == 0) sums[e] = s;
  }
  __syncthreads();
  if (threadIdx.x >= 64) return;
  const int e = min(lane, p.E - 1);
  const double N = sums[n - 1];
  double l = lane < p.E ? sums[e] * sums[p.E + e] : 0.0;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) l += __shfl_xor(l, o, 64);
  if (lane < p.E) p.counts[lane] = (int)sums[p.E + e];
  if (lane == 0) {
    p.counts[p.E] = (int)N;
    p.loss[0] = N > 0.0 ? (float)(p.E * l / (2.0 * N * N)) : 0.0f;
    p.loss[1] = N > 0.0 ? (float)(sums[n - 2] / N) : 0.0f;
  }
}

// A workgroup of 8 waves takes tiles of 16 MT tokens. The waves split d, 64 values (whole
// lines of bf16) in turn, the next ones' loads under way while one multiplies; their logits
// are added in LDS in a fixed order. Large tiles read Wr (from L2) less often, small ones
// fill the chip at fewer tokens. EF: experts / 16, rounded up.
template <int ND, int WD, int EF, int MT>
__global__ __launch_bounds__(512) void balance_fwd_kernel(BalanceP p) {
  constexpr int TT = 16 * MT, LD = 16 * EF + 4;  // tokens; a token's logits in LDS
  __shared__ __align__(16) float sl[4][TT * LD];
  __shared__ float sz[TT], sps[8][64];
  __shared__ int scnt[65];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int i16 = lane & 15, g = lane >> 4;
  if (tid < 65) scnt[tid] = 0;
  // thread e: the workgroup's sum of probs; thread 0: of lse^2. In 64 bits from tile to tile: a
  // workgroup takes any number of them (in fp32 the losses of 2^24 like tokens were off by 530
  // and 51 * 2^-24)
  double psum = 0.0, zsum = 0.0;
  for (int64_t tile = blockIdx.x; tile < p.tiles; tile += gridDim.x) {
    const int64_t t0 = tile * TT;
    f32x4_v acc[MT][EF];
#pragma unroll
    for (int a = 0; a < MT; ++a)
#pragma unroll
      for (int b = 0; b < EF; ++b) acc[a][b] = f32x4_v{0.0f, 0.0f, 0.0f, 0.0f};
    // Steps of 32 of d; n's rows (from HBM) are read four steps ahead (two where registers
    // end), Wr's (from L2) two.
    // A wave's step s: values 512 (s / 2) + 64 wave + 32 (s % 2) ..
    constexpr int AHEAD = MT * EF > 16 ? 2 : 4;
    Raw8<ND> ra[AHEAD][MT];
    Raw8<WD> rb[2][EF];
    // in a workgroup that starts at 0; others start elsewhere and wrap round, so that they do
    // not all read the same lines of Wr at once.
    const int turns = (p.d + 511) / 512, start = blockIdx.x % turns;
    auto first = [&](int s) {
      const int turn = s >> 1;
      return turn < turns ? 512 * (turn + start - (turn + start >= turns ? turns : 0)) + 64 * wave + 32 * (s & 1) + 8 * g : p.d;
    };
    constexpr int NS = ND == LC_FP32 ? 4 : 2, WS = WD == LC_FP32 ? 4 : 2;
    const int rows = (int)min(p.T - t0, (int64_t)TT);
    const auto rn = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<char *>(static_cast<const char *>(p.n) + t0 * p.d * NS), 0, rows * p.d * NS, 0x00020000);
    const auto rw = __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p.wr), 0, p.E * p.d * WS, 0x00020000);
    auto fetch_a = [&](Raw8<ND> (&x)[MT], int k) {
#pragma unroll
      for (int a = 0; a < MT; ++a)
        x[a].load(rn, k < p.d ? (uint32_t)((16 * a + i16) * p.d + k) * NS : 0x80000000u);
    };
    auto fetch_b = [&](Raw8<WD> (&x)[EF], int k) {
#pragma unroll
      for (int b = 0; b < EF; ++b) x[b].load(rw, k < p.d ? (uint32_t)((16 * b + i16) * p.d + k) * WS : 0x80000000u);
    };
    auto multiply = [&](const Raw8<ND> (&x)[MT], const Raw8<WD> (&y)[EF]) {
      bf16x8_v fa[MT][kPieces<ND>];
#pragma unroll
      for (int a = 0; a < MT; ++a) x[a].pieces(fa[a]);
#pragma unroll
      for (int b = 0; b < EF; ++b) {
        bf16x8_v fb[kPieces<WD>];
        y[b].pieces(fb);
#pragma unroll
        for (int a = 0; a < MT; ++a) acc[a][b] = mul_pieces(fb, fa[a], acc[a][b]);
      }
    };
#pragma unroll
    for (int s = 0; s < AHEAD; ++s) fetch_a(ra[s], first(s));
#pragma unroll
    for (int s = 0; s < 2; ++s) fetch_b(rb[s], first(s));
    for (int s0 = 0; s0 < 2 * turns; s0 += 4) {
#pragma unroll
      for (int u = 0; u < 4; ++u) {  // (steps past the last: zeros)
        multiply(ra[u % AHEAD], rb[u & 1]);
        fetch_b(rb[u & 1], first(s0 + u + 2));
        fetch_a(ra[u % AHEAD], first(s0 + u + AHEAD));
      }
    }
    // lane: token 16 a + i16, experts 16 b + 4 g ..; waves 4 to 7 hand theirs to waves 0 to 3
    auto place = [&](int w, int a, int b) { return reinterpret_cast<f32x4_v *>(&sl[w][(16 * a + i16) * LD + 16 * b + 4 * g]); };
    __syncthreads();  // the last tile's readers are done
    if (wave >= 4) {
#pragma unroll
      for (int a = 0; a < MT; ++a)
#pragma unroll
        for (int b = 0; b < EF; ++b) *place(wave - 4, a, b) = acc[a][b];
    }
    constexpr bool MANY = kPieces<ND> + kPieces<WD> > 2;
    int odd = 0;  // a NaN among the products
    if constexpr (MANY) {
#pragma unroll
      for (int a = 0; a < MT; ++a)
#pragma unroll
        for (int b = 0; b < EF; ++b)
#pragma unroll
          for (int c = 0; c < 4; ++c) odd |= acc[a][b][c] != acc[a][b][c] ? 1 : 0;
      odd = __syncthreads_or(odd);
    } else {
      __syncthreads();
    }
    if (wave < 4) {
#pragma unroll
      for (int a = 0; a < MT; ++a)
#pragma unroll
        for (int b = 0; b < EF; ++b) *place(wave, a, b) = acc[a][b] + *place(wave, a, b);
    }
    __syncthreads();
    // Pieces leave a NaN where a value is infinite (times a piece of 0, or of the other sign):
    // a wave for each such logit adds the values themselves. (8192 tokens x 4096, 64 experts, fp32:
    // 70 us, one token of NaN 114, all of them 600.)
    if constexpr (MANY) {
      if (odd) {
        for (int tl = 0; tl < rows; ++tl) {
          if (p.mask && p.mask[t0 + tl] == 0) continue;
          for (int e = wave; e < p.E; e += 8) {
            const int at = tl * LD + e;
            float v = sl[0][at] + sl[1][at] + sl[2][at] + sl[3][at];
            if (v == v) continue;
            v = 0.0f;
            for (int k = 8 * lane; k < p.d; k += 512) {
              Raw8<ND> x;
              Raw8<WD> y;
              x.load(rn, (uint32_t)(tl * p.d + k) * NS);
              y.load(rw, (uint32_t)(e * p.d + k) * WS);
#pragma unroll
              for (int c = 0; c < 8; ++c) v = fmaf(x.value(c), y.value(c), v);
            }
            v = wave_sum(v);
            if (lane < 4) sl[lane][at] = lane == 0 ? v : 0.0f;
          }
        }
        __syncthreads();
      }
    }
    // 8 lanes per token, experts j, j + 8, ...
    const int j = tid & 7;
    for (int tl = tid >> 3; tl < TT; tl += 64) {
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
      // (a token's logits are read and overwritten by its own 8 lanes, which run together)
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
    }
    __syncthreads();
    {  // wave w: tokens w TT / 8 .. of expert `lane`
      float v = 0.0f;
      if (lane < 16 * EF)
#pragma unroll
        for (int i = 0; i < TT / 8; ++i) v += sl[0][(wave * (TT / 8) + i) * LD + lane];
      sps[wave][lane] = v;
    }
    __syncthreads();
    if (tid < 64) {
      float v = 0.0f, z = 0.0f;
#pragma unroll
      for (int u = 0; u < 8; ++u) v += sps[u][tid];
      psum += v;
      for (int i = tid; i < TT; i += 64) z += sz[i];
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) z += __shfl_xor(z, o, 64);
      zsum += z;
    }
  }
  __syncthreads();  // counts
  if (gridDim.x == 1 && tid < 64) {  // a single workgroup finishes by itself
    const int c = scnt[tid], N = scnt[64];
    double l = tid < p.E ? psum * c : 0.0;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) l += __shfl_xor(l, o, 64);
    if (tid < p.E) p.counts[tid] = c;
    if (tid == 0) {
      const double n = N;
      p.counts[p.E] = N;
      p.loss[0] = N > 0 ? (float)(p.E * l / (2.0 * n * n)) : 0.0f;
      p.loss[1] = N > 0 ? (float)(zsum / n) : 0.0f;
    }
    return;
  }
  float *const q = p.part + blockIdx.x;
  if (tid < p.E) {
    q[tid * kFwdBlocks] = (float)psum;
    q[(p.E + tid) * kFwdBlocks] = __int_as_float(scnt[tid]);
  }
  if (tid == 0) {
    q[2 * p.E * kFwdBlocks] = (float)zsum;
    q[(2 * p.E + 1) * kFwdBlocks] = __int_as_float(scnt[64]);
  }
}

constexpr int kBwdTokens = 32;
constexpr int kBwdCols = 256;

// A workgroup of 8 waves takes kBwdCols columns (32 per wave) and a split's tokens, 32 at a
// time; a tile's loads are under way while the one before is multiplied. dl of a tile is
// formed in LDS in three bf16 pieces, a row per token: read by rows for dn = dl Wr, with
// transposing reads (tokens along k) for dWr = dl^T n, n's rows likewise. Wr's fragments
// stay in registers for all tiles, dWr's sums too. Row r of a fragment b of columns is
// column 8 (r / 4) + 4 b + r % 4 of the wave's 32, which leaves a lane 8 neighbouring ones.
template <int ND, int WD, int EF>
__global__ __launch_bounds__(512, kPieces<ND> + kPieces<WD> == 2 ? 4 : 2) void balance_bwd_kernel(BalanceP p) {
  constexpr int PN = kPieces<ND>, PW = kPieces<WD>, KE = (EF + 1) / 2;
  // Rows in LDS without bank conflicts, 16-bit values: [token][expert] rows of LE, 8 experts
  // at 8 c at 8 (c ^ (row / 4 % 2)); rows of LN columns, 4 columns at 4 c at 4 (c ^ (row / 2 %
  // 2)). Read across, 16 lanes take 8 bytes each of 4 rows: next to each other of a dl row,
  // 16 bytes apart of the others.
  constexpr int LE = 80, LN = kBwdCols + 32;
  __shared__ __align__(16) uint16_t s_te[3][kBwdTokens * LE];
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
  for (int i = tid; i < kBwdTokens * LE; i += 512) s_te[0][i] = s_te[1][i] = s_te[2][i] = 0;

  // Wr fragments: k experts 32 k + 8 g ..
  const int colf = 8 * (i16 >> 2) + (i16 & 3);
  // (bf16 Wr: rows in LDS, read across like n's, which leaves registers for a second
  // workgroup)
  constexpr bool WL = PW == 1;
  __shared__ __align__(16) uint16_t s_w[WL ? 32 * KE * LN : 8];
  if constexpr (WL) {
    for (int i = tid; i < 32 * KE * (kBwdCols / 8); i += 512) {
      const int e = i / (kBwdCols / 8), c = i % (kBwdCols / 8) * 8;
      u32x4_v v = u32x4_v{0, 0, 0, 0};
      if (p.dn && e < p.E && c0 + c < p.d)
        v = *reinterpret_cast<const u32x4_v *>(static_cast<const bf16_t *>(p.wr) + (int64_t)e * p.d + c0 + c);
      *reinterpret_cast<u32x4_v *>(&s_w[e * LN + c]) = (e >> 1 & 1) ? u32x4_v{v[2], v[3], v[0], v[1]} : v;
    }
  }
  // each 16 lanes: rows (k) 8 g + i16 / 4 (and + 4), four columns of run i16 % 4, from
  // columns lo of the first and hi of the second rows on
  auto across = [&](const uint16_t *rows, int ld, int lo, int hi) -> bf16x8_v {
    typedef __attribute__((address_space(3))) s16x4_v lds_v4;
    const uint16_t *const at = rows + (8 * g + (i16 >> 2)) * ld;
    const s16x4_v v[2] = {
        __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4 *)LDS_AS(char, const_cast<uint16_t *>(at + lo))),
        __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4 *)LDS_AS(char, const_cast<uint16_t *>(at + 4 * ld + hi)))};
    return __builtin_bit_cast(bf16x8_v, v);
  };
  // fragment b of the wave's columns of rows of LN; experts 16 a .. of dl's rows
  auto columns = [&](const uint16_t *rows, int b) {
    const int at = 32 * wave + 8 * (i16 & 3) + 4 * (b ^ (i16 >> 3));
    return across(rows, LN, at, at);
  };
  auto experts = [&](const uint16_t *rows, int a) {
    const int at = 16 * a + 4 * (i16 & 3);
    return across(rows, LE, at, at ^ 8);
  };
  bf16x8_v fw[2][KE][PW];
#pragma unroll
  for (int b = 0; b < 2 && !WL; ++b)
#pragma unroll
    for (int k = 0; k < KE; ++k) {
      float x[8];
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        const int e = 32 * k + 8 * g + c, col = cw + colf + 4 * b;
        x[c] = 0.0f;
        if (p.dn && e < p.E && col < p.d) {
          const int64_t at = (int64_t)e * p.d + col;
          if constexpr (WD == LC_FP32) x[c] = static_cast<const float *>(p.wr)[at];
          else if constexpr (WD == LC_BF16) x[c] = bf2f(static_cast<const bf16_t *>(p.wr)[at]);
          else x[c] = (float)static_cast<const _Float16 *>(p.wr)[at];
        }
      }
      u32x4_v v[PW];
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        uint32_t s[PW];
        split_bf16<PW>(x[2 * c], x[2 * c + 1], s);
#pragma unroll
        for (int i = 0; i < PW; ++i) v[i][c] = s[i];
      }
#pragma unroll
      for (int i = 0; i < PW; ++i) fw[b][k][i] = __builtin_bit_cast(bf16x8_v, v[i]);
    }
  f32x4_v aw[EF][2];  // dWr: experts 16 a + i16, columns 8 g + 4 b ..
#pragma unroll
  for (int a = 0; a < EF; ++a)
#pragma unroll
    for (int b = 0; b < 2; ++b) aw[a][b] = f32x4_v{0.0f, 0.0f, 0.0f, 0.0f};

  // What a thread reads of a tile. dl: token tid / 16, experts 4 (tid % 16) ..; n: rows
  // tid / 32 and + 16, columns 8 (tid % 32) ..; dres as the products leave dn: token 16 a +
  // i16, columns 8 g + 4 b ... All of it, and dn's stores, are buffer accesses without a
  // branch: what is not there lies past the buffer's end. Behind a branch the compiler
  // cannot count the accesses in flight and waits for all of them, stores too, where it
  // needs the first.
  constexpr uint32_t NONE = 0x80000000u;
  const int tl = tid >> 4, e4 = 4 * (tid & 15), nr = tid >> 5, nc = 8 * (tid & 31);
  constexpr int NS = ND == LC_FP32 ? 4 : 2;
  const int rs = p.dres_dt == LC_FP32 ? 4 : 2, os = p.dn_dt == LC_FP32 ? 4 : 2;
  const uint32_t off_n = c0 + nc < p.d ? (uint32_t)(nr * p.d + c0 + nc) * NS : NONE;
  const uint32_t off_c = cw + 8 * g < p.d ? (uint32_t)(i16 * p.d + cw + 8 * g) : NONE;  // (in values)
  auto rows_of = [&](const void *base, int64_t tile, int have, int64_t width, int size) {
    return __builtin_amdgcn_make_buffer_rsrc(
        const_cast<char *>(static_cast<const char *>(base) + tile * kBwdTokens * width * size), 0,
        base ? (int)(have * width * size) : 0, 0x00020000);
  };
  auto have_of = [&](int64_t tile) {
    return tile < tile1 ? (int)min(p.T - tile * kBwdTokens, (int64_t)kBwdTokens) : 0;
  };
  struct Tile {
    uint32_t pr[4], lse;
    uint64_t sel, w, dw;  // pairs
    uint8_t mask, mask_n[2];
    Raw8<ND> n[2];
  };
  typedef __attribute__((ext_vector_type(2))) uint32_t u32x2_v;
  auto fetch = [&](Tile &x, int64_t tile) {
    const int have = have_of(tile);
    const auto m = rows_of(p.mask, tile, have, 1, 1);
    x.mask = __builtin_amdgcn_raw_buffer_load_b8(m, tl, 0, 0);
    const auto q = rows_of(p.dw ? p.sel : nullptr, tile, have, 2, 4), w = rows_of(p.w, tile, have, 2, 4),
               dw = rows_of(p.dw, tile, have, 2, 4);
    x.sel = __builtin_bit_cast(uint64_t, __builtin_amdgcn_raw_buffer_load_b64(q, 8 * tl, 0, 0));
    x.w = __builtin_bit_cast(uint64_t, __builtin_amdgcn_raw_buffer_load_b64(w, 8 * tl, 0, 0));
    x.dw = __builtin_bit_cast(uint64_t, __builtin_amdgcn_raw_buffer_load_b64(dw, 8 * tl, 0, 0));
    x.lse = __builtin_amdgcn_raw_buffer_load_b32(rows_of(p.lse, tile, have, 1, 4), 4 * tl, 0, 0);
    const auto pr = rows_of(p.probs, tile, have, p.E, 4);
#pragma unroll
    for (int c = 0; c < 4; ++c)
      x.pr[c] = __builtin_amdgcn_raw_buffer_load_b32(pr, e4 + c < p.E ? (uint32_t)(tl * p.E + e4 + c) * 4 : NONE, 0, 0);
    const auto n = rows_of(p.dwr ? p.n : nullptr, tile, have, p.d, NS);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      x.mask_n[u] = __builtin_amdgcn_raw_buffer_load_b8(m, nr + 16 * u, 0, 0);
      x.n[u].load(n, off_n + (off_n == NONE ? 0u : (uint32_t)(16 * u * p.d) * NS));
    }
  };
  u32x4_v res[2][2];  // eight values: one word of 16-bit ones, two of fp32
  auto fetch_res = [&](int64_t tile) {
    const auto r = rows_of(p.dn ? p.dres : nullptr, tile, have_of(tile), p.d, rs);
#pragma unroll
    for (int a = 0; a < 2; ++a) {
      const uint32_t at = off_c == NONE ? NONE : (off_c + (uint32_t)(16 * a * p.d)) * rs;
      res[a][0] = __builtin_bit_cast(u32x4_v, __builtin_amdgcn_raw_buffer_load_b128(r, (int)at, 0, 0));
      if (rs == 4) res[a][1] = __builtin_bit_cast(u32x4_v, __builtin_amdgcn_raw_buffer_load_b128(r, (int)(at + 16), 0, 0));
    }
  };
  auto add_res = [&](float (&v)[8], const u32x4_v (&r)[2]) {
    if (p.dres_dt == LC_FP32) {
#pragma unroll
      for (int c = 0; c < 8; ++c) v[c] += __uint_as_float(r[c >> 2][c & 3]);
    } else if (p.dres_dt == LC_BF16) {
#pragma unroll
      for (int c = 0; c < 8; ++c) v[c] += __uint_as_float(c & 1 ? r[0][c >> 1] & 0xFFFF0000u : r[0][c >> 1] << 16);
    } else {
      const f16x8_v h = __builtin_bit_cast(f16x8_v, r[0]);
#pragma unroll
      for (int c = 0; c < 8; ++c) v[c] += (float)h[c];
    }
  };
  auto work = [&](Tile &x, int64_t tile) {
    const int have = have_of(tile);
    __syncthreads();  // the last tile's fragments are read
    {
      const bool live = tl < have && (!p.mask || x.mask != 0);
      float pr[4], dot = 0.0f;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        pr[c] = live ? __uint_as_float(x.pr[c]) : 0.0f;
        dot += pr[c] * s_f[e4 + c];
      }
#pragma unroll
      for (int o = 1; o < 16; o *= 2) dot += __shfl_xor(dot, o, 64);
      const float z = live ? cz * __uint_as_float(x.lse) : 0.0f;
      const int e0 = (int)(uint32_t)x.sel, e1 = (int)(x.sel >> 32);
      const bool pair = live && p.dw, ok0 = pair && e0 >= 0 && e0 < p.E, ok1 = pair && e1 >= 0 && e1 < p.E && e1 != e0;
      const float w0 = ok0 ? __uint_as_float((uint32_t)x.w) : 0.0f, w1 = ok1 ? __uint_as_float((uint32_t)(x.w >> 32)) : 0.0f;
      const float d0 = ok0 ? __uint_as_float((uint32_t)x.dw) : 0.0f, d1 = ok1 ? __uint_as_float((uint32_t)(x.dw >> 32)) : 0.0f;
      const float inner = w0 * d0 + w1 * d1, g0 = w0 * (d0 - inner), g1 = w1 * (d1 - inner);
      if (e4 < 16 * EF) {
        float v[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const int e = e4 + c;
          v[c] = pr[c] * (cb * (s_f[e] - dot) + z);
          v[c] += ok0 && e == e0 ? g0 : ok1 && e == e1 ? g1 : 0.0f;
          if (!live || e >= p.E) v[c] = 0.0f;
        }
        uint32_t s[2][3];
        split_bf16<3>(v[0], v[1], s[0]);
        split_bf16<3>(v[2], v[3], s[1]);
#pragma unroll
        for (int i = 0; i < 3; ++i)
          *reinterpret_cast<uint2 *>(&s_te[i][tl * LE + (e4 ^ 8 * (tl >> 2 & 1))]) = make_uint2(s[0][i], s[1][i]);
      }
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      bf16x8_v f[PN];
      x.n[u].pieces(f);
      const bool live = !p.mask || x.mask_n[u] != 0, swap = nr >> 1 & 1;
#pragma unroll
      for (int i = 0; i < PN; ++i) {
        const u32x4_v v = live ? __builtin_bit_cast(u32x4_v, f[i]) : u32x4_v{0, 0, 0, 0};
        *reinterpret_cast<u32x4_v *>(&s_n[i][(nr + 16 * u) * LN + nc]) = swap ? u32x4_v{v[2], v[3], v[0], v[1]} : v;
      }
    }
    fetch(x, tile + 1);
    __syncthreads();
    {
#pragma unroll
      for (int a = 0; a < 2; ++a) {  // tokens 16 a + i16
        f32x4_v s[2] = {f32x4_v{0.0f, 0.0f, 0.0f, 0.0f}, f32x4_v{0.0f, 0.0f, 0.0f, 0.0f}};
#pragma unroll
        for (int k = 0; k < KE; ++k) {
          bf16x8_v fd[3];
#pragma unroll
          for (int i = 0; i < 3; ++i)
            fd[i] = *reinterpret_cast<const bf16x8_v *>(&s_te[i][(16 * a + i16) * LE + 32 * k + 8 * (g ^ (i16 >> 2 & 1))]);
#pragma unroll
          for (int b = 0; b < 2; ++b) {
            if constexpr (WL) fw[b][k][0] = columns(s_w + 32 * k * LN, b);
            s[b] = mul_pieces(fw[b][k], fd, s[b]);
          }
        }
        const auto out = rows_of(p.dn, tile, have, p.d, os);
        float v[8] = {s[0][0], s[0][1], s[0][2], s[0][3], s[1][0], s[1][1], s[1][2], s[1][3]};
        add_res(v, res[a]);
        const uint32_t at = off_c == NONE ? NONE : (off_c + (uint32_t)(16 * a * p.d)) * os;
        if (p.dn_dt == LC_FP32) {
          const f32x4_v lo = f32x4_v{v[0], v[1], v[2], v[3]}, hi = f32x4_v{v[4], v[5], v[6], v[7]};
          __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4_v, lo), out, (int)at, 0, 0);
          __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4_v, hi), out, (int)(at + 16), 0, 0);
        } else if (p.dn_dt == LC_BF16) {
          const bf16x8_v o = {(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3],
                              (__bf16)v[4], (__bf16)v[5], (__bf16)v[6], (__bf16)v[7]};
          __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4_v, o), out, (int)at, 0, 0);
        } else {
          const f16x8_v o = {(_Float16)v[0], (_Float16)v[1], (_Float16)v[2], (_Float16)v[3],
                             (_Float16)v[4], (_Float16)v[5], (_Float16)v[6], (_Float16)v[7]};
          __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4_v, o), out, (int)at, 0, 0);
        }
      }
      fetch_res(tile + 1);
    }
    {
      bf16x8_v fn[2][PN];
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < PN; ++i) fn[b][i] = columns(s_n[i], b);
#pragma unroll
      for (int a = 0; a < EF; ++a) {
        bf16x8_v fd[3];
#pragma unroll
        for (int i = 0; i < 3; ++i) fd[i] = experts(s_te[i], a);
#pragma unroll
        for (int b = 0; b < 2; ++b) aw[a][b] = mul_pieces(fn[b], fd, aw[a][b]);
      }
    }
  };
  Tile x;
  fetch(x, tile0);
  fetch_res(tile0);
  for (int64_t tile = tile0; tile < tile1; ++tile) work(x, tile);
  if (p.dwr) {
    float *const out = p.splits > 1 ? p.part + (int64_t)split * p.E * p.d : p.dwr;
    const bool add = p.splits == 1 && !p.store;
#pragma unroll
    for (int a = 0; a < EF; ++a)
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const int e = 16 * a + i16, col = cw + 8 * g + 4 * b;
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

// Parts of the tokens in the backward: as many workgroups as run at once, two per compute unit
int bwd_splits(int64_t T, int64_t d) {
  const int64_t chunks = (d + kBwdCols - 1) / kBwdCols, tiles = (T + kBwdTokens - 1) / kBwdTokens;
  const int64_t want = chunks < 512 ? 512 / chunks : 1;
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
  if (a.d % 8 || a.d > (1 << 20)) return fail(LC_ERR_UNSUPPORTED, "moe balance: d %% 8 != 0 or d > 2^20");
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
  // Tokens per tile / 16: the least rounds of tiles over the compute units by a tile's
  // expected time, which grows with its tokens and by 32 tokens' worth for its reads of Wr: every
  // number of tokens up to 28672 then takes one round. Both sides, us (4096 x 64 experts, 2048 x
  // 8), by this rule and by the fastest of 1, 2, 4 and 5: 10000 tokens (3) 36.7, 41.3 and 16.1, 17.1;
  // 16411 (5) 51.8, 77.0 by 4 and 21.2, 25.2 by 1; 24000 (6) 71.6, 92.5 and 25.3, 28.4; 28000 (7) 85.1,
  // 94.2 and 27.9, 31.6. (Above 16 experts 7 spills 10 to 49 registers, above 48 6 spills 31, nearly
  // all of them outside the loop over d.) 8 is left out: 30000 tokens 109.2, by 4 95.5, and 30.5, by 4 32.3. Tiles of more than 32
  // tokens are for bf16 (the others' registers end there).
  const bool wide = a.n_dtype == LC_BF16 && a.w_dtype == LC_BF16;
  int mt = 1;
  int64_t least = 0;
  for (int m = 1; m <= 7; ++m) {
    if (m > 2 && !wide) break;
    const int64_t tiles = (a.T + 16 * m - 1) / (16 * m), time = (tiles + 255) / 256 * (m + 2);
    if (m == 1 || time < least) {
      least = time;
      mt = m;
    }
  }
  p.tiles = (a.T + 16 * mt - 1) / (16 * mt);
  const int nblk = (int)(p.tiles < kFwdBlocks ? p.tiles : kFwdBlocks);
  if (nblk > 0) {
    with_dtype(a.n_dtype, [&](auto nd) {
      with_dtype(a.w_dtype, [&](auto wd) {
        with_experts(a.E, [&](auto ef) {
          constexpr int ND = decltype(nd)::value, WD = decltype(wd)::value, EF = decltype(ef)::value;
          const dim3 grid((unsigned)nblk), threads(512);
          if constexpr (ND == LC_BF16 && WD == LC_BF16) {
            if (mt == 3) hipLaunchKernelGGL((balance_fwd_kernel<ND, WD, EF, 3>), grid, threads, 0, s, p);
            if (mt == 4) hipLaunchKernelGGL((balance_fwd_kernel<ND, WD, EF, 4>), grid, threads, 0, s, p);
            if (mt == 5) hipLaunchKernelGGL((balance_fwd_kernel<ND, WD, EF, 5>), grid, threads, 0, s, p);
            if (mt == 6) hipLaunchKernelGGL((balance_fwd_kernel<ND, WD, EF, 6>), grid, threads, 0, s, p);
            if (mt == 7) hipLaunchKernelGGL((balance_fwd_kernel<ND, WD, EF, 7>), grid, threads, 0, s, p);
          }
          if (mt == 2) hipLaunchKernelGGL((balance_fwd_kernel<ND, WD, EF, 2>), grid, threads, 0, s, p);
          if (mt == 1) hipLaunchKernelGGL((balance_fwd_kernel<ND, WD, EF, 1>), grid, threads, 0, s, p);
        });
      });
    });
    LC_TRY(check_launch("balance_fwd_kernel"));
  }
  if (nblk == 1) return LC_OK;
  hipLaunchKernelGGL(balance_finish_kernel, dim3(1), dim3(1024), 0, s, p, nblk);
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
                           dim3(grid), dim3(512), 0, s, p);
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
