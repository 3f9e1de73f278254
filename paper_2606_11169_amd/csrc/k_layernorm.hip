// LayerNorm forward and backward (HBM-bound row kernels).
//
//   forward:  mu = mean_k x, r = 1/sqrt(mean_k (x - mu)^2 + eps), y = (x - mu) r g + b
//   backward: xh = (x - mu) r, t = dy g,
//             dx = dres + r (t - mean_k t - xh mean_k(t xh)),
//             dg += sum_t dy xh, db += sum_t dy
//
// Every tensor is read once and written once: a row stays in registers between its
// sums and its write (8 to 65536 values forward, 16384 backward), the variance is a second sum
// over the registers, of differences to the mean (sums of squares would lose it in rows far from
// 0). Shorter and longer rows are read three times forward; backward once by the weight
// gradients' launch and twice by the rows', so x and dy come from HBM at least twice there.
//
// Rows are read in runs of 8 values at any alignment (the instruction takes any address); the
// last run of a row whose length is no multiple of 8 begins 8 values before the row's end, and the
// values that it shares with the run before count once in the sums and are written twice, alike
// (but once by the backward of two runs per lane, which reads dres late, where dx may lie over it).
// Whether a tensor has 2 or 4 bytes per value is a template argument (straight-line loads); which
// 16-bit type is a run-time choice of the conversion.
//
// The weight gradients are sums over rows. A backward workgroup keeps its rows' share of
// its columns in registers over all of its rows (one or two workgroups per compute unit, so the
// shares stay a small part of the traffic), adds its row slots through LDS in order, and a second
// kernel adds the workgroups' shares of each column in order: the same bits every run.
//
// Measured (shortest launches of a trace): 16411 rows of 8192, bf16, forward 107 us (98 back to
// back), backward with a residual 201 + 5, 5.0 and 5.3 TB/s (a large copy reaches 5.1 to 5.5 here);
// 4096 of 4096, fp32 in, 17.3 and 44 + 4; 3001 of 1155 bf16 6.3 and 13 + 2.7, 9 of 768 2.7, bound by
// the latency of loads, sums and launches.
#include "common.hpp"

#include <algorithm>

namespace lc {
namespace {

constexpr int NTH = 256;        // forward, one to four waves per row
constexpr int LONG_ROWS = 64;   // rows of a block of the long rows' weight gradients

struct LnP {
  const void *x, *g, *b, *dy, *dres;
  void *y, *dx, *dx_copy;
  float *mean, *rstd;
  float *part;     // shares of dg, then db: [2, nblk, d]
  float *dg, *db;
  int64_t T, ld_x, ld_y, ld_dy, ld_dres, ld_dx;
  int64_t first;   // forward, long rows: the launch's first workgroup
  int d, lpr;      // lpr: lanes per row where several rows share a wave
  float eps;
  int x_dt, w_dt, out_dt, dy_dt, dres_dt, store, nblk;
};

__device__ __forceinline__ float ld1(const void *base, int64_t i, int dt) {
  if (dt == LC_FP32) return static_cast<const float *>(base)[i];
  if (dt == LC_BF16) return (float)static_cast<const __bf16 *>(base)[i];
  return (float)static_cast<const _Float16 *>(base)[i];
}
__device__ __forceinline__ void st1(void *base, int64_t i, int dt, float v) {
  if (dt == LC_FP32) static_cast<float *>(base)[i] = v;
  else if (dt == LC_BF16) static_cast<__bf16 *>(base)[i] = (__bf16)v;
  else static_cast<_Float16 *>(base)[i] = (_Float16)v;
}

// dy g, rounded (not fused into a following subtraction): the row's sums are of the same
// rounded values that they are subtracted from, so what cancels exactly does
__device__ __forceinline__ float scaled(float dy, float g) {
#pragma clang fp contract(off)
  return dy * g;
}

// sum over the lpr lanes of a row (a power of two up to 64, aligned), in every lane: pairs,
// quads, halves of 16 and 16 lanes by data-parallel moves, then rows and halves of the wave
// swapped. (Shuffles, twelve in a row of two sums, go through LDS: 9 x 768 forward 3.4 us, 2.7
// this way, 500 x 4096 4.7 and 4.4.)
template <int CTRL>
__device__ __forceinline__ float moved(float v) {
  return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), CTRL, 0xF, 0xF, true));
}
__device__ __forceinline__ float row_sum(float v, int lpr) {
  if (lpr > 1) v += moved<0xB1>(v);   // quad_perm 1 0 3 2
  if (lpr > 2) v += moved<0x4E>(v);   // quad_perm 2 3 0 1
  if (lpr > 4) v += moved<0x141>(v);  // row_half_mirror
  if (lpr > 8) v += moved<0x140>(v);  // row_mirror
  if (lpr > 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  if (lpr > 32) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  return v;
}

// ---------------------------------------------------------------- runs of 8 values
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4_v;
typedef u32x4_v u32x4_any __attribute__((aligned(2)));
// 8 values of SZ bytes as they lie in memory (SZ = 0: of a size known at run time)
template <int SZ> struct Raw { u32x4_v v[SZ == 2 ? 1 : 2]; };

template <int SZ>
__device__ __forceinline__ void load_raw(const void *base, int64_t i, int dt, Raw<SZ> &r) {
  const bool wide = SZ ? SZ == 4 : dt == LC_FP32;
  const u32x4_any *at = reinterpret_cast<const u32x4_any *>(static_cast<const char *>(base) + i * (wide ? 4 : 2));
  r.v[0] = at[0];
  if constexpr (SZ != 2) {
    if (wide) r.v[1] = at[1];
  }
}
__device__ __forceinline__ void half_values(u32x4_v v, int dt, float (&x)[8]) {
  if (dt == LC_BF16) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(v[i] << 16);
      x[2 * i + 1] = __uint_as_float(v[i] & 0xFFFF0000u);
    }
  } else {
    const f16x8_v h = __builtin_bit_cast(f16x8_v, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (float)h[i];
  }
}
template <int SZ>
__device__ __forceinline__ void values(const Raw<SZ> &r, int dt, float (&x)[8]) {
  if constexpr (SZ != 2) {
    if (SZ == 4 || dt == LC_FP32) {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(r.v[i >> 2][i & 3]);
      return;
    }
  }
  half_values(r.v[0], dt, x);
}
template <int SZ>
__device__ __forceinline__ void load8(const void *base, int64_t i, int dt, float (&x)[8]) {
  Raw<SZ> r;
  load_raw<SZ>(base, i, dt, r);
  values<SZ>(r, dt, x);
}
template <int SZ>
__device__ __forceinline__ void store8(void *base, int64_t i, int dt, const float (&x)[8]) {
  const bool wide = SZ ? SZ == 4 : dt == LC_FP32;
  u32x4_any *at = reinterpret_cast<u32x4_any *>(static_cast<char *>(base) + i * (wide ? 4 : 2));
  if (wide) {
    u32x4_v a, b;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      a[e] = __float_as_uint(x[e]);
      b[e] = __float_as_uint(x[e + 4]);
    }
    at[0] = a;
    at[1] = b;
    return;
  }
  if (dt == LC_BF16) {
    bf16x8_v h;
#pragma unroll
    for (int e = 0; e < 8; ++e) h[e] = (__bf16)x[e];
    at[0] = __builtin_bit_cast(u32x4_v, h);
  } else {
    f16x8_v h;
#pragma unroll
    for (int e = 0; e < 8; ++e) h[e] = (_Float16)x[e];
    at[0] = __builtin_bit_cast(u32x4_v, h);
  }
}

// run n of a row of d >= 8 values: its first value (d or more: no run), and how many of its
// values the run before holds already
__device__ __forceinline__ int run_at(int n, int d, int &skip) {
  const int c = 8 * n, at = min(c, d - 8);
  skip = c - at;
  return c < d ? at : d;
}

// ---------------------------------------------------------------- forward
// WPR waves per row, each lane U runs; U = 1: 64 / lpr rows per wave (lpr < 64 up to 256 values).
// Two runs per lane and as many waves as that takes: few rows of 4096 to 8192 values are held
// by more of the chip than with eight runs (60 rows of 8192 7.3 -> 3.8 us, 500 of 4096 7.7 ->
// 4.7), many lose nothing (16411 x 8192 102 -> 98 us, 4096 x 4096 fp32 in, bf16 out 23.8 -> 22.5).
// Rows of 1025 to 2048 have no barrier with four runs, which many of them gain by (8000 x 2048
// 15.9 -> 15.1 us; 3001 x 1155 6.1 with two waves, 6.3 with one).
template <int WPR, int U, int XS, int WS, int YS>
__global__ __launch_bounds__(WPR > 4 ? 64 * WPR : NTH) void layernorm_fwd_kernel(LnP p) {
  constexpr int NW = WPR > 4 ? WPR : NTH / 64;
  __shared__ float red[2][NW];
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  const int lpr = U == 1 ? p.lpr : 64;
  const int64_t blk = p.first + blockIdx.x;
  const int64_t row = U == 1 ? (blk * NW + wv) * (64 / lpr) + lane / lpr : blk * (NW / WPR) + wv / WPR;
  const bool ok = row < p.T;
  const int l = U == 1 ? lane % lpr : (wv % WPR) * 64 + lane;
  const void *x = static_cast<const char *>(p.x) + row * p.ld_x * XS;
  float v[U][8];
  int at[U], skip[U];
  float s = 0.0f;
  Raw<XS> raw[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    at[u] = run_at(l + 64 * WPR * u, p.d, skip[u]);
    if (!ok) at[u] = p.d;
    if (at[u] < p.d) load_raw<XS>(x, at[u], p.x_dt, raw[u]);
  }
#pragma unroll
  for (int u = 0; u < U; ++u)
    if (at[u] < p.d) {
      values<XS>(raw[u], p.x_dt, v[u]);
#pragma unroll
      for (int e = 0; e < 8; ++e) s += e >= skip[u] ? v[u][e] : 0.0f;
    }
  auto total = [&](float t, int which) {
    if constexpr (U == 1) return row_sum(t, lpr);
    t = row_sum(t, 64);
    if constexpr (WPR > 1) {
      if (lane == 0) red[which][wv] = t;
      __syncthreads();
      t = red[which][wv / WPR * WPR];
#pragma unroll
      for (int w = 1; w < WPR; ++w) t += red[which][wv / WPR * WPR + w];
    }
    return t;
  };
  const float mu = total(s, 0) / (float)p.d;
  float q = 0.0f;
#pragma unroll
  for (int u = 0; u < U; ++u)
    if (at[u] < p.d) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        v[u][e] -= mu;
        q += e >= skip[u] ? v[u][e] * v[u][e] : 0.0f;
      }
    }
  const float r = 1.0f / sqrtf(total(q, 1) / (float)p.d + p.eps);
  if (!ok) return;
  if (l == 0) {
    p.mean[row] = mu;
    p.rstd[row] = r;
  }
  void *y = static_cast<char *>(p.y) + row * p.ld_y * YS;
#pragma unroll
  for (int u = 0; u < U; ++u)
    if (at[u] < p.d) {
      float g[8], b[8];
      load8<WS>(p.g, at[u], p.w_dt, g);
      if (p.b) {
        load8<WS>(p.b, at[u], p.w_dt, b);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) b[e] = 0.0f;
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) v[u][e] = v[u][e] * r * g[e] + b[e];
      store8<YS>(y, at[u], p.out_dt, v[u]);
    }
}

__device__ __forceinline__ float block_sum(float v, float *red) {
  v = row_sum(v, 64);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  return (red[0] + red[1]) + (red[2] + red[3]);
}

// A thread's sum of up to 65536 values of a row, four by four, with what each addition of four rounds
// off carried along (added up plainly, 2^24 equal values are off by the same direction's rounding
// 65536 times: their mean by 6.5e-4 of them, now 1e-7; with four loads at a time 512 x 100000 fp32
// forward 536 -> 351 us, backward 717 -> 565)
struct Sum {
  float s = 0.0f, lost = 0.0f;
  __device__ __forceinline__ void add(const float (&x)[4]) {
#pragma clang fp contract(off)
    const float y = ((x[0] + x[1]) + (x[2] + x[3])) - lost, t = s + y, e = (t - s) - y;
    lost = fabsf(e) < INFINITY ? e : 0.0f;  // (an infinite sum has lost nothing)
    s = t;
  }
};

// the values at k, k + NTH, k + 2 NTH, k + 3 NTH of d from `row` on (past the end: some value of them)
__device__ __forceinline__ void ld4(const void *base, int64_t row, int k, int d, int dt, float (&v)[4]) {
  int64_t at[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) at[i] = row + min(k + i * NTH, d - 1);
  if (dt == LC_FP32) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = static_cast<const float *>(base)[at[i]];
  } else if (dt == LC_BF16) {
    bf16_t h[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = static_cast<const bf16_t *>(base)[at[i]];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = bf2f(h[i]);
  } else {
    _Float16 h[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = static_cast<const _Float16 *>(base)[at[i]];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = (float)h[i];
  }
}

// rows shorter than a run or longer than registers hold: a workgroup per row, value by value
__global__ __launch_bounds__(NTH) void layernorm_fwd_any_kernel(LnP p) {
  __shared__ float red[4];
  const int64_t t = p.first + blockIdx.x;
  Sum s, v;
  for (int k = threadIdx.x; k < p.d; k += 4 * NTH) {
    float x[4];
    ld4(p.x, t * p.ld_x, k, p.d, p.x_dt, x);
#pragma unroll
    for (int i = 1; i < 4; ++i)
      if (k + i * NTH >= p.d) x[i] = 0.0f;
    s.add(x);
  }
  const float mu = block_sum(s.s, red) / (float)p.d;
  for (int k = threadIdx.x; k < p.d; k += 4 * NTH) {
    float x[4];
    ld4(p.x, t * p.ld_x, k, p.d, p.x_dt, x);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = k + i * NTH < p.d ? (x[i] - mu) * (x[i] - mu) : 0.0f;
    v.add(x);
  }
  const float r = 1.0f / sqrtf(block_sum(v.s, red) / (float)p.d + p.eps);
  if (threadIdx.x == 0) {
    p.mean[t] = mu;
    p.rstd[t] = r;
  }
  for (int k = threadIdx.x; k < p.d; k += NTH) {
    const float xh = (ld1(p.x, t * p.ld_x + k, p.x_dt) - mu) * r;
    st1(p.y, t * p.ld_y + k, p.out_dt, xh * ld1(p.g, k, p.w_dt) + (p.b ? ld1(p.b, k, p.w_dt) : 0.0f));
  }
}

// ---------------------------------------------------------------- backward
// Rows of 8 to 16384 values. A row is held by lpr lanes (a power of two; up to 64 of a wave, or
// whole waves), lane l of it the runs l and (U = 2, rows over 8192) l + lpr; the workgroup takes
// NTB / lpr rows at a time. U = 1: the loads run AHEAD = 2 such steps before the sums (one step
// ahead 16411 x 8192 bf16 take 217 us, two 201; sizes that leave fewer rows per workgroup lie
// within 3%); two runs per lane leave no registers for that, nor for the gain. A row's
// sums over several waves go through LDS, buffered twice, one barrier per step.
template <int DYS, int XS, int OS, int U, int NTB>
__global__ __launch_bounds__(NTB) void layernorm_bwd_kernel(LnP p) {
  constexpr int RS = OS;
  constexpr int AHEAD = U == 1 ? 2 : 1;
  constexpr bool HOLD = U == 1;  // the gain in registers
  __shared__ __align__(16) float red[U * NTB * 8];
  __shared__ float dots[2][2][NTB / 64];
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  const int lpr = p.lpr, slots = NTB / lpr, slot = threadIdx.x / lpr, l = threadIdx.x % lpr;
  int at[U], skip[U];
  float g[U][8], ag[U][8], ab[U][8];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    at[u] = run_at(l + lpr * u, p.d, skip[u]);
    if (HOLD && at[u] < p.d) load8<0>(p.g, at[u], p.w_dt, g[u]);
#pragma unroll
    for (int e = 0; e < 8; ++e) ag[u][e] = ab[u][e] = 0.0f;
  }
  struct In {
    Raw<DYS> y[U];
    Raw<XS> x[U];
    Raw<RS> r[U];
    float mu, rstd;
  } in[AHEAD];
  auto load = [&](In &i, int64_t row) {
    if (row >= p.T) return;
    i.mu = p.mean[row];
    i.rstd = p.rstd[row];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (at[u] < p.d) {
        load_raw<DYS>(p.dy, row * p.ld_dy + at[u], p.dy_dt, i.y[u]);
        load_raw<XS>(p.x, row * p.ld_x + at[u], p.x_dt, i.x[u]);
        if (HOLD && p.dres) load_raw<RS>(p.dres, row * p.ld_dres + at[u], p.dres_dt, i.r[u]);
      }
  };
  const int64_t step = (int64_t)gridDim.x * slots;
  int64_t r0 = (int64_t)blockIdx.x * slots, row = r0 + slot;
  int odd = 0;
  auto one = [&](In &i) {  // the rows of a step, loaded into i
    const bool ok = row < p.T;
    float xh[U][8], t[U][8], o[U][8];
    float st = 0.0f, sx = 0.0f;
    if (!HOLD) load(i, row);
    const float rc = i.rstd, mu = i.mu;
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (ok && at[u] < p.d) {
        values<DYS>(i.y[u], p.dy_dt, t[u]);
        values<XS>(i.x[u], p.x_dt, xh[u]);
        if (HOLD && p.dres) {
          values<RS>(i.r[u], p.dres_dt, o[u]);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) o[u][e] = 0.0f;
        }
        if (!HOLD) load8<0>(p.g, at[u], p.w_dt, g[u]);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          xh[u][e] = (xh[u][e] - mu) * rc;
          ag[u][e] += t[u][e] * xh[u][e];
          ab[u][e] += t[u][e];
          t[u][e] = scaled(t[u][e], g[u][e]);
          st += e >= skip[u] ? t[u][e] : 0.0f;
          sx += e >= skip[u] ? t[u][e] * xh[u][e] : 0.0f;
        }
      }
    if (HOLD) load(i, row + AHEAD * step);
    if (lpr <= 64) {
      st = row_sum(st, lpr);
      sx = row_sum(sx, lpr);
    } else {
      st = row_sum(st, 64);
      sx = row_sum(sx, 64);
      if (lane == 0) {
        dots[odd][0][wv] = st;
        dots[odd][1][wv] = sx;
      }
      // (dx may lie over dres, whose shared values another wave stores from here on: the run's last value
      // is waited for, loads return in order)
      if (HOLD) asm volatile("" ::"v"(o[0][7]));
      __syncthreads();
      const int w0 = slot * (lpr / 64);
      st = dots[odd][0][w0];
      sx = dots[odd][1][w0];
      for (int w = 1; w < lpr / 64; ++w) {
        st += dots[odd][0][w0 + w];
        sx += dots[odd][1][w0 + w];
      }
    }
    if (ok) {
      st /= (float)p.d;
      sx /= (float)p.d;
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (at[u] < p.d) {
          if (!HOLD && p.dres) load8<RS>(p.dres, row * p.ld_dres + at[u], p.dres_dt, o[u]);
#pragma unroll
          for (int e = 0; e < 8; ++e) o[u][e] += rc * (t[u][e] - st - xh[u][e] * sx);
          if (!HOLD && skip[u] && p.dres) {
            // (dx may lie over dres, and the shared values belong to another wave, which may not have
            // read them, or have stored dx over what was read here: dx and its copy are left to it)
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (e >= skip[u]) {
                st1(p.dx, row * p.ld_dx + at[u] + e, p.out_dt, o[u][e]);
                if (p.dx_copy) st1(p.dx_copy, row * p.ld_dx + at[u] + e, LC_BF16, o[u][e]);
              }
          } else {
            store8<OS>(p.dx, row * p.ld_dx + at[u], p.out_dt, o[u]);
            if (p.dx_copy) store8<2>(p.dx_copy, row * p.ld_dx + at[u], LC_BF16, o[u]);
          }
        }
    }
    r0 += step;
    row += step;
    odd ^= 1;
  };
  if (HOLD) {
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) load(in[i], row + i * step);
  }
#pragma unroll 1
  while (r0 < p.T) {
    one(in[0]);
    if (AHEAD == 1) continue;
    if (r0 >= p.T) break;
    one(in[AHEAD - 1]);
  }
  if (!p.dg && !p.db) return;
  // the row slots in order, column by column
#pragma unroll 1
  for (int which = 0; which < 2; ++which) {
    float *const dst = which ? p.db : p.dg;
    if (!dst) continue;
    __syncthreads();
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (at[u] < p.d) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (e >= skip[u]) red[slot * U * lpr * 8 + at[u] + e] = which ? ab[u][e] : ag[u][e];
      }
    __syncthreads();
    for (int k = threadIdx.x; k < p.d; k += NTB) {
      float s = red[k];
      for (int i = 1; i < slots; ++i) s += red[i * U * lpr * 8 + k];
      if (gridDim.x > 1) p.part[((int64_t)which * p.nblk + blockIdx.x) * p.d + k] = s;
      else dst[k] = p.store ? s : dst[k] + s;
    }
  }
}

// dg, db [k] (+)= the workgroups' shares: sixteen slices of consecutive workgroups, each in
// order with its loads in flight together, then the slices in order
constexpr int SLICES = 16;
__global__ __launch_bounds__(64 * SLICES) void layernorm_final_kernel(LnP p) {
  __shared__ float sl[SLICES][64];
  float *const dst = blockIdx.y ? p.db : p.dg;
  if (!dst) return;
  const int i = threadIdx.x >> 6, kc = threadIdx.x & 63;
  const int k = blockIdx.x * 64 + kc;
  const int per = (p.nblk + SLICES - 1) / SLICES, b0 = i * per, b1 = min(p.nblk, b0 + per);
  const float *part = p.part + (int64_t)blockIdx.y * p.nblk * p.d + k;
  float s = 0.0f;
  if (k < p.d) {
    int b = b0;
    for (; b + 8 <= b1; b += 8) {
      float v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = part[(int64_t)(b + j) * p.d];
#pragma unroll
      for (int j = 0; j < 8; ++j) s += v[j];
    }
    for (; b < b1; ++b) s += part[(int64_t)b * p.d];
  }
  sl[i][kc] = s;
  __syncthreads();
  if (i == 0 && k < p.d) {
#pragma unroll
    for (int j = 1; j < SLICES; ++j) s += sl[j][kc];
    dst[k] = p.store ? s : dst[k] + s;
  }
}

// Rows shorter than a run or longer than registers hold: the shares of blocks of LONG_ROWS
// rows (before dx, which may lie over dy), then a workgroup per row, value by value.
__global__ __launch_bounds__(NTH) void layernorm_part_any_kernel(LnP p) {
  const int k = blockIdx.x * NTH + threadIdx.x;
  if (k >= p.d) return;
  for (int64_t blk = blockIdx.y; blk < p.nblk; blk += gridDim.y) {
    const int64_t t0 = blk * LONG_ROWS, t1 = min(p.T, t0 + LONG_ROWS);
    float g = 0.0f, b = 0.0f;
    for (int64_t t = t0; t < t1; ++t) {
      const float dy = ld1(p.dy, t * p.ld_dy + k, p.dy_dt);
      g += dy * ((ld1(p.x, t * p.ld_x + k, p.x_dt) - p.mean[t]) * p.rstd[t]);
      b += dy;
    }
    p.part[blk * p.d + k] = g;
    p.part[(p.nblk + blk) * p.d + k] = b;
  }
}
__global__ __launch_bounds__(NTH) void layernorm_bwd_any_kernel(LnP p) {
  __shared__ float red[4];
  const int64_t t = p.first + blockIdx.x;
  const float mu = p.mean[t], r = p.rstd[t];
  Sum su, sq;
  for (int k = threadIdx.x; k < p.d; k += 4 * NTH) {
    float u[4], g[4], x[4];
    ld4(p.dy, t * p.ld_dy, k, p.d, p.dy_dt, u);
    ld4(p.g, 0, k, p.d, p.w_dt, g);
    ld4(p.x, t * p.ld_x, k, p.d, p.x_dt, x);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bool on = k + i * NTH < p.d;
      u[i] = on ? scaled(u[i], g[i]) : 0.0f;
      x[i] = on ? u[i] * ((x[i] - mu) * r) : 0.0f;
    }
    su.add(u);
    sq.add(x);
  }
  const float s = block_sum(su.s, red) / (float)p.d, q = block_sum(sq.s, red) / (float)p.d;
  for (int k = threadIdx.x; k < p.d; k += NTH) {
    const float u = scaled(ld1(p.dy, t * p.ld_dy + k, p.dy_dt), ld1(p.g, k, p.w_dt));
    const float xh = (ld1(p.x, t * p.ld_x + k, p.x_dt) - mu) * r;
    float o = r * (u - s - xh * q);
    if (p.dres) o += ld1(p.dres, t * p.ld_dres + k, p.dres_dt);
    st1(p.dx, t * p.ld_dx + k, p.out_dt, o);
    if (p.dx_copy) st1(p.dx_copy, t * p.ld_dx + k, LC_BF16, o);
  }
}

// ---------------------------------------------------------------- host
constexpr int MAXD_FWD = 65536, MAXD_BWD = 16384;  // in registers
constexpr int MAXD = 1 << 24;

int lanes_of(int64_t d, int most) {  // the power of two of lanes that hold a row, 8 values each
  int l = 1;
  while (l < most && 8ll * l < d) l *= 2;
  return l;
}
// Backward: threads per workgroup (512 rather than 1024 where a row of one run per lane fits
// them: 100 x 768 9.3 -> 8.1 us, 4096 x 4096 56 -> 54), and at most one workgroup per compute
// unit: more shares cost the final sum more than their rows gain (4096 rows of 4096, fp32: 256
// workgroups 54 us with it, 512 57, 1024 60; 20000 x 768 34 and 38). Rows of 16 bits have half the
// bytes in flight per workgroup; from 4096 of them on two workgroups of 512 threads per unit gain
// (20000 x 3000 115 -> 85 us, 20000 x 1536 53 -> 44, 8000 x 4096 51 -> 44, 4000 x 1280 18.6 ->
// 18.1; but 3000 x 2048 17.5 -> 19.4, and with 1024 threads 16411 x 8192 168 -> 177).
int bwd_threads(int64_t d) { return d <= 4096 ? 512 : 1024; }
bool bwd_in_registers(int64_t d) { return d >= 8 && d <= MAXD_BWD; }
int64_t blocks_of(int64_t T, int64_t d, bool half) {
  if (!bwd_in_registers(d)) return (T + LONG_ROWS - 1) / LONG_ROWS;
  const int nt = bwd_threads(d), slots = nt / lanes_of(d, nt);
  return std::min<int64_t>(half && nt == 512 && T >= 4096 ? 512 : 256, (T + slots - 1) / slots);
}
size_t scratch_of(int64_t T, int64_t d) {  // for any types
  return T <= 0 || T > INT32_MAX || d <= 0 || d > MAXD ? 0 : (size_t)blocks_of(T, d, true) * (size_t)d * 2 * sizeof(float);
}

lc_status check(const lc_layernorm_args &a, bool bwd) {
  if (a.T < 0 || a.d <= 0) return fail(LC_ERR_INVALID_ARG, "layernorm: T must be 0 or more, d positive");
  if (a.d > MAXD) return fail(LC_ERR_UNSUPPORTED, "layernorm: rows of more than 2^24 values");
  if (a.T > INT32_MAX) return fail(LC_ERR_UNSUPPORTED, "layernorm: 2^31 or more rows");
  if (!valid_dtype(a.x_dtype) || !valid_dtype(a.w_dtype) || !valid_dtype(a.out_dtype))
    return fail(LC_ERR_INVALID_ARG, "layernorm: unknown dtype");
  auto ld_ok = [&](int64_t ld) { return ld == 0 || (ld >= a.d && ld <= INT64_MAX / 4 / (a.T + 1)); };
  if (!ld_ok(a.ld_x) || !(bwd ? ld_ok(a.ld_dy) && ld_ok(a.ld_dx) && (!a.dres || ld_ok(a.ld_dres)) : ld_ok(a.ld_y)))
    return fail(LC_ERR_INVALID_ARG, "layernorm: leading dimension smaller than d (or past 64 bits)");
  if (a.T == 0) return LC_OK;
  if (!a.x || !a.g || !a.mean || !a.rstd) return fail(LC_ERR_INVALID_ARG, "layernorm: null pointer");
  if (!aligned16(a.x) || !aligned16(a.g) || !aligned16(a.mean) || !aligned16(a.rstd))
    return fail(LC_ERR_INVALID_ARG, "layernorm: unaligned pointer");
  if (!bwd) {
    if (!a.y || !aligned16(a.y) || !aligned16(a.b))
      return fail(LC_ERR_INVALID_ARG, "layernorm: bad bias or output pointer");
    return LC_OK;
  }
  if (!valid_dtype(a.dy_dtype) || (a.dres && !valid_dtype(a.dres_dtype)))
    return fail(LC_ERR_INVALID_ARG, "layernorm: unknown dtype");
  if (!a.dy || !a.dx || !aligned16(a.dy) || !aligned16(a.dx) || !aligned16(a.dres) || !aligned16(a.dx_copy) ||
      !aligned16(a.dg_accum) || !aligned16(a.db_accum))
    return fail(LC_ERR_INVALID_ARG, "layernorm: bad backward pointer");
  if ((a.dg_accum || a.db_accum) &&
      (!a.scratch || !aligned16(a.scratch) || a.scratch_bytes < scratch_of(a.T, a.d)))
    return fail(LC_ERR_WORKSPACE, "layernorm: scratch smaller than lc_layernorm_scratch_bytes (or unaligned)");
  return LC_OK;
}

LnP params(const lc_layernorm_args &a) {
  LnP p{};
  auto ld = [&](int64_t v) { return v ? v : a.d; };
  p.x = a.x; p.g = a.g; p.b = a.b; p.dy = a.dy; p.dres = a.dres;
  p.y = a.y; p.dx = a.dx; p.dx_copy = a.dx_copy;
  p.mean = a.mean; p.rstd = a.rstd;
  p.dg = a.dg_accum; p.db = a.db_accum;
  p.T = a.T;
  p.d = (int)a.d;
  p.ld_x = ld(a.ld_x); p.ld_y = ld(a.ld_y); p.ld_dy = ld(a.ld_dy); p.ld_dres = ld(a.ld_dres); p.ld_dx = ld(a.ld_dx);
  p.eps = a.eps;
  p.x_dt = a.x_dtype; p.w_dt = a.w_dtype; p.out_dt = a.out_dtype; p.dy_dt = a.dy_dtype; p.dres_dt = a.dres_dtype;
  p.store = a.store_dg != 0;
  p.part = static_cast<float *>(a.scratch);
  return p;
}

// calls f(sizes...) with each type's size (2 or 4 bytes) as a compile-time constant
template <typename F> void with_size(int dt, F f) {
  if (dt == LC_FP32) f(std::integral_constant<int, 4>{});
  else f(std::integral_constant<int, 2>{});
}

template <int WPR, int U>
void fwd_shape(LnP p, hipStream_t s) {
  constexpr int NW = WPR > 4 ? WPR : NTH / 64;
  constexpr uint32_t PART = 1u << 21;
  const int64_t rows = U == 1 ? NW * (64 / p.lpr) : NW / WPR;
  with_size(p.x_dt, [&](auto xs) {
    with_size(p.w_dt, [&](auto ws) {
      with_size(p.out_dt, [&](auto ys) {
        const uint32_t n = (uint32_t)((p.T + rows - 1) / rows);
        // in parts under a launch's limit of 2^32 work-items (launch_parts is for up to 512 threads)
        for (uint32_t first = 0; first < n; first += PART) {
          p.first = first;
          hipLaunchKernelGGL((layernorm_fwd_kernel<WPR, U, decltype(xs)::value, decltype(ws)::value, decltype(ys)::value>),
                             dim3(std::min(PART, n - first)), dim3(64 * NW), 0, s, p);
        }
      });
    });
  });
}

lc_status forward(const lc_layernorm_args &a, hipStream_t s) {
  LC_TRY(check(a, false));
  if (a.T == 0) return LC_OK;
  LnP p = params(a);
  p.lpr = lanes_of(a.d, 64);
  if (p.d < 8 || p.d > MAXD_FWD) {
    launch_parts((uint32_t)p.T, [&](uint32_t first, uint32_t count) {
      p.first = first;
      hipLaunchKernelGGL(layernorm_fwd_any_kernel, dim3(count), dim3(NTH), 0, s, p);
    });
  } else if (p.d <= 512) {
    fwd_shape<1, 1>(p, s);
  } else if (p.d <= 1024) {
    fwd_shape<1, 2>(p, s);
  } else if (p.d <= 2048) {
    if (p.T >= 4096) fwd_shape<1, 4>(p, s);
    else fwd_shape<2, 2>(p, s);
  } else if (p.d <= 4096) {
    fwd_shape<4, 2>(p, s);
  } else if (p.d <= 8192) {
    fwd_shape<8, 2>(p, s);
  } else if (p.d <= 16384) {
    fwd_shape<16, 2>(p, s);
  } else {
    fwd_shape<16, 8>(p, s);
  }
  return check_launch("layernorm_fwd_kernel");
}

template <int U, int NTB>
void bwd_shape(const LnP &p, hipStream_t s) {
  const dim3 grid((unsigned)p.nblk), block(NTB);
  // (the residual's gradient of another size than dx: every size at run time)
  if (p.dres && (p.dres_dt == LC_FP32) != (p.out_dt == LC_FP32)) {
    hipLaunchKernelGGL((layernorm_bwd_kernel<0, 0, 0, U, NTB>), grid, block, 0, s, p);
    return;
  }
  with_size(p.dy_dt, [&](auto ds) {
    with_size(p.x_dt, [&](auto xs) {
      with_size(p.out_dt, [&](auto os) {
        hipLaunchKernelGGL((layernorm_bwd_kernel<decltype(ds)::value, decltype(xs)::value, decltype(os)::value, U, NTB>),
                           grid, block, 0, s, p);
      });
    });
  });
}

lc_status backward(const lc_layernorm_args &a, hipStream_t s) {
  LC_TRY(check(a, true));
  if (a.T == 0) return LC_OK;
  LnP p = params(a);
  p.nblk = (int)blocks_of(a.T, a.d, a.x_dtype != LC_FP32 && a.dy_dtype != LC_FP32);
  p.lpr = lanes_of(a.d, bwd_threads(a.d));
  const bool sums = p.dg || p.db;
  if (bwd_in_registers(a.d)) {
    if (p.d <= 4096) bwd_shape<1, 512>(p, s);
    else if (p.d <= 8192) bwd_shape<1, 1024>(p, s);
    else bwd_shape<2, 1024>(p, s);
    LC_TRY(check_launch("layernorm_bwd_kernel"));
    if (!sums || p.nblk == 1) return LC_OK;
  } else {
    if (sums) {
      const dim3 grid(ceil_div((size_t)p.d, NTH), std::min(p.nblk, 1024));
      hipLaunchKernelGGL(layernorm_part_any_kernel, grid, dim3(NTH), 0, s, p);
      LC_TRY(check_launch("layernorm_part_any_kernel"));
    }
    launch_parts((uint32_t)p.T, [&](uint32_t first, uint32_t count) {
      p.first = first;
      hipLaunchKernelGGL(layernorm_bwd_any_kernel, dim3(count), dim3(NTH), 0, s, p);
    });
    LC_TRY(check_launch("layernorm_bwd_any_kernel"));
    if (!sums) return LC_OK;
  }
  hipLaunchKernelGGL(layernorm_final_kernel, dim3(ceil_div((size_t)p.d, 64), 2), dim3(64 * SLICES), 0, s, p);
  return check_launch("layernorm_final_kernel");
}

}  // namespace
}  // namespace lc

extern "C" {

lc_status lc_layernorm_forward(const lc_layernorm_args *args, void *stream) {
  if (!args) return lc::fail(LC_ERR_INVALID_ARG, "layernorm: null args");
  return lc::forward(*args, static_cast<hipStream_t>(stream));
}

lc_status lc_layernorm_backward(const lc_layernorm_args *args, void *stream) {
  if (!args) return lc::fail(LC_ERR_INVALID_ARG, "layernorm: null args");
  return lc::backward(*args, static_cast<hipStream_t>(stream));
}

size_t lc_layernorm_scratch_bytes(int64_t T, int64_t d) { return lc::scratch_of(T, d); }

}  // extern "C"
