// Sliding-window causal attention with sinks over packed sequences, fp32: one wave per
// query (key) row and head, the head's features over its lanes.
#include "attn_window.hpp"

#include <math.h>

namespace lc {
namespace {

constexpr int NTH = 256;

struct WinP {
  const void *q, *k, *v, *dout;
  void *o, *dq, *dk, *dv;
  float *lse, *D;
  const int32_t *off;
  int64_t ld_q, ld_k, ld_v, ld_o, ld_do, ld_dq, ld_dk, ld_dv;
  int T, B, H, Hkv, G, hd, window, n_sink, dt, o_dt;
  float scale;
};

__device__ __forceinline__ float ld1(const void *base, int64_t i, int dt) {
  if (dt == LC_FP32) return static_cast<const float *>(base)[i];
  if (dt == LC_BF16) return (float)static_cast<const __bf16 *>(base)[i];
  return (float)static_cast<const _Float16 *>(base)[i];
}
__device__ __forceinline__ void st1(void *base, int64_t i, int dt, float v) {
  if (dt == LC_FP32) static_cast<float *>(base)[i] = v;
  else static_cast<__bf16 *>(base)[i] = (__bf16)v;
}

__device__ __forceinline__ int offset_at(const WinP &p, int b) {
  return p.off ? min(max(p.off[b], 0), p.T) : b * (p.T / p.B);
}
// the rows [start, end) of the sequence that holds row i (start = end: none)
__device__ __forceinline__ void sequence_of(const WinP &p, int i, int &start, int &end) {
  int lo = 0, hi = p.B;  // offset_at(lo) <= i < offset_at(hi) once narrowed
  start = end = 0;
  if (i < offset_at(p, 0) || i >= offset_at(p, p.B)) return;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (offset_at(p, mid) <= i) lo = mid;
    else hi = mid;
  }
  start = offset_at(p, lo);
  end = offset_at(p, hi);
}

struct Row2 { float a, b; };
__device__ __forceinline__ Row2 row2(const void *base, int64_t at, int dt, int hd, int lane) {
  Row2 r = {0.0f, 0.0f};
  if (lane < hd) r.a = ld1(base, at + lane, dt);
  if (lane + 64 < hd) r.b = ld1(base, at + lane + 64, dt);
  return r;
}
__device__ __forceinline__ void put2(void *base, int64_t at, int dt, int hd, int lane, Row2 r) {
  if (lane < hd) st1(base, at + lane, dt, r.a);
  if (lane + 64 < hd) st1(base, at + lane + 64, dt, r.b);
}
__device__ __forceinline__ float dot2(Row2 x, Row2 y) { return wave_sum(x.a * y.a + x.b * y.b); }

// calls f(j) for every key that row i sees
template <typename F>
__device__ __forceinline__ void keys_of(const WinP &p, int i, int start, F f) {
  const int w0 = max(start, i - p.window + 1 > i ? start : i - p.window + 1);
  for (int j = start; j < w0 && j - start < p.n_sink; ++j) f(j);
  for (int j = w0; j <= i; ++j) f(j);
}

template <bool DQ>
__global__ __launch_bounds__(NTH) void window_rows_kernel(WinP p) {
  const int lane = threadIdx.x & 63, h = blockIdx.y, kvh = h / p.G;
  const int i = (int)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (i >= p.T) return;
  int start, end;
  sequence_of(p, i, start, end);
  if (start == end) return;
  const int64_t hq = (int64_t)h * p.hd, hk = (int64_t)kvh * p.hd;
  const Row2 q = row2(p.q, i * p.ld_q + hq, p.dt, p.hd, lane);
  const int64_t si = (int64_t)h * p.T + i;
  Row2 acc = {0.0f, 0.0f};
  if constexpr (!DQ) {
    float m = -INFINITY, l = 0.0f;
    keys_of(p, i, start, [&](int j) {
      const float s = dot2(q, row2(p.k, j * p.ld_k + hk, p.dt, p.hd, lane)) * p.scale;
      const Row2 v = row2(p.v, j * p.ld_v + hk, p.dt, p.hd, lane);
      const float mn = fmaxf(m, s), mu = mn == -INFINITY ? 0.0f : mn;
      const float alpha = expf(m - mu), w = expf(s - mu);
      acc.a = acc.a * alpha + w * v.a;
      acc.b = acc.b * alpha + w * v.b;
      l = l * alpha + w;
      m = mn;
    });
    acc.a /= l;
    acc.b /= l;
    put2(p.o, i * p.ld_o + hq, p.o_dt, p.hd, lane, acc);
    if (lane == 0) p.lse[si] = m + logf(l);
  } else {
    const Row2 d = row2(p.dout, i * p.ld_do + hq, p.o_dt, p.hd, lane);
    const float D = dot2(d, row2(p.o, i * p.ld_o + hq, p.o_dt, p.hd, lane)), L = p.lse[si];
    if (lane == 0) p.D[si] = D;
    keys_of(p, i, start, [&](int j) {
      const Row2 k = row2(p.k, j * p.ld_k + hk, p.dt, p.hd, lane);
      const float s = dot2(q, k) * p.scale, dp = dot2(d, row2(p.v, j * p.ld_v + hk, p.dt, p.hd, lane));
      const float ds = expf(s - L) * (dp - D) * p.scale;
      acc.a += ds * k.a;
      acc.b += ds * k.b;
    });
    put2(p.dq, i * p.ld_dq + hq, p.o_dt, p.hd, lane, acc);
  }
}

__global__ __launch_bounds__(NTH) void window_keys_kernel(WinP p) {
  const int lane = threadIdx.x & 63, kvh = blockIdx.y;
  const int j = (int)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (j >= p.T) return;
  int start, end;
  sequence_of(p, j, start, end);
  if (start == end) return;
  const int64_t hk = (int64_t)kvh * p.hd;
  const Row2 k = row2(p.k, j * p.ld_k + hk, p.dt, p.hd, lane), v = row2(p.v, j * p.ld_v + hk, p.dt, p.hd, lane);
  Row2 dk = {0.0f, 0.0f}, dv = {0.0f, 0.0f};
  const int last = j - start < p.n_sink || p.window >= end - j ? end : j + p.window;
  for (int g = 0; g < p.G; ++g) {
    const int h = kvh * p.G + g;
    const int64_t hq = (int64_t)h * p.hd;
    for (int i = j; i < last; ++i) {
      const Row2 q = row2(p.q, i * p.ld_q + hq, p.dt, p.hd, lane), d = row2(p.dout, i * p.ld_do + hq, p.o_dt, p.hd, lane);
      const int64_t si = (int64_t)h * p.T + i;
      const float P = expf(dot2(q, k) * p.scale - p.lse[si]);
      const float ds = P * (dot2(d, v) - p.D[si]) * p.scale;
      dk.a += ds * q.a;
      dk.b += ds * q.b;
      dv.a += P * d.a;
      dv.b += P * d.b;
    }
  }
  put2(p.dk, j * p.ld_dk + hk, p.o_dt, p.hd, lane, dk);
  put2(p.dv, j * p.ld_dv + hk, p.o_dt, p.hd, lane, dv);
}

WinP params(const lc_window_attn_args &a) {
  WinP p{};
  p.q = a.q; p.k = a.k; p.v = a.v; p.dout = a.dout;
  p.o = a.o; p.dq = a.dq; p.dk = a.dk; p.dv = a.dv;
  p.lse = a.lse;
  p.D = static_cast<float *>(a.scratch);
  p.off = a.seq_offsets;
  p.ld_q = a.ld_q; p.ld_k = a.ld_k; p.ld_v = a.ld_v; p.ld_o = a.ld_o;
  p.ld_do = a.ld_dout; p.ld_dq = a.ld_dq; p.ld_dk = a.ld_dk; p.ld_dv = a.ld_dv;
  p.T = (int)a.T;
  p.B = a.B;
  p.H = a.H;
  p.Hkv = a.Hkv ? a.Hkv : a.H;
  p.G = p.H / p.Hkv;
  p.hd = a.hd;
  p.window = a.window;
  p.n_sink = a.n_sink;
  p.dt = a.dtype;
  p.o_dt = a.o_dtype;
  p.scale = 1.0f / sqrtf((float)a.hd);
  return p;
}

}  // namespace

lc_status window_f32_fwd_launch(const lc_window_attn_args &a, hipStream_t s) {
  const WinP p = params(a);
  hipLaunchKernelGGL(window_rows_kernel<false>, dim3((p.T + 3) / 4, p.H), dim3(NTH), 0, s, p);
  return check_launch("window_rows_kernel");
}

lc_status window_f32_bwd_launch(const lc_window_attn_args &a, hipStream_t s) {
  const WinP p = params(a);
  hipLaunchKernelGGL(window_rows_kernel<true>, dim3((p.T + 3) / 4, p.H), dim3(NTH), 0, s, p);
  LC_TRY(check_launch("window_rows_kernel"));
  hipLaunchKernelGGL(window_keys_kernel, dim3((p.T + 3) / 4, p.Hkv), dim3(NTH), 0, s, p);
  return check_launch("window_keys_kernel");
}

}  // namespace lc
