// Sliding-window causal attention with sinks over packed sequences: one wave per
// query (key) row and head, the head's features over its lanes.
#include "common.hpp"

#include <math.h>

namespace lc {
namespace {

constexpr int NTH = 256;
constexpr int MAXHD = 128;

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

size_t scratch_of(int64_t T, int64_t H) { return T <= 0 || H <= 0 ? 0 : (size_t)T * (size_t)H * sizeof(float); }

lc_status check(const lc_window_attn_args &a, bool bwd) {
  if (a.T < 0 || a.B < 1 || a.H < 1 || a.hd < 1)
    return fail(LC_ERR_INVALID_ARG, "window attention: T must be 0 or more, B, H and hd positive");
  if (a.T >= (int64_t)1 << 30) return fail(LC_ERR_UNSUPPORTED, "window attention: 2^30 or more rows");
  if (a.B > 1 << 20) return fail(LC_ERR_UNSUPPORTED, "window attention: more than 2^20 sequences");
  if (a.Hkv < 0 || (a.Hkv > 0 && a.H % a.Hkv))
    return fail(LC_ERR_INVALID_ARG, "window attention: Hkv (%d) must be 0 or divide H (%d)", a.Hkv, a.H);
  if (a.window < 1 || a.n_sink < 0)
    return fail(LC_ERR_INVALID_ARG, "window attention: window must be 1 or more, n_sink 0 or more");
  if (!a.seq_offsets && a.T % a.B)
    return fail(LC_ERR_INVALID_ARG, "window attention: without seq_offsets T must be a multiple of B");
  if (a.dtype == LC_BF16 || a.dtype == LC_FP16) {
    if (a.o_dtype != LC_BF16) return fail(LC_ERR_UNSUPPORTED, "window attention: o/gradients must be bf16");
    if (a.hd != 64 && a.hd != 128)
      return fail(LC_ERR_UNSUPPORTED, "window attention (matrix cores): head_dim must be 64 or 128");
  } else if (a.dtype == LC_FP32) {
    if (a.o_dtype != LC_FP32) return fail(LC_ERR_UNSUPPORTED, "window attention fp32: o must be fp32");
    if (a.hd > MAXHD || a.hd % 2) return fail(LC_ERR_UNSUPPORTED, "window attention fp32: even head_dim <= 128");
  } else {
    return fail(LC_ERR_INVALID_ARG, "window attention: unknown dtype");
  }
  const int64_t qw = (int64_t)a.H * a.hd, kw = (int64_t)(a.Hkv ? a.Hkv : a.H) * a.hd;
  if (qw > INT32_MAX) return fail(LC_ERR_UNSUPPORTED, "window attention: H * hd of 2^31 or more");
  const int64_t most = (int64_t)1 << 30;  // (a row's bytes stay below 2^32)
  auto ld_bad = [&](int64_t ld, int64_t w) { return ld < w || ld > most || (a.dtype != LC_FP32 && ld % 8); };
  if (ld_bad(a.ld_q, qw) || ld_bad(a.ld_k, kw) || ld_bad(a.ld_v, kw) || ld_bad(a.ld_o, qw) ||
      (bwd && (ld_bad(a.ld_dout, qw) || ld_bad(a.ld_dq, qw) || ld_bad(a.ld_dk, kw) || ld_bad(a.ld_dv, kw))))
    return fail(LC_ERR_INVALID_ARG, "window attention: a leading dimension is smaller than heads * hd, larger "
                "than 2^30 or (16 bits) not a multiple of 8");
  if (a.T == 0) return LC_OK;
  auto bad = [](const void *x) { return !x || !aligned16(x); };
  if (bad(a.q) || bad(a.k) || bad(a.v) || bad(a.o) || bad(a.lse))
    return fail(LC_ERR_INVALID_ARG, "window attention: null or unaligned pointer");
  if (reinterpret_cast<uintptr_t>(a.seq_offsets) & 3)
    return fail(LC_ERR_INVALID_ARG, "window attention: unaligned seq_offsets");
  if (bwd) {
    if (bad(a.dout) || bad(a.dq) || bad(a.dk) || bad(a.dv))
      return fail(LC_ERR_INVALID_ARG, "window attention: null or unaligned gradient pointer");
    if (bad(a.scratch) || a.scratch_bytes < scratch_of(a.T, a.H))
      return fail(LC_ERR_WORKSPACE, "window attention: scratch smaller than "
                  "lc_window_attention_scratch_bytes (or unaligned)");
  }
  return LC_OK;
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

lc_status forward(const lc_window_attn_args &a, hipStream_t s) {
  LC_TRY(check(a, false));
  if (a.T == 0) return LC_OK;
  const WinP p = params(a);
  hipLaunchKernelGGL(window_rows_kernel<false>, dim3((p.T + 3) / 4, p.H), dim3(NTH), 0, s, p);
  return check_launch("window_rows_kernel");
}

lc_status backward(const lc_window_attn_args &a, hipStream_t s) {
  LC_TRY(check(a, true));
  if (a.T == 0) return LC_OK;
  const WinP p = params(a);
  hipLaunchKernelGGL(window_rows_kernel<true>, dim3((p.T + 3) / 4, p.H), dim3(NTH), 0, s, p);
  LC_TRY(check_launch("window_rows_kernel"));
  hipLaunchKernelGGL(window_keys_kernel, dim3((p.T + 3) / 4, p.Hkv), dim3(NTH), 0, s, p);
  return check_launch("window_keys_kernel");
}

}  // namespace
}  // namespace lc

extern "C" {

lc_status lc_window_attention_forward(const lc_window_attn_args *args, void *stream) {
  if (!args) return lc::fail(LC_ERR_INVALID_ARG, "window attention: null args");
  return lc::forward(*args, static_cast<hipStream_t>(stream));
}

lc_status lc_window_attention_backward(const lc_window_attn_args *args, void *stream) {
  if (!args) return lc::fail(LC_ERR_INVALID_ARG, "window attention: null args");
  return lc::backward(*args, static_cast<hipStream_t>(stream));
}

size_t lc_window_attention_scratch_bytes(int32_t dtype, int64_t T, int32_t H, int32_t Hkv, int32_t hd,
                                         int32_t window, int32_t n_sink) {
  (void)dtype; (void)Hkv; (void)hd; (void)window; (void)n_sink;
  return lc::scratch_of(T, H);
}

}  // extern "C"
