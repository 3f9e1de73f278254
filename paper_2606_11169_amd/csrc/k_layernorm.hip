// LayerNorm forward and backward.
//
//   forward:  mu = mean_k x, r = 1/sqrt(mean_k (x - mu)^2 + eps), y = (x - mu) r g + b
//   backward: xh = (x - mu) r, t = dy g,
//             dx = dres + r (t - mean_k t - xh mean_k(t xh)),
//             dg += sum_t dy xh, db += sum_t dy
#include "common.hpp"

namespace lc {
namespace {

constexpr int NTH = 256;
constexpr int ROWS = 16;  // rows per block of the weight gradients' partial sums

struct LnP {
  const void *x, *g, *b, *dy, *dres;
  void *y, *dx, *dx_copy;
  float *mean, *rstd;
  float *pg, *pb;  // partial sums of dg and db, [nblk, d] each
  float *dg, *db;
  int64_t T, d, ld_x, ld_y, ld_dy, ld_dres, ld_dx;
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

__device__ __forceinline__ float block_sum(float v, float *red) {
  v = wave_sum(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  return (red[0] + red[1]) + (red[2] + red[3]);
}

__global__ __launch_bounds__(NTH) void layernorm_fwd_kernel(LnP p) {
  __shared__ float red[4];
  const int64_t t = blockIdx.x;
  float s = 0.0f, v = 0.0f;
  for (int64_t k = threadIdx.x; k < p.d; k += NTH) s += ld1(p.x, t * p.ld_x + k, p.x_dt);
  const float mu = block_sum(s, red) / (float)p.d;
  for (int64_t k = threadIdx.x; k < p.d; k += NTH) {
    const float c = ld1(p.x, t * p.ld_x + k, p.x_dt) - mu;
    v += c * c;
  }
  const float r = 1.0f / sqrtf(block_sum(v, red) / (float)p.d + p.eps);
  if (threadIdx.x == 0) {
    p.mean[t] = mu;
    p.rstd[t] = r;
  }
  for (int64_t k = threadIdx.x; k < p.d; k += NTH) {
    const float xh = (ld1(p.x, t * p.ld_x + k, p.x_dt) - mu) * r;
    st1(p.y, t * p.ld_y + k, p.out_dt, xh * ld1(p.g, k, p.w_dt) + (p.b ? ld1(p.b, k, p.w_dt) : 0.0f));
  }
}

// partial sums of the weight gradients over ROWS rows
__global__ __launch_bounds__(NTH) void layernorm_partial_kernel(LnP p) {
  const int64_t k = (int64_t)blockIdx.x * NTH + threadIdx.x;
  if (k >= p.d) return;
  const int64_t t0 = (int64_t)blockIdx.y * ROWS, t1 = min(p.T, t0 + ROWS);
  float g = 0.0f, b = 0.0f;
  for (int64_t t = t0; t < t1; ++t) {
    const float dy = ld1(p.dy, t * p.ld_dy + k, p.dy_dt);
    g += dy * ((ld1(p.x, t * p.ld_x + k, p.x_dt) - p.mean[t]) * p.rstd[t]);
    b += dy;
  }
  p.pg[blockIdx.y * p.d + k] = g;
  p.pb[blockIdx.y * p.d + k] = b;
}

__global__ __launch_bounds__(NTH) void layernorm_final_kernel(LnP p) {
  const int64_t k = (int64_t)blockIdx.x * NTH + threadIdx.x;
  if (k >= p.d) return;
  float g = 0.0f, b = 0.0f;
  for (int i = 0; i < p.nblk; ++i) {
    g += p.pg[i * p.d + k];
    b += p.pb[i * p.d + k];
  }
  if (p.dg) p.dg[k] = p.store ? g : p.dg[k] + g;
  if (p.db) p.db[k] = p.store ? b : p.db[k] + b;
}

__global__ __launch_bounds__(NTH) void layernorm_bwd_kernel(LnP p) {
  __shared__ float red[4];
  const int64_t t = blockIdx.x;
  const float mu = p.mean[t], r = p.rstd[t];
  float s = 0.0f, q = 0.0f;
  for (int64_t k = threadIdx.x; k < p.d; k += NTH) {
    const float u = scaled(ld1(p.dy, t * p.ld_dy + k, p.dy_dt), ld1(p.g, k, p.w_dt));
    s += u;
    q += u * ((ld1(p.x, t * p.ld_x + k, p.x_dt) - mu) * r);
  }
  s = block_sum(s, red) / (float)p.d;
  q = block_sum(q, red) / (float)p.d;
  for (int64_t k = threadIdx.x; k < p.d; k += NTH) {
    const float u = scaled(ld1(p.dy, t * p.ld_dy + k, p.dy_dt), ld1(p.g, k, p.w_dt));
    const float xh = (ld1(p.x, t * p.ld_x + k, p.x_dt) - mu) * r;
    float o = r * (u - s - xh * q);
    if (p.dres) o += ld1(p.dres, t * p.ld_dres + k, p.dres_dt);
    st1(p.dx, t * p.ld_dx + k, p.out_dt, o);
    if (p.dx_copy) st1(p.dx_copy, t * p.ld_dx + k, LC_BF16, o);
  }
}

int64_t blocks_of(int64_t T) { return (T + ROWS - 1) / ROWS; }
size_t scratch_of(int64_t T, int64_t d) {
  return T <= 0 || d <= 0 ? 0 : (size_t)blocks_of(T) * (size_t)d * 2 * sizeof(float);
}

lc_status check(const lc_layernorm_args &a, bool bwd) {
  if (a.T < 0 || a.d <= 0) return fail(LC_ERR_INVALID_ARG, "layernorm: T must be 0 or more, d positive");
  if (a.d > INT32_MAX || a.T > INT32_MAX) return fail(LC_ERR_UNSUPPORTED, "layernorm: 2^31 or more rows or values");
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
  p.T = a.T; p.d = a.d;
  p.ld_x = ld(a.ld_x); p.ld_y = ld(a.ld_y); p.ld_dy = ld(a.ld_dy); p.ld_dres = ld(a.ld_dres); p.ld_dx = ld(a.ld_dx);
  p.eps = a.eps;
  p.x_dt = a.x_dtype; p.w_dt = a.w_dtype; p.out_dt = a.out_dtype; p.dy_dt = a.dy_dtype; p.dres_dt = a.dres_dtype;
  p.store = a.store_dg != 0;
  p.nblk = (int)blocks_of(a.T);
  p.pg = static_cast<float *>(a.scratch);
  p.pb = p.pg ? p.pg + (size_t)p.nblk * a.d : nullptr;
  return p;
}

lc_status forward(const lc_layernorm_args &a, hipStream_t s) {
  LC_TRY(check(a, false));
  if (a.T == 0) return LC_OK;
  const LnP p = params(a);
  hipLaunchKernelGGL(layernorm_fwd_kernel, dim3((unsigned)p.T), dim3(NTH), 0, s, p);
  return check_launch("layernorm_fwd_kernel");
}

lc_status backward(const lc_layernorm_args &a, hipStream_t s) {
  LC_TRY(check(a, true));
  if (a.T == 0) return LC_OK;
  const LnP p = params(a);
  const unsigned cols = ceil_div((size_t)p.d, NTH);
  const bool sums = p.dg || p.db;
  if (sums) {  // before dx, which may lie over dy
    hipLaunchKernelGGL(layernorm_partial_kernel, dim3(cols, (unsigned)p.nblk), dim3(NTH), 0, s, p);
    LC_TRY(check_launch("layernorm_partial_kernel"));
    hipLaunchKernelGGL(layernorm_final_kernel, dim3(cols), dim3(NTH), 0, s, p);
    LC_TRY(check_launch("layernorm_final_kernel"));
  }
  hipLaunchKernelGGL(layernorm_bwd_kernel, dim3((unsigned)p.T), dim3(NTH), 0, s, p);
  return check_launch("layernorm_bwd_kernel");
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
