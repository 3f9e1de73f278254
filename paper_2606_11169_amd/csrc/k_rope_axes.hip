// Rotary positions with several axes (time, height, width): the rotation of head
// rows, its transpose, and the cos/sin table.
//
// Pair i turns by pos[axis(i)] f_i. In turns that is pos f_i / (2 pi); its fraction
// is formed exactly in integers: F_i = round(2^64 f_i / (2 pi)) (computed in 80-bit
// floating point on the host), and pos F_i mod 2^64 is the fraction of a turn in
// units of 2^-64, off by at most 2^31 (2^-1 + 2^-64 relative of F_i's own rounding),
// under 1e-8 rad at any position. The nearest multiple of a quarter turn is split
// off in integers too, so sin and cos are taken of at most pi/4, where their Taylor
// series to x^11 and x^12 are exact to fp32.
#include "common.hpp"

#include <math.h>

namespace lc {
namespace {

constexpr int NTH = 256;
constexpr int MAXPAIR = 128;

struct RopeP {
  uint64_t turn[MAXPAIR];  // 2^64 f / (2 pi) of every pair
  uint8_t axis[MAXPAIR];   // (pairs past the sections: turn 0)
  const int32_t *pos;
  int64_t ld_pos;
  const void *x;
  void *y;
  int64_t ld_x, ld_y, T;
  float *cos, *sin;
  int heads, half, x_dt, y_dt;
  float sign;  // 1 forward, -1 backward
};

// cos and sin of the angle 2 pi u / 2^64
__device__ __forceinline__ void cos_sin(uint64_t u, float &c, float &s) {
  const uint32_t quarter = (uint32_t)((u + (1ull << 61)) >> 62);
  const int64_t rest = (int64_t)(u - ((uint64_t)quarter << 62));  // within an eighth of a turn
  const float x = (float)rest * 3.40612158008655459e-19f;         // 2 pi / 2^64
  const float x2 = x * x;
  const float sx = x + x * x2 * (-1.6666667e-1f + x2 * (8.3333333e-3f + x2 * (-1.9841270e-4f +
                   x2 * (2.7557319e-6f + x2 * -2.5052108e-8f))));
  const float cx = 1.0f + x2 * (-0.5f + x2 * (4.1666667e-2f + x2 * (-1.3888889e-3f + x2 * (2.4801587e-5f +
                   x2 * (-2.7557319e-7f + x2 * 2.0876757e-9f)))));
  const float a = quarter & 1 ? sx : cx, b = quarter & 1 ? cx : sx;
  c = quarter == 1 || quarter == 2 ? -a : a;
  s = quarter & 2 ? -b : b;
}

__device__ __forceinline__ void pair_cos_sin(const RopeP &p, int64_t t, int i, float &c, float &s) {
  const int64_t at = p.pos[p.axis[i] * p.ld_pos + t];
  cos_sin((uint64_t)at * p.turn[i], c, s);
}

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

// one workgroup per token
__global__ __launch_bounds__(NTH) void rope_axes_kernel(RopeP p) {
  const int64_t t = blockIdx.x;
  for (int n = threadIdx.x; n < p.heads * p.half; n += NTH) {
    const int h = n / p.half, i = n % p.half;
    float c, s;
    pair_cos_sin(p, t, i, c, s);
    s *= p.sign;
    const int64_t at = (int64_t)h * 2 * p.half + i;
    const float a = ld1(p.x, t * p.ld_x + at, p.x_dt), b = ld1(p.x, t * p.ld_x + at + p.half, p.x_dt);
    st1(p.y, t * p.ld_y + at, p.y_dt, a * c - b * s);
    st1(p.y, t * p.ld_y + at + p.half, p.y_dt, b * c + a * s);
  }
}

__global__ __launch_bounds__(NTH) void rope_table_kernel(RopeP p) {
  const int64_t n = (int64_t)blockIdx.x * NTH + threadIdx.x;
  if (n >= p.T * p.half) return;
  float c, s;
  pair_cos_sin(p, n / p.half, (int)(n % p.half), c, s);
  p.cos[n] = c;
  p.sin[n] = s;
}

enum Kind { FORWARD, BACKWARD, TABLE };

lc_status check(const lc_rope_axes_args &a, Kind kind) {
  if (a.T < 0) return fail(LC_ERR_INVALID_ARG, "rope axes: T must be 0 or more");
  if (a.T > INT32_MAX) return fail(LC_ERR_UNSUPPORTED, "rope axes: 2^31 or more tokens");
  if (a.hd < 2 || a.hd % 2 || a.hd > 2 * MAXPAIR)
    return fail(LC_ERR_UNSUPPORTED, "rope axes: hd must be even, 2 to %d", 2 * MAXPAIR);
  if (a.n_axes < 1 || a.n_axes > 4) return fail(LC_ERR_INVALID_ARG, "rope axes: 1 to 4 axes");
  int64_t sum = 0;
  for (int i = 0; i < a.n_axes; ++i) {
    if (a.sections[i] < 0) return fail(LC_ERR_INVALID_ARG, "rope axes: negative section");
    sum += a.sections[i];
  }
  if (sum < 1 || sum > a.hd / 2)
    return fail(LC_ERR_INVALID_ARG, "rope axes: the sections must sum to 1 .. hd/2 pairs");
  if (a.freq != LC_ROPE_FREQ_HEAD && a.freq != LC_ROPE_FREQ_AXIS)
    return fail(LC_ERR_INVALID_ARG, "rope axes: unknown freq");
  if (!(a.base >= 1.0f) || !(a.base < INFINITY)) return fail(LC_ERR_INVALID_ARG, "rope axes: base must be finite, 1 or more");
  if (a.n_axes > 1 && a.ld_pos < a.T) return fail(LC_ERR_INVALID_ARG, "rope axes: ld_pos smaller than T");
  if (kind != TABLE) {
    const int64_t width = (int64_t)a.n_heads * a.hd;
    if (a.n_heads <= 0 || width > INT32_MAX) return fail(LC_ERR_INVALID_ARG, "rope axes: bad number of heads");
    if (!valid_dtype(a.x_dtype) || !valid_dtype(a.y_dtype)) return fail(LC_ERR_INVALID_ARG, "rope axes: unknown dtype");
    const int64_t most = INT64_MAX / 4 / (a.T + 1);
    if (a.ld_x < width || a.ld_y < width || a.ld_x > most || a.ld_y > most)
      return fail(LC_ERR_INVALID_ARG, "rope axes: leading dimension smaller than n_heads * hd (or past 64 bits)");
  }
  if (a.T == 0) return LC_OK;
  if (!a.pos || (reinterpret_cast<uintptr_t>(a.pos) & 3)) return fail(LC_ERR_INVALID_ARG, "rope axes: null or unaligned pos");
  if (kind == TABLE) {
    if (!a.cos || !a.sin || !aligned16(a.cos) || !aligned16(a.sin))
      return fail(LC_ERR_INVALID_ARG, "rope axes: null or unaligned table");
  } else if (!a.x || !a.y || !aligned16(a.x) || !aligned16(a.y)) {
    return fail(LC_ERR_INVALID_ARG, "rope axes: null or unaligned pointer");
  }
  return LC_OK;
}

RopeP params(const lc_rope_axes_args &a, Kind kind) {
  RopeP p{};
  const long double turns = powl(2.0L, 63) / 3.14159265358979323846264338327950288L;  // 2^64 / (2 pi)
  int i = 0;
  for (int ax = 0; ax < a.n_axes; ++ax) {
    const int n = a.freq == LC_ROPE_FREQ_AXIS ? a.sections[ax] : a.hd / 2;
    const long double step = n > 0 ? powl((long double)a.base, -1.0L / n) : 1.0L;
    long double f = a.freq == LC_ROPE_FREQ_AXIS ? 1.0L : powl((long double)a.base, -(long double)i / n);
    for (int j = 0; j < a.sections[ax]; ++j, ++i, f *= step) {
      p.turn[i] = (uint64_t)llroundl(f * turns);  // (at most 2^62)
      p.axis[i] = (uint8_t)ax;
    }
  }
  p.pos = a.pos;
  p.ld_pos = a.ld_pos;
  p.x = a.x;
  p.y = a.y;
  p.ld_x = a.ld_x;
  p.ld_y = a.ld_y;
  p.T = a.T;
  p.cos = a.cos;
  p.sin = a.sin;
  p.heads = a.n_heads;
  p.half = a.hd / 2;
  p.x_dt = a.x_dtype;
  p.y_dt = a.y_dtype;
  p.sign = kind == BACKWARD ? -1.0f : 1.0f;
  return p;
}

lc_status run(const lc_rope_axes_args *args, Kind kind, void *stream) {
  if (!args) return fail(LC_ERR_INVALID_ARG, "rope axes: null args");
  LC_TRY(check(*args, kind));
  if (args->T == 0) return LC_OK;
  const RopeP p = params(*args, kind);
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (kind == TABLE) {
    hipLaunchKernelGGL(rope_table_kernel, dim3(ceil_div((size_t)p.T * p.half, NTH)), dim3(NTH), 0, s, p);
    return check_launch("rope_table_kernel");
  }
  hipLaunchKernelGGL(rope_axes_kernel, dim3((unsigned)p.T), dim3(NTH), 0, s, p);
  return check_launch("rope_axes_kernel");
}

}  // namespace
}  // namespace lc

extern "C" {

lc_status lc_rope_axes_forward(const lc_rope_axes_args *args, void *stream) {
  return lc::run(args, lc::FORWARD, stream);
}
lc_status lc_rope_axes_backward(const lc_rope_axes_args *args, void *stream) {
  return lc::run(args, lc::BACKWARD, stream);
}
lc_status lc_rope_axes_table(const lc_rope_axes_args *args, void *stream) {
  return lc::run(args, lc::TABLE, stream);
}

}  // extern "C"
