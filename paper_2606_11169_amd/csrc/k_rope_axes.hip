// Rotary positions with several axes (time, height, width): the rotation of head
// rows, its transpose, and the cos/sin table.
//
// Pair i turns by pos[axis(i)] f_i. In turns that is pos f_i / (2 pi); its fraction
// is formed exactly in integers: F_i = round(2^64 f_i / (2 pi)) (computed in 80-bit
// floating point on the host, f_i by at most 127 products of 2^-63 each), and pos F_i
// mod 2^64 is the fraction of a turn in units of 2^-64. At position 2^31 that is off by
// F_i's half unit, 2^31 2^-65 turns < 1e-9 rad, and by f_i's error, i 2^-63 f_i 2^31 <
// 2^-25 rad (f_i = 1 throughout; 1e-9 rad with base 10000). The nearest multiple of a
// quarter turn is split off in integers too, so sin and cos are taken of at most pi/4, where
// their Taylor series to x^11 and x^12 are exact to fp32.
//
// The rotation is bound by the memory traffic of the head rows (each read and written
// once). A token's cos and sin are formed once for all of its heads: hd / 2 pairs are
// RUN = 8 (4, 2, 1) consecutive ones per lane, the lanes of a group hold a head's pairs, and
// the wave's groups walk the token's heads with the same cos and sin in registers. Few
// tokens share out their heads over more waves instead, so that the chip is filled. Measured: 32760
// tokens of 24 heads of 128, bf16, 76 us, 5.3 TB/s (a large copy reaches 5.1 to 5.5 here); 1601 of 40
// heads 8.6 us, a launch and two dependent loads; a table of 8192 x 64 4.0 us.
#include "common.hpp"

#include <math.h>

namespace lc {
namespace {

constexpr int NTH = 256;
constexpr int MAXPAIR = 128;

// N: pairs that it has room for (64: up to 128 values per head; the arguments of a launch cost
// host time by their size)
template <int N> struct RopeP {
  uint64_t turn[N];  // 2^64 f / (2 pi) of every pair (past the sections: 0)
  int32_t end[3];    // first pair past the section of axis 0, 1, 2
  const int32_t *pos;
  int64_t ld_pos;
  const void *x;
  void *y;
  int64_t ld_x, ld_y, T;
  float *cos, *sin;
  int heads, half, axes, x_dt, y_dt;
  int turned;      // pairs in the sections
  int lpg, share;  // lanes per group; waves that share a token's heads
  int64_t first;   // the launch's first workgroup
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

// (a pair past the sections takes the last axis' position times 0)
template <typename P>
__device__ __forceinline__ void pair_cos_sin(const P &p, int64_t t, int i, float &c, float &s) {
  const int axis = min((i >= p.end[0]) + (i >= p.end[1]) + (i >= p.end[2]), p.axes - 1);
  const int64_t at = p.pos[axis * p.ld_pos + t];
  cos_sin((uint64_t)at * p.turn[i], c, s);
}

// RUN consecutive values of a row at any alignment (the instruction takes any address), as
// floats and back; SZ bytes per value, the 16-bit type a run-time choice of the conversion
template <int N> struct Words;
template <> struct Words<4> { typedef uint32_t type __attribute__((aligned(2))); };
template <> struct Words<8> { typedef __attribute__((ext_vector_type(2))) uint32_t v; typedef v type __attribute__((aligned(2))); };
template <> struct Words<16> { typedef __attribute__((ext_vector_type(4))) uint32_t v; typedef v type __attribute__((aligned(2))); };

template <int SZ, int RUN> struct Vals {
  static constexpr int BYTES = SZ * RUN;
  uint32_t w[BYTES < 4 ? 1 : BYTES / 4];
  __device__ __forceinline__ void load(const char *at) {
    if constexpr (BYTES >= 16) {
#pragma unroll
      for (int i = 0; i < BYTES / 16; ++i)
        __builtin_memcpy(w + 4 * i, reinterpret_cast<const Words<16>::type *>(at) + i, 16);
    } else if constexpr (BYTES == 8) {
      __builtin_memcpy(w, reinterpret_cast<const Words<8>::type *>(at), 8);
    } else if constexpr (BYTES == 4) {
      w[0] = *reinterpret_cast<const Words<4>::type *>(at);
    } else {
      w[0] = *reinterpret_cast<const uint16_t *>(at);
    }
  }
  __device__ __forceinline__ void store(char *at) const {
    if constexpr (BYTES >= 16) {
#pragma unroll
      for (int i = 0; i < BYTES / 16; ++i)
        __builtin_memcpy(reinterpret_cast<Words<16>::type *>(at) + i, w + 4 * i, 16);
    } else if constexpr (BYTES == 8) {
      __builtin_memcpy(reinterpret_cast<Words<8>::type *>(at), w, 8);
    } else if constexpr (BYTES == 4) {
      *reinterpret_cast<Words<4>::type *>(at) = w[0];
    } else {
      *reinterpret_cast<uint16_t *>(at) = (uint16_t)w[0];
    }
  }
  __device__ __forceinline__ float get(int i, int dt) const {
    if constexpr (SZ == 4) return __uint_as_float(w[i]);
    const uint16_t h = (uint16_t)(w[i >> 1] >> (16 * (i & 1)));
    return dt == LC_BF16 ? __uint_as_float((uint32_t)h << 16) : (float)__builtin_bit_cast(_Float16, h);
  }
  __device__ __forceinline__ void put(const float (&x)[RUN], int dt) {
#pragma unroll
    for (int i = 0; i < RUN; ++i) {
      if constexpr (SZ == 4) {
        w[i] = __float_as_uint(x[i]);
      } else {
        const uint16_t h = dt == LC_BF16 ? __builtin_bit_cast(uint16_t, (__bf16)x[i])
                                         : __builtin_bit_cast(uint16_t, (_Float16)x[i]);
        if (i & 1) w[i >> 1] |= (uint32_t)h << 16;
        else w[i >> 1] = h;
      }
    }
  }
};

// Groups of p.lpg lanes (a power of two; lane l holds pairs RUN l ..) take a token's heads in
// turn; a group's heads are h0, h0 + stride, ..., those of `p.share` waves side by side.
template <int XS, int YS, int RUN, int N>
__global__ __launch_bounds__(NTH) void rope_axes_kernel(RopeP<N> p) {
  const int lane = threadIdx.x & 63, l = lane % p.lpg;
  const int64_t w = (p.first + blockIdx.x) * (NTH / 64) + (threadIdx.x >> 6);
  const int64_t t = w / p.share;
  if (t >= p.T) return;  // (a whole wave)
  const int groups = 64 / p.lpg, stride = groups * p.share;
  const int64_t hd = 2 * p.half;
  const int h0 = (int)(w % p.share) * groups + lane / p.lpg;
  const char *x = static_cast<const char *>(p.x) + t * p.ld_x * XS;
  char *y = static_cast<char *>(p.y) + t * p.ld_y * YS;
  // (RUN = 1: up to 127 pairs on 64 lanes)
  constexpr int ROUNDS = RUN == 1 && N > 64 ? 2 : 1;
  Vals<XS, RUN> a, b;
  auto first = [&](int i0) {
    if (i0 < p.half && h0 < p.heads) {
      a.load(x + (h0 * hd + i0) * XS);
      b.load(x + (h0 * hd + i0 + p.half) * XS);
    }
  };
  first(RUN * l);  // (on their way while cos and sin are formed)
  // pairs `lane` and lane + 64
  float c0 = 1.0f, s0 = 0.0f, c1 = 1.0f, s1 = 0.0f;
  if (lane < p.half) pair_cos_sin(p, t, lane, c0, s0);
  if (N > 64 && lane + 64 < p.half) pair_cos_sin(p, t, lane + 64, c1, s1);
#pragma unroll
  for (int round = 0; round < ROUNDS; ++round) {
    const int i0 = RUN * (l + p.lpg * round);
    if (round) {
      if (p.lpg >= p.half) break;
      first(i0);
    }
    float c[RUN], s[RUN];
#pragma unroll
    for (int i = 0; i < RUN; ++i) {
      const int from = (i0 + i) & 63;
      c[i] = __shfl(c0, from, 64);
      s[i] = __shfl(s0, from, 64);
      if (N > 64) {
        const float ch = __shfl(c1, from, 64), sh = __shfl(s1, from, 64);
        c[i] = i0 + i < 64 ? c[i] : ch;
        s[i] = i0 + i < 64 ? s[i] : sh;
      }
      s[i] *= p.sign;
    }
    if (i0 >= p.half) continue;
    const bool stays = i0 + RUN > p.turned;  // some pair of the run lies past the sections
    int h = h0;
    while (h < p.heads) {
      const int hn = h + stride;
      Vals<XS, RUN> an, bn;
      if (hn < p.heads) {
        an.load(x + (hn * hd + i0) * XS);
        bn.load(x + (hn * hd + i0 + p.half) * XS);
      }
      float u[RUN], v[RUN];
#pragma unroll
      for (int i = 0; i < RUN; ++i) {
        const float ai = a.get(i, p.x_dt), bi = b.get(i, p.x_dt);
        u[i] = ai * c[i] - bi * s[i];
        v[i] = bi * c[i] + ai * s[i];
      }
      if (stays) {  // (whatever its partner holds: inf 0 is NaN)
#pragma unroll
        for (int i = 0; i < RUN; ++i)
          if (i0 + i >= p.turned) {
            u[i] = a.get(i, p.x_dt);
            v[i] = b.get(i, p.x_dt);
          }
      }
      Vals<YS, RUN> o;
      o.put(u, p.y_dt);
      o.store(y + (h * hd + i0) * YS);
      o.put(v, p.y_dt);
      o.store(y + (h * hd + i0 + p.half) * YS);
      a = an;
      b = bn;
      h = hn;
    }
  }
}

template <int N>
__global__ __launch_bounds__(NTH) void rope_table_kernel(RopeP<N> p) {
  const int64_t n = (p.first + blockIdx.x) * NTH + threadIdx.x;
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

template <int N>
RopeP<N> params(const lc_rope_axes_args &a, Kind kind) {
  RopeP<N> p{};
  const long double turns = 0x1p63L / 3.14159265358979323846264338327950288L;  // 2^64 / (2 pi)
  // f goes down by the same factor from pair to pair (over the head, or from 1 in each section)
  const bool own = a.freq == LC_ROPE_FREQ_AXIS;
  long double f = 1.0L, step = 1.0L;
  int i = 0, run = 0;
  for (int ax = 0; ax < a.n_axes; ++ax) {
    const int n = own ? a.sections[ax] : a.hd / 2;
    if (n > 0 && n != run) {
      step = powl((long double)a.base, -1.0L / n);
      run = n;
    }
    if (own) f = 1.0L;
    for (int j = 0; j < a.sections[ax]; ++j, ++i, f *= step) p.turn[i] = (uint64_t)llroundl(f * turns);  // (under 2^62)
    if (ax < 3) p.end[ax] = i;
  }
  p.turned = i;
  for (int ax = a.n_axes; ax < 3; ++ax) p.end[ax] = N;
  p.axes = a.n_axes;
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

template <int XS, int YS, int N>
void rotate(RopeP<N> p, hipStream_t s) {
  // the longest run that a head's pairs consist of (16-byte accesses at 8 values of 16 bits)
  const int run = p.half % 8 == 0 ? 8 : p.half % 4 == 0 ? 4 : p.half % 2 == 0 ? 2 : 1;
  p.lpg = 1;
  while (p.lpg * run < p.half && p.lpg < 64) p.lpg *= 2;
  const int groups = 64 / p.lpg;
  // waves that share a token: up to one per `groups` heads while the tokens' waves are fewer
  // than 16 per compute unit
  p.share = 1;
  while (p.share * groups < p.heads && p.T * p.share < 4096) p.share *= 2;
  const int64_t wgs = (p.T * p.share + NTH / 64 - 1) / (NTH / 64);
  launch_parts((uint32_t)wgs, [&](uint32_t first, uint32_t count) {
    p.first = first;
    if (run == 8) hipLaunchKernelGGL((rope_axes_kernel<XS, YS, 8, N>), dim3(count), dim3(NTH), 0, s, p);
    else if (run == 4) hipLaunchKernelGGL((rope_axes_kernel<XS, YS, 4, N>), dim3(count), dim3(NTH), 0, s, p);
    else if (run == 2) hipLaunchKernelGGL((rope_axes_kernel<XS, YS, 2, N>), dim3(count), dim3(NTH), 0, s, p);
    else hipLaunchKernelGGL((rope_axes_kernel<XS, YS, 1, N>), dim3(count), dim3(NTH), 0, s, p);
  });
}

template <int N>
lc_status launch(const lc_rope_axes_args &a, Kind kind, hipStream_t s) {
  RopeP<N> p = params<N>(a, kind);
  if (kind == TABLE) {
    launch_parts(ceil_div((size_t)p.T * p.half, NTH), [&](uint32_t first, uint32_t count) {
      p.first = first;
      hipLaunchKernelGGL(rope_table_kernel<N>, dim3(count), dim3(NTH), 0, s, p);
    });
    return check_launch("rope_table_kernel");
  }
  if (p.x_dt == LC_FP32) {
    if (p.y_dt == LC_FP32) rotate<4, 4, N>(p, s);
    else rotate<4, 2, N>(p, s);
  } else {
    if (p.y_dt == LC_FP32) rotate<2, 4, N>(p, s);
    else rotate<2, 2, N>(p, s);
  }
  return check_launch("rope_axes_kernel");
}

lc_status run(const lc_rope_axes_args *args, Kind kind, void *stream) {
  if (!args) return fail(LC_ERR_INVALID_ARG, "rope axes: null args");
  LC_TRY(check(*args, kind));
  if (args->T == 0) return LC_OK;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  return args->hd <= 128 ? launch<64>(*args, kind, s) : launch<MAXPAIR>(*args, kind, s);
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
