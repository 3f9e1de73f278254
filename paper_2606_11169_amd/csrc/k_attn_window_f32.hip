// Sliding-window causal attention with sinks over packed sequences, the fp32 path, on the
// fp32 matrix instruction (fragments, merge and the treatment of non-finite values at masked
// pairs: attn_f32.hpp; windows, sinks and packed rows: k_attn_window.hip).
//
// A workgroup owns 16 packed rows of one head, whatever sequences they belong to, and its
// four waves take the visible blocks of 32 keys in turn: the first row's sinks, then from its window on.
// dK/dV: 16 key rows of a key/value head; the waves (eight of head_dim above 64) take (query
// head, block of 32 queries) in turn, up to the end of the window of the last key or, where a sink is among the keys,
// of its sequence.
//
// Measured: 600 tokens in 4 sequences, 12 heads of 64, window 128: forward 13 us, dQ 17, dK/dV 23, where
// a single workgroup of one block takes 7.5, 9 and 9.6: a chain of dependent loads (offsets, rows,
// keys, values) with 0.9 us of products per block. 2000 causal tokens, 12 heads: of 64 128, 180 and
// 230 us, 31 to 35% of the fp32 matrix rate, of 128 225, 333 and 420, 36 to 38%: each wave brings its
// blocks' rows itself, 32 KB per 128 products of head_dim 64, and waits for them.
#include "attn_f32.hpp"
#include "attn_window.hpp"

namespace lc {
namespace {

struct WinF {
  const float *q, *k, *v, *dout;
  float *o, *dq, *dk, *dv;
  float *lse, *D;
  const int32_t *off;
  int64_t ld_q, ld_k, ld_v, ld_o, ld_do, ld_dq, ld_dk, ld_dv;
  int T, B, S, H, Hkv, G, hd, window, n_sink;
  int first;  // the launch's first workgroup
  int vec_q, vec_k, vec_v, vec_o, vec_do;  // rows are made of whole 16-byte runs
  float scale;
};

__device__ __forceinline__ int col_min(int x) {  // over the 16 columns, alike in the four groups
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) x = min(x, __shfl_xor(x, o, 64));
  return x;
}
__device__ __forceinline__ int col_max16(int x) {
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) x = max(x, __shfl_xor(x, o, 64));
  return x;
}

// 16 query rows from q0 on: what this lane's row (column c) sees, and the workgroup's blocks
struct Rows {
  int row, start, wlo, nwin, ns, wmax, last;
  int sb0, nsb, wb0, nit;
  __device__ __forceinline__ int block(int it) const { return it < nsb ? sb0 + it : wb0 + it - nsb; }
  __device__ __forceinline__ bool sees(int key) const {
    return (uint32_t)(key - wlo) < (uint32_t)nwin || (uint32_t)(key - start) < (uint32_t)ns;
  }
  __device__ __forceinline__ bool all(int k0, int q0) const { return k0 >= wmax && k0 + KB - 1 <= q0; }
};
__device__ __forceinline__ bool rows_of(const WinF &p, int q0, int lane, Rows &R) {
  const Sequences sq(p.off, p.S, p.T, p.B, lane);
  const int r0 = max(q0, sq.first), r1 = min(q0 + QR, sq.last) - 1;
  int b0, s0, e0;
  if (r0 > r1 || !sq.of_wave(r0, lane, b0, s0, e0)) return false;
  const int W = p.window;
  R.wb0 = max(s0, r0 - W + 1) / KB;
  const int lr = min(r1, e0 - 1), cnt = min(p.n_sink, max(s0, lr - W + 1) - s0);
  R.sb0 = s0 / KB;
  R.nsb = cnt > 0 ? max(0, min((s0 + cnt - 1) / KB, R.wb0 - 1) - R.sb0 + 1) : 0;
  R.nit = max(0, R.nsb + r1 / KB - R.wb0 + 1);
  R.row = q0 + (lane & 15);
  bool ok = R.row >= r0 && R.row <= r1;
  R.start = s0;
  if (r1 >= e0) {  // (more than one sequence)
    int end;
    ok = sq.of_lane(R.row, b0, R.start, end) && ok;
  }
  R.wlo = max(R.start, R.row - W + 1);
  R.nwin = ok ? max(0, R.row - R.wlo + 1) : 0;
  R.ns = ok ? min(p.n_sink, R.wlo - R.start) : 0;
  R.wmax = col_max16(ok ? R.wlo : 0x7FFFFFFF);
  return true;
}

// Block of rows and head of a workgroup, heads fastest
__device__ __forceinline__ void place(const WinF &p, int heads, int &r0, int &h) {
  const int i = p.first + (int)blockIdx.x;
  r0 = i / heads * QR;
  h = i % heads;
}

template <int NI>
__global__ __launch_bounds__(NTF) void window_f32_fwd_kernel(WinF p) {
  __shared__ __align__(16) float so[Merge<NI>::FLOATS];
  __shared__ float sm[NW][QR], sl[NW][QR], sf[NW + 1][QR];
  __shared__ int live[QR];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, g = lane >> 4, c = lane & 15;
  int q0, h;
  place(p, p.H, q0, h);
  Rows R;
  if (!rows_of(p, q0, lane, R)) return;
  const int64_t hk = (int64_t)(h / p.G) * p.hd;
  const float *K = p.k + hk, *V = p.v + hk;
  const int last = p.T - 1;
  float qf[NI][4];
  load_frag<NI>(p.q + min(R.row, last) * p.ld_q + (int64_t)h * p.hd, g, p.hd, p.vec_q, qf);
  f32x4_v o[NI];
#pragma unroll
  for (int i = 0; i < NI; ++i) o[i] = f32x4_v{0.0f, 0.0f, 0.0f, 0.0f};
  float m = -INFINITY, l = 0.0f;
  auto vis = [&](int key) { return R.sees(key); };
  for (int it = w; it < R.nit; it += NW) {
    const int k0 = R.block(it) * KB;
    f32x4_v s[2];
    float mx = -INFINITY;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      float kf[NI][4];
      load_frag<NI>(K + (int64_t)min(k0 + 16 * t + c, last) * p.ld_k, g, p.hd, p.vec_k, kf);
      s[t] = score<NI>(kf, qf);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        s[t][r] = vis(k0 + 16 * t + 4 * g + r) ? s[t][r] * p.scale : -INFINITY;
        mx = fmaxf(mx, s[t][r]);
      }
    }
    const float mn = fmaxf(m, col_max(mx));
    const float mu = mn == -INFINITY ? 0.0f : mn;  // nothing seen yet: weights of 0
    const float alpha = expf(m - mu);
#pragma unroll
    for (int i = 0; i < NI; ++i) o[i] *= alpha;
    l *= alpha;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        s[t][r] = expf(s[t][r] - mu);
        l += s[t][r];
      }
    m = mn;
    accumulate<NI>(o, s, V, p.ld_v, k0, last, p.hd, p.vec_v, lane, !R.all(k0, q0), vis);
  }
  l = col_sum(l);
  Merge<NI>::put(so, o, w, lane);
  if (g == 0) {
    sm[w][c] = m;
    sl[w][c] = l;
  }
  __syncthreads();
  if (tid < QR) {  // weights of the waves' shares of query q0 + tid
    float mm = sm[0][tid];
#pragma unroll
    for (int i = 1; i < NW; ++i) mm = fmaxf(mm, sm[i][tid]);
    const float mu = mm == -INFINITY ? 0.0f : mm;
    float L = 0.0f;
#pragma unroll
    for (int i = 0; i < NW; ++i) {
      sf[i][tid] = expf(sm[i][tid] - mu);
      L += sf[i][tid] * sl[i][tid];
    }
    sf[NW][tid] = L;
    live[tid] = R.nwin > 0;  // (thread tid holds row q0 + tid)
    if (R.nwin > 0) p.lse[(int64_t)h * p.T + q0 + tid] = mm + logf(L);
  }
  __syncthreads();
  for (int x = tid; x < QR * p.hd; x += NTF) {
    const int qr = x / p.hd, e = x % p.hd;
    if (!live[qr]) continue;
    float v = 0.0f;
#pragma unroll
    for (int i = 0; i < NW; ++i) v += sf[i][qr] * so[(i * QR + qr) * Merge<NI>::LD + e];
    p.o[(q0 + qr) * p.ld_o + (int64_t)h * p.hd + e] = v / sf[NW][qr];
  }
}

// per 16 queries: D (written for the dK/dV kernel) and dQ. Bound to two waves per SIMD: above
// head_dim 64 it would take registers of one (2000 causal tokens, 12 heads of 128: 508 -> 333 us)
template <int NI>
__global__ __launch_bounds__(NTF, 2) void window_f32_dq_kernel(WinF p) {
  __shared__ __align__(16) float sq[Merge<NI>::FLOATS];
  __shared__ int live[QR];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, g = lane >> 4, c = lane & 15;
  int q0, h;
  place(p, p.H, q0, h);
  Rows R;
  if (!rows_of(p, q0, lane, R)) return;
  if (tid < QR) live[tid] = R.nwin > 0;
  const int64_t hq = (int64_t)h * p.hd, hk = (int64_t)(h / p.G) * p.hd;
  const float *K = p.k + hk, *V = p.v + hk;
  const int last = p.T - 1, qc = min(R.row, last);
  auto vis = [&](int key) { return R.sees(key); };
  float qf[NI][4], df[NI][4];
  load_frag<NI>(p.q + qc * p.ld_q + hq, g, p.hd, p.vec_q, qf);
  load_frag<NI>(p.dout + qc * p.ld_do + hq, g, p.hd, p.vec_do, df);
  float Dq = 0.0f;
  {
    float of[NI][4];
    load_frag<NI>(p.o + qc * p.ld_o + hq, g, p.hd, p.vec_o, of);
#pragma unroll
    for (int j = 0; j < NI; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) Dq += df[j][e] * of[j][e];
  }
  Dq = col_sum(Dq);
  const int64_t si = (int64_t)h * p.T + qc;
  const float L = p.lse[si];
  if (w == 0 && g == 0 && R.nwin > 0) p.D[si] = Dq;
  f32x4_v acc[NI];
#pragma unroll
  for (int i = 0; i < NI; ++i) acc[i] = f32x4_v{0.0f, 0.0f, 0.0f, 0.0f};
  for (int it = w; it < R.nit; it += NW) {
    const int k0 = R.block(it) * KB;
    f32x4_v ds[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      float kf[NI][4], vf[NI][4];
      const int64_t kr = min(k0 + 16 * t + c, last);
      load_frag<NI>(K + kr * p.ld_k, g, p.hd, p.vec_k, kf);
      load_frag<NI>(V + kr * p.ld_v, g, p.hd, p.vec_v, vf);
      const f32x4_v s = score<NI>(kf, qf), dp = score<NI>(vf, df);
#pragma unroll
      for (int r = 0; r < 4; ++r)
        ds[t][r] = vis(k0 + 16 * t + 4 * g + r) ? expf(s[r] * p.scale - L) * (dp[r] - Dq) : 0.0f;
    }
    accumulate<NI>(acc, ds, K, p.ld_k, k0, last, p.hd, p.vec_k, lane, !R.all(k0, q0), vis);
  }
  Merge<NI>::put(sq, acc, w, lane);
  __syncthreads();
  for (int x = tid; x < QR * p.hd; x += NTF) {
    const int r = x / p.hd, e = x % p.hd;
    if (live[r]) p.dq[(q0 + r) * p.ld_dq + hq + e] = Merge<NI>::sum(sq, r, e) * p.scale;
  }
}

// rows 16 t + 4 g + r of a block at r0 (at most row `last`), features NI c ..: accumulate_rows' operand
template <int NI>
__device__ __forceinline__ void load_rows(float (&x)[2][4][NI], const float *x0, int64_t ld, int r0, int last, int hd,
                                          bool vec, int lane) {
  const int g = lane >> 4, c = lane & 15;
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r)
      load_run<NI>(x0 + (int64_t)min(r0 + 16 * t + 4 * g + r, last) * ld, NI * c, hd, vec, x[t][r]);
}

// accumulate (attn_f32.hpp) with the rows' values in x, loaded earlier
template <int NI, typename F>
__device__ __forceinline__ void accumulate_rows(f32x4_v (&acc)[NI], const f32x4_v (&w)[2], const float (&x)[2][4][NI],
                                           const float *x0, int64_t ld, int r0, int last, int hd, int lane,
                                           bool masked, F vis) {
  const int g = lane >> 4, c = lane & 15;
  if (masked) {
    bool bad = false;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int i = 0; i < NI; ++i) bad |= !(fabsf(x[t][r][i]) < INFINITY);
    if (__any(bad)) {
#pragma unroll 1
      for (int n = 0; n < 32; ++n) {
        const int row = r0 + n, t = n >> 4, r = n & 3;
        float mine = 0.0f;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (u == t && e == r) mine = w[u][e];
        const float wv = __shfl(mine, c + 16 * ((n >> 2) & 3), 64);
        if (row > last || !vis(row)) continue;
#pragma unroll
        for (int i = 0; i < NI; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int f = NI * (4 * g + e) + i;
            if (f < hd) acc[i][e] += wv * x0[(int64_t)row * ld + f];
          }
      }
      return;
    }
  }
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int i = 0; i < NI; ++i) acc[i] = mfma4(x[t][r][i], w[t][r], acc[i]);
}

// per 16 keys and key/value head: dK, dV summed over the head's query heads (needs D from the
// kernel above)
template <int NI> constexpr int dkdv_waves() { return NI == 8 ? 8 : NW; }  // (why: KVL)

template <int NI>
__global__ __launch_bounds__(64 * dkdv_waves<NI>(), 2) void window_f32_dkdv_kernel(WinF p) {
  // Whether a block's loads are all issued before its products (both halves' fragments, the
  // second products' rows, lse and D): at head_dim up to 32 the registers are there (2000 tokens,
  // 12/4 heads of 32, window 700 190 -> 148 us).
  constexpr bool EARLY = NI < 4;
  // Above 64 K's and V's fragments, alike in all waves, are read from LDS for every half block, so
  // that two waves fit a SIMD (2000 causal tokens, 12 heads of 128: 538 -> 410 us), and they are one
  // workgroup's eight, so that few key/value heads have them too (2000 tokens, 12/4 heads of 80, window
  // 700: 393 us with four waves of any registers, 284).
  constexpr bool KVL = NI == 8;
  __shared__ __align__(16) float sk[Merge<NI, dkdv_waves<NI>()>::FLOATS], sv[Merge<NI, dkdv_waves<NI>()>::FLOATS];
  __shared__ int live[QR];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, g = lane >> 4, c = lane & 15;
  int k0, kvh;
  place(p, p.Hkv, k0, kvh);
  const Sequences sq(p.off, p.S, p.T, p.B, lane);
  const int r1 = min(k0 + QR, sq.last) - 1, last = p.T - 1;
  int b, s, e;
  if (r1 < max(k0, sq.first) || !sq.of_wave(r1, lane, b, s, e)) return;
  // this lane's key kj: the queries [kj, kj + cnt) see it
  const int kj = k0 + c;
  int ks = s, ke = e, cnt = 0;
  bool ok = kj <= r1;
  if (s > k0) ok = sq.of_lane(kj, 0, ks, ke) && ok;
  if (ok)
    cnt = max(0, kj - ks < p.n_sink || p.window >= ke - kj ? ke - kj : p.window);
  if (tid < QR) live[tid] = cnt > 0;
  const int qend = col_max16(kj + cnt), hi_min = col_min(cnt ? kj + cnt : -1);
  const int64_t hk = (int64_t)kvh * p.hd, kr = min(kj, last);
  float kf[KVL ? 1 : NI][4], vf[KVL ? 1 : NI][4];
  float4 *const kl = reinterpret_cast<float4 *>(sk) + lane, *const vl = reinterpret_cast<float4 *>(sv) + lane;
  if constexpr (KVL) {
    if (w < 2) {
      float x[NI][4];
      load_frag<NI>((w ? p.v + kr * p.ld_v : p.k + kr * p.ld_k) + hk, g, p.hd, w ? p.vec_v : p.vec_k, x);
#pragma unroll
      for (int j = 0; j < NI; ++j) (w ? vl : kl)[64 * j] = make_float4(x[j][0], x[j][1], x[j][2], x[j][3]);
    }
    __syncthreads();
  } else {
    load_frag<NI>(p.k + kr * p.ld_k + hk, g, p.hd, p.vec_k, kf);
    load_frag<NI>(p.v + kr * p.ld_v + hk, g, p.hd, p.vec_v, vf);
  }
  f32x4_v dk[NI], dv[NI];
#pragma unroll
  for (int i = 0; i < NI; ++i) dk[i] = dv[i] = f32x4_v{0.0f, 0.0f, 0.0f, 0.0f};
  // units: (query head of the group, block of 32 queries that reach the keys)
  const int qb0 = k0 / KB, nqb = max(0, (qend + KB - 1) / KB - qb0);
  for (int u = w; u < p.G * nqb; u += dkdv_waves<NI>()) {
    const int h = kvh * p.G + u / nqb, q0 = (qb0 + u % nqb) * KB;
    const int64_t hq = (int64_t)h * p.hd;
    const float *Q = p.q + hq, *dO = p.dout + hq;
    const float *lse = p.lse + (int64_t)h * p.T, *D = p.D + (int64_t)h * p.T;
    f32x4_v pr[2], ds[2];
    auto vis = [&](int qi) { return (uint32_t)(qi - kj) < (uint32_t)cnt; };
    float qf[2][NI][4], df[2][NI][4], L[2][4], Dq[2][4], xq[2][4][NI], xo[2][4][NI];
    auto load = [&](int t) {
      const int64_t qr = min(q0 + 16 * t + c, last);
      load_frag<NI>(Q + qr * p.ld_q, g, p.hd, p.vec_q, qf[t]);
      load_frag<NI>(dO + qr * p.ld_do, g, p.hd, p.vec_do, df[t]);
    };
    auto load_stats = [&](int t) {
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int at = min(q0 + 16 * t + 4 * g + r, last);
        L[t][r] = lse[at];
        Dq[t][r] = D[at];
      }
    };
    if (EARLY) {
      load(0);
      load(1);
      load_stats(0);
      load_stats(1);
      load_rows<NI>(xo, dO, p.ld_do, q0, last, p.hd, p.vec_do, lane);
      load_rows<NI>(xq, Q, p.ld_q, q0, last, p.hd, p.vec_q, lane);
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      if (!EARLY) load(t);
      f32x4_v s4 = {0.0f, 0.0f, 0.0f, 0.0f}, dp = s4;
      if constexpr (KVL) {
        asm volatile("" ::: "memory");  // (not kept from the half block before)
#pragma unroll
        for (int j = 0; j < NI; ++j) {
          const float4 k4 = kl[64 * j], v4 = vl[64 * j];
          const float ke[4] = {k4.x, k4.y, k4.z, k4.w}, ve[4] = {v4.x, v4.y, v4.z, v4.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            s4 = mfma4(qf[t][j][e], ke[e], s4);
            dp = mfma4(df[t][j][e], ve[e], dp);
          }
        }
      } else {
        s4 = score<NI>(qf[t], kf);
        dp = score<NI>(df[t], vf);
      }
      if (!EARLY) load_stats(t);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float P = expf(s4[r] * p.scale - L[t][r]);
        const bool on = vis(q0 + 16 * t + 4 * g + r);
        pr[t][r] = on ? P : 0.0f;
        ds[t][r] = on ? P * (dp[r] - Dq[t][r]) : 0.0f;
      }
    }
    const bool masked = q0 < k0 + QR - 1 || q0 + KB > hi_min;
    if (!EARLY) load_rows<NI>(xo, dO, p.ld_do, q0, last, p.hd, p.vec_do, lane);
    accumulate_rows<NI>(dv, pr, xo, dO, p.ld_do, q0, last, p.hd, lane, masked, vis);
    if (!EARLY) load_rows<NI>(xq, Q, p.ld_q, q0, last, p.hd, p.vec_q, lane);
    accumulate_rows<NI>(dk, ds, xq, Q, p.ld_q, q0, last, p.hd, lane, masked, vis);
  }
  if (KVL) __syncthreads();  // (the last reads of K and V)
  Merge<NI, dkdv_waves<NI>()>::put(sk, dk, w, lane);
  Merge<NI, dkdv_waves<NI>()>::put(sv, dv, w, lane);
  __syncthreads();
  for (int x = tid; x < QR * p.hd; x += 64 * dkdv_waves<NI>()) {
    const int r = x / p.hd, el = x % p.hd;
    if (!live[r]) continue;
    p.dk[(k0 + r) * p.ld_dk + hk + el] = Merge<NI, dkdv_waves<NI>()>::sum(sk, r, el) * p.scale;
    p.dv[(k0 + r) * p.ld_dv + hk + el] = Merge<NI, dkdv_waves<NI>()>::sum(sv, r, el);
  }
}

WinF params(const lc_window_attn_args &a) {
  WinF p{};
  p.q = static_cast<const float *>(a.q);
  p.k = static_cast<const float *>(a.k);
  p.v = static_cast<const float *>(a.v);
  p.dout = static_cast<const float *>(a.dout);
  p.o = static_cast<float *>(a.o);
  p.dq = static_cast<float *>(a.dq);
  p.dk = static_cast<float *>(a.dk);
  p.dv = static_cast<float *>(a.dv);
  p.lse = a.lse;
  p.D = static_cast<float *>(a.scratch);
  p.off = a.seq_offsets;
  p.ld_q = a.ld_q; p.ld_k = a.ld_k; p.ld_v = a.ld_v; p.ld_o = a.ld_o;
  p.ld_do = a.ld_dout; p.ld_dq = a.ld_dq; p.ld_dk = a.ld_dk; p.ld_dv = a.ld_dv;
  p.T = (int)a.T;
  p.B = a.B;
  p.S = (int)(a.T / a.B);
  p.H = a.H;
  p.Hkv = a.Hkv ? a.Hkv : a.H;
  p.G = p.H / p.Hkv;
  p.hd = a.hd;
  p.window = a.window;
  p.n_sink = a.n_sink;
  p.scale = 1.0f / sqrtf((float)a.hd);
  // (the tensors' pointers are 16-byte aligned)
  auto vec = [&](int64_t ld) { return a.hd % 4 == 0 && ld % 4 == 0; };
  p.vec_q = vec(a.ld_q); p.vec_k = vec(a.ld_k); p.vec_v = vec(a.ld_v); p.vec_o = vec(a.ld_o); p.vec_do = vec(a.ld_dout);
  return p;
}

// calls f with NI (16-feature blocks, a power of two) for head_dim hd <= 128
template <typename F>
void with_blocks(int hd, F f) {
  if (hd <= 16) f(std::integral_constant<int, 1>{});
  else if (hd <= 32) f(std::integral_constant<int, 2>{});
  else if (hd <= 64) f(std::integral_constant<int, 4>{});
  else f(std::integral_constant<int, 8>{});
}

// Launches f(params, grid) with one workgroup per block of 16 rows and head
template <typename F>
lc_status run(const WinF &p, int heads, const char *what, F f) {
  const int64_t n = ((int64_t)p.T + QR - 1) / QR * heads;
  if (n > INT32_MAX) return fail(LC_ERR_UNSUPPORTED, "window attention fp32: 2^31 or more blocks of rows");
  launch_parts((uint32_t)n, [&](uint32_t first, uint32_t count) {
    WinF q = p;
    q.first = (int)first;
    f(q, dim3(count));
  });
  return check_launch(what);
}

}  // namespace

lc_status window_f32_fwd_launch(const lc_window_attn_args &a, hipStream_t s) {
  const WinF p = params(a);
  return run(p, p.H, "window_f32_fwd_kernel", [&](const WinF &q, dim3 grid) {
    with_blocks(p.hd, [&](auto ni) {
      hipLaunchKernelGGL((window_f32_fwd_kernel<decltype(ni)::value>), grid, dim3(NTF), 0, s, q);
    });
  });
}

lc_status window_f32_bwd_launch(const lc_window_attn_args &a, hipStream_t s) {
  const WinF p = params(a);
  LC_TRY(run(p, p.H, "window_f32_dq_kernel", [&](const WinF &q, dim3 grid) {
    with_blocks(p.hd, [&](auto ni) {
      hipLaunchKernelGGL((window_f32_dq_kernel<decltype(ni)::value>), grid, dim3(NTF), 0, s, q);
    });
  }));
  return run(p, p.Hkv, "window_f32_dkdv_kernel", [&](const WinF &q, dim3 grid) {
    with_blocks(p.hd, [&](auto ni) {
      hipLaunchKernelGGL((window_f32_dkdv_kernel<decltype(ni)::value>), grid, dim3(64 * dkdv_waves<decltype(ni)::value>()), 0, s, q);
    });
  });
}

}  // namespace lc
