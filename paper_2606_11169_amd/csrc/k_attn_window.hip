// Sliding-window causal attention with sinks over packed sequences on CDNA4 matrix cores
// (head_dim 64 or 128, fp16 or bf16 q/k/v, fp32 softmax and accumulation), forward and
// backward. The fp32 path is k_attn_window_f32.hip.
//
// The products, the online softmax and the LDS row tiles are those of causal attention
// (k_attn.hip): S^T = K Q^T with one query per lane pair, O^T += V^T P^T with the score
// registers as operand; backward dQ^T += K^T dS^T over keys, dV^T += dO^T P and dK^T += Q^T dS
// over queries, P recomputed from the log-sum-exp. P and dS are rounded once, to the type of
// the product that takes them.
//
// fp16 q, k, v: a gradient's range does not fit fp16, its rows' do. A query's dO is multiplied by
// the power of two that brings its largest value into [2^14, 2^15) (row_scale), and its dS by one that
// keeps the largest seen so far between 2^3 and 2^15, lowered (with the sums formed so far, as a
// softmax's with its maximum) when a block's exceeds that. So dP = dO V^T and dQ = dS K are fp16
// products of the caller's own k and v, undone in fp32, and besides dS's rounding either loses 2^-28
// of the row's largest value, whatever v's size and the number of keys (with dO's scale alone, rows
// of 4100 keys with v near 1e-3 were off by up to 4.9 times what the roundings allow; 32768 tokens,
// 16/4 heads, window 4096 backward 4.55 -> 4.60 ms by it, 8192 x 32 of 64 428 -> 434 us). dV and dK
// sum over queries, so P and dS are bf16 there, and q's rows are rounded to bf16 on their way from
// LDS. (With bf16 copies of q, k and v for every gradient product the gradients were 1.85 times as far
// from 64 bits as their last rounding alone, now 1.45, like those of bf16 inputs.)
//
// Work is laid over the packed rows, not over the sequences: a workgroup owns consecutive
// rows whatever sequences they belong to, each row knows its sequence's start (a search
// over the offsets, 64 per step), and the visible keys of a workgroup's rows are two runs
// of 64-row blocks: the first row's sinks, then everything from the first row's window on
// (sequences that start inside the workgroup's rows lie in the second run as a whole). So a
// grid has no empty workgroups however ragged the batch, and many short sequences share one.
//
// Masks: query i sees key j in [wlo_i, i] or [start_i, start_i + ns_i) (its window, and
// its sinks before the window); seen from key j the queries are [j, hi_j). Each is one
// unsigned comparison per pair, made only in blocks where some pair of the wave is masked.
//
// A masked pair has weight 0, but 0 times an infinite or NaN value is NaN. Where a
// workgroup's result is not finite it makes a second pass with the second products of its
// masked blocks pair by pair, leaving out the masked ones: a value that a result does not
// depend on never reaches it, and finite data pay one look at the result.
//
// Measured, bf16: one sequence of 32768, 16/4 heads of 128, window 4096, 64 sinks: forward 1030 us, dQ
// 1410, dK/dV 2050, 1.02, 1.11 and 1.02 PFLOP/s of the products over visible pairs (2, 3 and 4 of
// them); the matrix cores are 48, 56 and 51% busy, vector units 43, 44 and 35%, LDS 24 to 32%: two
// waves per SIMD alternate between products and exponentials and overlap in part. One of 4096, 32 heads,
// window 1024, 4 sinks: all of it 377 us, 70% of that rate: chains of 18 blocks each with its start,
// three of them a window's edges and the sinks'. 77 tokens in 5 sequences, 8 heads of 64, forward: 7.2,
// offsets, rows and keys loaded one after the other.
#include "attn_tiles.hpp"
#include "attn_window.hpp"

#include <math.h>

namespace lc {
namespace {

constexpr int KB = 64;         // keys (or queries) per inner block
constexpr int MAXSINK = 256;   // sinks whose dK/dV work is split over chunks of queries

// ---------------------------------------------------------------- row tiles
// [64 rows][HD] tiles of 2-byte elements in HD / 8 load runs (one wave instruction each,
// 16 bytes per lane, lanes of a row in address order). HD = 128: run q holds rows f(q) + 16 p,
// p = 0..3, f swapping bit pairs (k_attn.hip). HD = 64: run q holds the rows whose bit 0 is
// bit 2 of q and whose bits 2, 3 are its bits 0, 1; p gives bits 1, 4, 5. In both, 16
// consecutive rows of one 16-byte chunk, and four consecutive rows of 64 bytes, touch every
// bank once, rows 16 on sit 256 bytes on and rows 8 on two runs on, so that fragment
// addresses are a per-lane base plus immediates.
template <int HD> struct Tile {
  static constexpr int NR = HD / 8;
  static constexpr int BYTES = NR * RUNB;
  __device__ __forceinline__ static int lane_row(int lane) {  // row of a run that a lane brings
    return HD == 128 ? 16 * (lane >> 4) : ((lane >> 3 & 1) << 1) + ((lane >> 4) << 4);
  }
  __device__ __forceinline__ static int lane_chunk(int lane) { return lane & (HD / 8 - 1); }
  __device__ __forceinline__ static int run_row(int run) {
    return HD == 128 ? ((run & 3) << 2) | ((run >> 2) & 3) : ((run >> 2) & 1) + ((run & 3) << 2);
  }
  __device__ __forceinline__ static int row_off(int r) {  // byte offset of tile row r
    return HD == 128 ? (((r & 3) << 2) | ((r >> 2) & 3)) * RUNB + (r >> 4) * 256
                     : (((r & 1) << 2) | ((r >> 2) & 3)) * RUNB + ((r >> 1) & 1) * 128 + (r >> 4) * 256;
  }
  // MFMA operand of 32 rows: + (row0 / 16) * 256 + 32 s (columns 16 s + 8 (lane / 32))
  __device__ __forceinline__ static uint32_t rows_lane(int lane) {
    return (uint32_t)(row_off(lane & 31) + (lane >> 5) * 16);
  }
  // MFMA operand of 32 columns in an accumulator's row order (frag_cols_x)
  __device__ __forceinline__ static uint32_t cols_lane(int lane) {
    const int i16 = lane & 15, hf = lane >> 5, b4 = (lane >> 4) & 1;
    return (uint32_t)(row_off(4 * hf + (i16 >> 2)) + (16 * b4 + 4 * (i16 & 3)) * 2);
  }
};

// The lane's number, with head_dim 128 formed anew where it is used: what depends on it need not be
// held across a loop whose registers are full. (The reload of a spilled register also waits for
// every load that is on its way to LDS: dK/dV of 32768 tokens, 16/4 heads, window 4096 2456 us with
// one such reload per block, 2169 without. head_dim 64 has registers to spare: 8192 x 32/8 heads 190
// us, 210 this way.)
template <int HD>
__device__ __forceinline__ int lane_again(int lane) {
  if (HD == 64) return lane;
  uint32_t zero = 0;
  asm volatile("" : "+v"(zero));
  return (int)__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, zero));
}

template <typename VT>
__device__ __forceinline__ VT frag_at(const lds_t *t) {
  return *reinterpret_cast<const __attribute__((address_space(3))) VT *>(t);
}

// A [64][HD] block of rows from row r0 of a matrix on (fewer at its end: rows past the last
// read as zero), one buffer per block, so that offsets stay 32-bit in matrices of any size
template <int HD>
__device__ __forceinline__ i32x4_v block_rsrc(const void *base, int64_t ld, int col0, int r0, int T) {
  const int rows = min(KB, T - r0);
  return make_rsrc(static_cast<const char *>(base) + ((int64_t)r0 * ld + col0) * 2,
                   (uint32_t)(((int64_t)(rows - 1) * ld + HD) * 2));
}

struct WinP {
  const void *q, *k, *v;
  __bf16 *o;
  float *lse;
  const __bf16 *dout;
  __bf16 *dq, *dk, *dv;
  float *D, *nl2;              // [H, T]: rowsum(dO * O) (fp16: scaled) and -lse log2(e)
  float *inv;                  // fp16 inputs: the inverses of dO's row scales, [H, T]
  float *share, *slots;
  const int32_t *off;
  int64_t ld_q, ld_k, ld_v, ld_o, ld_do, ld_dq, ld_dk, ld_dv;
  int T, B, S, H, Hkv, G, window, n_sink;
  int gh, nq;                  // forward, dQ: heads per workgroup, blocks of query rows
  int krows, GP, parts, period;       // dK/dV: keys, query heads per workgroup, blocks of a window (see the walk; 0: none)
  int chunk, chunks;
  int nmain, nsplit, nkb;      // dK/dV workgroups; blocks of krows keys that hold a sequence's sinks
  int first;                   // forward, dQ, dK/dV: the launch's first workgroup
  float scale;
};

// Workgroups are handed to the 8 XCDs in turn; each XCD gets a consecutive run of the n
// tasks (neighbouring row blocks of the same heads read the same keys: one L2 holds them).
// -1: no task.
__device__ __forceinline__ int xcd_task(int i, int n) {
  const int per = (n + 7) >> 3, t = (i & 7) * per + (i >> 3);
  return (i >> 3) < per && t < n ? t : -1;
}

__device__ __forceinline__ int wave_min32(int x) {  // over lanes alike in both halves
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x = min(x, __shfl_xor(x, o, 64));
  return __builtin_amdgcn_readfirstlane(x);
}
__device__ __forceinline__ int wave_max32(int x) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x = max(x, __shfl_xor(x, o, 64));
  return __builtin_amdgcn_readfirstlane(x);
}

// whether some accumulator is infinite or NaN
template <int NI>
__device__ __forceinline__ bool not_finite(const f32x16_v (&a)[NI]) {
  float t = 0.0f;
#pragma unroll
  for (int i = 0; i < NI; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) t = __builtin_fmaf(a[i][r], 0.0f, t);
  return t != t;
}

// acc[column e of the tile][lane] += w[row][lane] * tile[row][e] over 32 NJ rows from row0 on
// that vis(row - row0) lets the lane see, pair by pair. w: the score registers (rows in
// accumulator order), rounded to E as the product rounds them; TE: the tile's type.
template <typename E, typename TE, int HD, int NJ, typename F>
__device__ __forceinline__ void add_pairs(f32x16_v (&acc)[HD / 32], const f32x16_v (&w)[NJ], const lds_t *tile,
                                          int row0, int hf, F vis) {
#pragma unroll 1
  for (int n = 0; n < 32 * NJ; ++n) {
    const int reg = (n & 3) + 4 * ((n >> 3) & 3), j = n >> 5;
    float mine = 0.0f;
#pragma unroll
    for (int u = 0; u < NJ; ++u)
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (u == j && e == reg) mine = w[u][e];
    const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(mine), __float_as_uint(mine), false, false);
    const float wv = (float)(E)__uint_as_float((n >> 2) & 1 ? both[1] : both[0]);
    const bool on = vis(n);
    const lds_t *row = tile + Tile<HD>::row_off(row0 + n) + 8 * hf;
#pragma unroll
    for (int i = 0; i < HD / 32; ++i)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        typedef __attribute__((ext_vector_type(4))) TE e4;
        const e4 x = frag_at<e4>(row + (32 * i + 8 * g) * 2);
#pragma unroll
        for (int u = 0; u < 4; ++u)
          acc[i][4 * g + u] = on ? acc[i][4 * g + u] + wv * (float)x[u] : acc[i][4 * g + u];
      }
  }
}

// ---------------------------------------------------------------- query blocks
// A workgroup's (group's) QW waves of 32 queries: gh heads of one key/value head x 32 QW / gh rows
// (wave w: head w % gh, rows 32 (w / gh) ..). What its rows see:
struct Rows {
  int row, start, wlo, nwin, ns;  // this lane's query (nwin = 0: of no sequence)
  int wmin, wmax, smin, smax, rmax, r0; // this wave's: window starts, sequence starts, last row, first row
  int sb0, nsb, wb0, nit;         // the workgroup's blocks: sink blocks sb0 .., then wb0 ..
  __device__ __forceinline__ int block(int it) const { return it < nsb ? sb0 + it : wb0 + it - nsb; }
  __device__ __forceinline__ bool active() const { return rmax >= 0; }
  // whether the wave sees some key of the block at k0, whether one of them may be a sink before a
  // window, and whether every row sees all of it
  __device__ __forceinline__ bool sinks(int k0, int n_sink) const { return k0 + KB > smin && k0 - smax < n_sink; }
  __device__ __forceinline__ bool any(int k0, int n_sink) const {
    return active() && k0 <= rmax && (k0 + KB > wmin || sinks(k0, n_sink));
  }
  __device__ __forceinline__ bool all(int k0) const { return k0 >= wmax && k0 + KB - 1 <= r0; }
  __device__ __forceinline__ bool sees(int key) const {
    return (uint32_t)(key - wlo) < (uint32_t)nwin || (uint32_t)(key - start) < (uint32_t)ns;
  }
};

// false: no row of the workgroup belongs to a sequence
template <int QW>
__device__ __forceinline__ bool rows_of(const WinP &p, int qb, int w, int lane, Rows &R) {
  const int qrows = 32 * QW / p.gh;
  const Sequences sq(p.off, p.S, p.T, p.B, lane);
  const int g0 = qb * qrows, r0 = max(g0, sq.first), r1 = min(g0 + qrows, sq.last) - 1;
  int b0, s0, e0;
  if (r0 > r1 || !sq.of_wave(r0, lane, b0, s0, e0)) return false;
  const int W = p.window;
  R.wb0 = max(s0, r0 - W + 1) >> 6;
  const int lr = min(r1, e0 - 1), cnt = min(p.n_sink, max(s0, lr - W + 1) - s0);
  R.sb0 = s0 >> 6;
  R.nsb = cnt > 0 ? max(0, min((s0 + cnt - 1) >> 6, R.wb0 - 1) - R.sb0 + 1) : 0;
  R.nit = max(0, R.nsb + (r1 >> 6) - R.wb0 + 1);
  R.r0 = g0 + 32 * (w / p.gh);
  R.row = R.r0 + (lane & 31);
  bool ok = R.row >= r0 && R.row <= r1;
  R.start = s0;
  if (r1 >= e0) {  // (more than one sequence)
    int end;
    ok = sq.of_lane(R.row, b0, R.start, end) && ok;
  }
  R.wlo = max(R.start, R.row - W + 1);
  R.nwin = ok ? max(0, R.row - R.wlo + 1) : 0;
  R.ns = ok ? min(p.n_sink, R.wlo - R.start) : 0;
  constexpr int NONE = 0x7FFFFFFF;
  R.wmin = wave_min32(ok ? R.wlo : NONE);
  R.wmax = wave_max32(ok ? R.wlo : NONE);
  R.smin = wave_min32(ok ? R.start : NONE);
  R.smax = wave_max32(ok ? R.start : -1);
  R.rmax = wave_max32(ok ? R.row : -1);
  return true;
}

// The workgroup's block of rows and first head, neighbouring blocks of a head next to each other, the last
// ones (under a window longer than the sequences the heaviest) first
__device__ __forceinline__ bool place(const WinP &p, int w, int &qb, int &h) {
  const int t = xcd_task(p.first + (int)blockIdx.x, p.nq * (p.H / p.gh));
  if (t < 0) return false;
  qb = p.nq - 1 - t % p.nq;
  h = t / p.nq * p.gh + w % p.gh;
  return true;
}

// 8 elements of a query row per 16 columns: the product's B operand
template <typename QV, int HD, typename E>
__device__ __forceinline__ void load_row(QV (&f)[HD / 16], const E *base, int64_t ld, int row, int T, int hf) {
  const E *at = base + (int64_t)min(row, T - 1) * ld + hf * 8;
#pragma unroll
  for (int es = 0; es < HD / 16; ++es) f[es] = *reinterpret_cast<const QV *>(at + es * 16);
}

// lane holds acc^T[e][row] for its own row; store that row
template <int HD>
__device__ __forceinline__ void store_bf16(__bf16 *row, const f32x16_v (&acc)[HD / 32], float mul, int hf) {
#pragma unroll
  for (int i = 0; i < HD / 32; ++i)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      bf16x4_v wv = {(__bf16)(acc[i][4 * g] * mul), (__bf16)(acc[i][4 * g + 1] * mul),
                     (__bf16)(acc[i][4 * g + 2] * mul), (__bf16)(acc[i][4 * g + 3] * mul)};
      *reinterpret_cast<bf16x4_v *>(row + i * 32 + 8 * g + 4 * hf) = wv;
    }
}
template <int HD>
__device__ __forceinline__ void store_f32(float *row, const f32x16_v (&acc)[HD / 32], int hf) {
#pragma unroll
  for (int i = 0; i < HD / 32; ++i)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      *reinterpret_cast<float4 *>(row + i * 32 + 8 * g + 4 * hf) =
          make_float4(acc[i][4 * g], acc[i][4 * g + 1], acc[i][4 * g + 2], acc[i][4 * g + 3]);
}

// ---------------------------------------------------------------- forward
// KG groups of QW waves own the same 32 QW queries (or 32 QW / gh of gh heads) and take the key blocks in
// turn, each with a ring of its own; their sums are joined at the end in group order, scaled to the
// common maximum. See row_shape for which.
template <int HD, int KG> constexpr int ring_stages() { return KG * 4 * Tile<HD>::BYTES <= 140 * 1024 ? 2 : 1; }

// A group's loads of K and V blocks: QW waves bring 2 NR / QW runs each
template <int HD, int QW>
__device__ __forceinline__ void load_kv(const WinP &p, int kvh, int kb, lds_t *st, int qw, int lane) {
  typedef Tile<HD> TL;
  constexpr int RPW = 2 * TL::NR / QW;
#pragma unroll
  for (int half = 0; half < (QW == 1 ? 2 : 1); ++half) {
    const int first = QW == 1 ? half * TL::NR : RPW * qw;
    const bool isK = QW == 1 ? half == 0 : qw < QW / 2;
    const int64_t ld = isK ? p.ld_k : p.ld_v;
    const uint32_t vo = (uint32_t)((TL::lane_row(lane) * ld + 8 * TL::lane_chunk(lane)) * 2);
    const uint32_t rowb = (uint32_t)(ld * 2);
    const i32x4_v rs = block_rsrc<HD>(isK ? p.k : p.v, ld, kvh * HD, kb * KB, p.T);
#pragma unroll
    for (int t = 0; t < (QW == 1 ? TL::NR : RPW); ++t)
      dma16(rs, st + (first + t) * RUNB, vo + rowb * (uint32_t)TL::run_row((first + t) % TL::NR));
  }
}

template <typename QE, int HD, int QW, int KG>
__global__ __launch_bounds__(64 * QW * KG, 2) void window_fwd_kernel(WinP p) {
  typedef typename V8<QE>::type QV;
  typedef Tile<HD> TL;
  constexpr int NES = HD / 16, NI = HD / 32, ST = ring_stages<HD, KG>();
  __shared__ __align__(16) char smem[KG * ST * 2 * TL::BYTES];  // per group, stage s: K tile | V tile
  const int tid = threadIdx.x, lane = tid & 63, hf = lane >> 5;
  const int w8 = __builtin_amdgcn_readfirstlane(tid >> 6), w = w8 % QW, kg = w8 / QW;
  lds_t *const L = LDS_AS(char, smem) + kg * ST * 2 * TL::BYTES;
  int qb, h;
  if (!place(p, w, qb, h)) return;
  Rows R;
  if (!rows_of<QW>(p, qb, w, lane, R)) return;
  const int kvh = h / p.G;
  const float sc = p.scale * LOG2E;
  auto load = [&](int it, lds_t *st) { load_kv<HD, QW>(p, kvh, R.block(it), st, w, lane); };
  auto next_stage = [&](int it) {  // after the block of step `it`
    if (ST == 1) {
      __syncthreads();
      if (it + KG < R.nit) load(it + KG, L);
    }
    wait_vm0();
    __syncthreads();
  };
  f32x16_v o[NI];
  float m, l;
  auto pass = [&](auto pairs_) {
    constexpr bool pairs = decltype(pairs_)::value;
    QV qf[NES];
    load_row<QV, HD>(qf, static_cast<const QE *>(p.q) + (int64_t)h * HD, p.ld_q, R.row, p.T, hf);
#pragma unroll
    for (int i = 0; i < NI; ++i) o[i] = zero16();
    m = -INFINITY;
    l = 0.0f;
    if (kg < R.nit) load(kg, L);
    wait_vm0();
    __syncthreads();
    for (int it = kg, i0 = 0; i0 < R.nit; it += KG, i0 += KG) {  // (as many steps in every group)
      const lds_t *cur = L + (ST == 2 ? (i0 / KG & 1) * 2 * TL::BYTES : 0);
      if (ST == 2 && it + KG < R.nit) load(it + KG, L + ((i0 / KG + 1) & 1) * 2 * TL::BYTES);
      const int k0 = R.block(it) * KB;
      if (it < R.nit && R.any(k0, p.n_sink)) {
        f32x16_v s[2] = {zero16(), zero16()};
        // K fragments are read one k-step ahead of the products that use them
        const lds_t *krow = cur + TL::rows_lane(lane);
        QV kf[2][2];
        kf[0][0] = frag_at<QV>(krow);
        kf[0][1] = frag_at<QV>(krow + 512);
#pragma unroll
        for (int es = 0; es < NES; ++es) {
          if (es + 1 < NES) {
            kf[(es + 1) & 1][0] = frag_at<QV>(krow + 32 * (es + 1));
            kf[(es + 1) & 1][1] = frag_at<QV>(krow + 512 + 32 * (es + 1));
          }
          __builtin_amdgcn_sched_barrier(0);  // (keeps the reads ahead of the products)
          s[0] = mfma(kf[es & 1][0], qf[es], s[0]);
          s[1] = mfma(kf[es & 1][1], qf[es], s[1]);
          __builtin_amdgcn_sched_barrier(0);
        }
        const bool masked = !R.all(k0);
        if (masked) {
          const int kw = k0 - R.wlo + 4 * hf, kst = k0 - R.start + 4 * hf;
          if (R.sinks(k0, p.n_sink)) {
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
              for (int r = 0; r < 16; ++r) {
                const int c = j * 32 + out_row(r, 0);
                if (!((uint32_t)(kw + c) < (uint32_t)R.nwin || (uint32_t)(kst + c) < (uint32_t)R.ns))
                  s[j][r] = -INFINITY;
              }
          } else {
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
              for (int r = 0; r < 16; ++r)
                if (!((uint32_t)(kw + j * 32 + out_row(r, 0)) < (uint32_t)R.nwin)) s[j][r] = -INFINITY;
          }
        }
        float mx0 = -INFINITY, mx1 = -INFINITY;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          mx0 = fmaxf(mx0, s[0][r]);
          mx1 = fmaxf(mx1, s[1][r]);
        }
        const float mx = max_with_partner(fmaxf(mx0, mx1)) * sc;
        // The reference maximum m only moves when a score exceeds it by more than 8
        // (base-2 exponent units): weights stay <= 2^8, and most blocks skip the rescale.
        if (__any(mx > m + 8.0f)) {
          const float mn = fmaxf(m, mx);
          const float alpha = mn > m ? ex2(m - mn) : 1.0f;
#pragma unroll
          for (int i = 0; i < NI; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[i][r] *= alpha;
          l *= alpha;
          m = mn;
        }
        const float mu = m == -INFINITY ? 0.0f : m;  // (no key seen yet: weights of 0)
        float ls[4] = {0.0f, 0.0f, 0.0f, 0.0f};      // four independent chains
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const float pv = ex2(__builtin_fmaf(s[j][r], sc, -mu));
            s[j][r] = pv;
            ls[2 * j + (r & 1)] += pv;
          }
        l += (ls[0] + ls[1]) + (ls[2] + ls[3]);
        if (masked && pairs) {
          add_pairs<QE, QE, HD, 2>(o, s, cur + TL::BYTES, 0, hf, [&](int n) { return R.sees(k0 + n); });
        } else {
          // V^T fragments of step n (keys 16 n ..) read while step n - 1 multiplies
          const uint32_t av = (uint32_t)(uintptr_t)(cur + TL::BYTES) + TL::cols_lane(lane);
          QV vfr[2][NI];
#pragma unroll
          for (int i = 0; i < NI; ++i) vfr[0][i] = frag_cols_x<QV>(av, i, 0);
#pragma unroll
          for (int n = 0; n < 4; ++n) {
            if (n + 1 < 4) {
#pragma unroll
              for (int i = 0; i < NI; ++i) vfr[(n + 1) & 1][i] = frag_cols_x<QV>(av, i, 16 * (n + 1));
            }
            const QV pf = pack8<QE>(s[n >> 1], 8 * (n & 1));
            __builtin_amdgcn_sched_barrier(0);  // (keeps the reads ahead of the products)
#pragma unroll
            for (int i = 0; i < NI; ++i) o[i] = mfma(vfr[n & 1][i], pf, o[i]);
            __builtin_amdgcn_sched_barrier(0);
          }
        }
      }
      next_stage(it);
    }
  };
  pass(std::false_type{});
  if (__syncthreads_or(not_finite(o))) pass(std::true_type{});
  if constexpr (KG > 1) {
    // (a group that saw no key of a row has m = -inf: weight 0)
    typedef __attribute__((address_space(3))) float lds_f;
    constexpr int N = HD / 2 + 2;
    lds_f *const red = reinterpret_cast<lds_f *>(LDS_AS(char, smem)) + w * (N * 64) + lane;
    constexpr int STEP = QW * N * 64;  // to the next group's
    if (kg > 0) {
      lds_f *const to = red + (kg - 1) * STEP;
#pragma unroll
      for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) to[(i * 16 + r) * 64] = o[i][r];
      to[(N - 2) * 64] = m;
      to[(N - 1) * 64] = l;
    }
    __syncthreads();
    if (kg > 0) return;
#pragma unroll
    for (int x = 0; x < KG - 1; ++x) {
      const lds_f *const from = red + x * STEP;
      const float m1 = from[(N - 2) * 64], mt = fmaxf(m, m1), mu = mt == -INFINITY ? 0.0f : mt;
      const float a0 = ex2(m - mu), a1 = ex2(m1 - mu);
#pragma unroll
      for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[i][r] = o[i][r] * a0 + from[(i * 16 + r) * 64] * a1;
      l = l * a0 + from[(N - 1) * 64] * a1;
      m = mt;
    }
  }
  if (R.nwin == 0) return;
  const float lt = sum_with_partner(l);
  store_bf16<HD>(p.o + (int64_t)R.row * p.ld_o + (int64_t)h * HD, o, 1.0f / lt, hf);
  if (hf == 0) p.lse[(int64_t)h * p.T + R.row] = (m + log2f(lt)) * LN2;
}

// ---------------------------------------------------------------- backward
// the power of two that brings a row's largest absolute value x into [2^14, 2^15), the top of fp16's
// range but one step (1 for a row of zeros, at most 2^112)
__device__ __forceinline__ float row_scale(float x) {
  const int e = (int)(__float_as_uint(x) >> 23);
  return x > 0.0f ? __uint_as_float((uint32_t)(268 - min(max(e, 29), 253)) << 23) : 1.0f;
}

// dQ, and what dK/dV needs of every query: D, -lse log2(e) and, for fp16 inputs, the inverse of its dO
// row's scale. LDS stage = K | V. QW, KG as in the forward.
//
// D of a row is taken from its o, which is rounded to bf16. With the exact D a row's dS sum to zero,
// so their sum is what D was off by, and dK's D gets it added (windows of 8: dk 1.62 times as far from
// 64 bits as its last rounding alone, now 1.41, all three gradients 1.53, now 1.47; sequences of 8
// tokens, fp16, 1.60 and 1.48; 8100 tokens, 32/8 heads 465 -> 470 us). dQ's own sums have used the other
// one, which would take another product to put right.
template <typename QE, int HD, int QW, int KG>
__global__ __launch_bounds__(64 * QW * KG, 2) void window_dq_kernel(WinP p) {
  typedef typename V8<QE>::type QV;
  typedef Tile<HD> TL;
  constexpr bool F16 = !std::is_same<QE, __bf16>::value;
  constexpr int NES = HD / 16, NI = HD / 32, ST = ring_stages<HD, KG>();
  __shared__ __align__(16) char smem[KG * ST * 2 * TL::BYTES];
  const int tid = threadIdx.x, lane = tid & 63, hf = lane >> 5;
  const int w8 = __builtin_amdgcn_readfirstlane(tid >> 6), w = w8 % QW, kg = w8 / QW;
  lds_t *const L = LDS_AS(char, smem) + kg * ST * 2 * TL::BYTES;
  int qb, h;
  if (!place(p, w, qb, h)) return;
  Rows R;
  if (!rows_of<QW>(p, qb, w, lane, R)) return;
  const int kvh = h / p.G;
  const float sc = p.scale * LOG2E;
  const bool ok = R.nwin > 0;
  auto load = [&](int it, lds_t *st) { load_kv<HD, QW>(p, kvh, R.block(it), st, w, lane); };
  auto next_stage = [&](int it) {  // after the block of step `it`
    if (ST == 1) {
      __syncthreads();
      if (it + KG < R.nit) load(it + KG, L);
    }
    wait_vm0();
    __syncthreads();
  };
  const int64_t si = (int64_t)h * p.T + min(R.row, p.T - 1);
  const float lse2 = ok ? p.lse[si] * LOG2E : INFINITY;  // (a row of no sequence: weights of 0)
  float Dq = 0.0f, scale = 1.0f;  // (D and dP in units of 1 / scale)
  int up = F16 ? 60 : 0;          // (dS in units of 2^-up / scale)
  float off[2] = {0.0f, 0.0f};    // the sums of the row's dS
  f32x16_v acc[NI];
  auto pass = [&](auto pairs_) {
    constexpr bool pairs = decltype(pairs_)::value;
    if (kg < R.nit) load(kg, L);
    QV qf[NES], df[NES];
    load_row<QV, HD>(qf, static_cast<const QE *>(p.q) + (int64_t)h * HD, p.ld_q, R.row, p.T, hf);
    bf16x8_v d16[NES];
    load_row<bf16x8_v, HD>(d16, p.dout + (int64_t)h * HD, p.ld_do, R.row, p.T, hf);
    if constexpr (!pairs) {
      // D of this query (its O row read while the first block streams in)
      bf16x8_v of[NES];
      load_row<bf16x8_v, HD>(of, static_cast<const __bf16 *>(p.o) + (int64_t)h * HD, p.ld_o, R.row, p.T, hf);
      float mx = 0.0f;
#pragma unroll
      for (int es = 0; es < NES; ++es)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          Dq += (float)d16[es][e] * (float)of[es][e];
          if (F16) mx = fmaxf(mx, fabsf((float)d16[es][e]));
        }
      Dq = sum_with_partner(Dq);
      if constexpr (F16) scale = row_scale(max_with_partner(mx));
    }
    if constexpr (F16) {
#pragma unroll
      for (int es = 0; es < NES; ++es)
#pragma unroll
        for (int e = 0; e < 8; ++e) df[es][e] = (QE)((float)d16[es][e] * scale);
      if constexpr (!pairs) Dq *= scale;
    } else {
#pragma unroll
      for (int es = 0; es < NES; ++es) df[es] = __builtin_bit_cast(QV, d16[es]);
    }
    if (!pairs && ok && hf == 0 && kg == 0) {
      p.nl2[si] = -lse2;
      if (F16) p.inv[si] = 1.0f / scale;
    }
#pragma unroll
    for (int i = 0; i < NI; ++i) acc[i] = zero16();
    wait_vm0();
    __syncthreads();
    for (int it = kg, i0 = 0; i0 < R.nit; it += KG, i0 += KG) {  // (as many steps in every group)
      const lds_t *cur = L + (ST == 2 ? (i0 / KG & 1) * 2 * TL::BYTES : 0);
      if (ST == 2 && it + KG < R.nit) load(it + KG, L + ((i0 / KG + 1) & 1) * 2 * TL::BYTES);
      const int k0 = R.block(it) * KB;
      if (it < R.nit && R.any(k0, p.n_sink)) {
        f32x16_v s[2] = {zero16(), zero16()}, dp[2] = {zero16(), zero16()};
        // K fragments are read one k-step ahead of their products, V fragments
        // two products ahead of theirs
        const lds_t *krow = cur + TL::rows_lane(lane), *vrow = krow + TL::BYTES;
        QV kf[2][2];
        kf[0][0] = frag_at<QV>(krow);
        kf[0][1] = frag_at<QV>(krow + 512);
#pragma unroll
        for (int es = 0; es < NES; ++es) {
          QV vf[2];
          vf[0] = frag_at<QV>(vrow + 32 * es);
          vf[1] = frag_at<QV>(vrow + 512 + 32 * es);
          __builtin_amdgcn_sched_barrier(0);
          s[0] = mfma(kf[es & 1][0], qf[es], s[0]);
          s[1] = mfma(kf[es & 1][1], qf[es], s[1]);
          if (es + 1 < NES) {
            kf[(es + 1) & 1][0] = frag_at<QV>(krow + 32 * (es + 1));
            kf[(es + 1) & 1][1] = frag_at<QV>(krow + 512 + 32 * (es + 1));
          }
          __builtin_amdgcn_sched_barrier(0);
          dp[0] = mfma(vf[0], df[es], dp[0]);
          dp[1] = mfma(vf[1], df[es], dp[1]);
          __builtin_amdgcn_sched_barrier(0);
        }
        const bool masked = !R.all(k0);
        const float nl = F16 ? (float)up - lse2 : -lse2;
        if (masked) {
#pragma unroll
          for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
              const float pv = ex2(__builtin_fmaf(s[j][r], sc, nl));
              dp[j][r] = R.sees(k0 + j * 32 + out_row(r, hf)) ? pv * (dp[j][r] - Dq) : 0.0f;
              if (!pairs) off[j] += dp[j][r];
            }
        } else {
#pragma unroll
          for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
              const float pv = ex2(__builtin_fmaf(s[j][r], sc, nl));
              dp[j][r] = pv * (dp[j][r] - Dq);
              if (!pairs) off[j] += dp[j][r];
            }
        }
        if constexpr (F16 && !pairs) {
          float mx = 0.0f;
#pragma unroll
          for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) mx = fmaxf(mx, fabsf(dp[j][r]));
          mx = max_with_partner(mx);
          if (__any(mx > 0x1p15f)) {
            const int down = mx > 0x1p15f ? min((int)(__float_as_uint(mx) >> 23) - 130, up + 100) : 0;
            const float by = __uint_as_float((uint32_t)(127 - down) << 23);
            up -= down;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              off[j] *= by;
#pragma unroll
              for (int r = 0; r < 16; ++r) dp[j][r] *= by;
            }
#pragma unroll
            for (int i = 0; i < NI; ++i)
#pragma unroll
              for (int r = 0; r < 16; ++r) acc[i][r] *= by;
          }
        }
        // K^T fragments: transposing reads of the K rows in dS's key order
        if (masked && pairs) {
          add_pairs<QE, QE, HD, 2>(acc, dp, cur, 0, hf, [&](int n) { return R.sees(k0 + n); });
        } else {
          const uint32_t ak = (uint32_t)(uintptr_t)cur + TL::cols_lane(lane_again<HD>(lane));
#pragma unroll
          for (int n = 0; n < 4; ++n) {
            const QV sf = pack8<QE>(dp[n >> 1], 8 * (n & 1));
#pragma unroll
            for (int i = 0; i < NI; ++i) acc[i] = mfma(frag_cols_x<QV>(ak, i, 16 * n), sf, acc[i]);
          }
        }
      }
      next_stage(it);
    }
  };
  pass(std::false_type{});
  float Dk = sum_with_partner(off[0] + off[1]);
  if (__syncthreads_or(not_finite(acc))) pass(std::true_type{});
  if constexpr (F16) {
    const float by = __uint_as_float((uint32_t)(127 - up) << 23);
    Dk *= by;
#pragma unroll
    for (int i = 0; i < NI; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][r] *= by;
  }
  if (kg == 0) Dk += Dq;
  if constexpr (KG > 1) {
    typedef __attribute__((address_space(3))) float lds_f;
    constexpr int N = HD / 2 + 1;
    lds_f *const red = reinterpret_cast<lds_f *>(LDS_AS(char, smem)) + w * (N * 64) + lane;
    constexpr int STEP = QW * N * 64;  // to the next group's
    if (kg > 0) {
#pragma unroll
      for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) red[(kg - 1) * STEP + (i * 16 + r) * 64] = acc[i][r];
      red[(kg - 1) * STEP + (N - 1) * 64] = Dk;
    }
    __syncthreads();
    if (kg > 0) return;
#pragma unroll
    for (int x = 0; x < KG - 1; ++x) {
#pragma unroll
      for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[i][r] += red[x * STEP + (i * 16 + r) * 64];
      Dk += red[x * STEP + (N - 1) * 64];
    }
  }
  if (ok && hf == 0) p.D[si] = Dk;
  if (ok) store_bf16<HD>(p.dq + (int64_t)R.row * p.ld_dq + (int64_t)h * HD, acc, p.scale / scale, hf);
}

// dK, dV. A workgroup of 2 NP waves owns 32 NP consecutive key rows of a key/value head and
// visits, for GP of the head's query heads, the query blocks that see them. Waves w and
// w + NP own the same 32 keys (K and V fragments in registers) and take the first and second 32
// queries of every 64-query block; at the end wave w + NP hands its sums to wave w, which
// adds them. QG groups of such waves own the same keys and take the (head, query block) units in
// turn, each with a ring of its own (QG = 2: key_rows). LDS stage = Q | dO | -lse log2(e) | D |
// (fp16: the scales' inverses) of one block.
//
// Sinks are seen by their whole sequence, so the workgroup that owns them would visit all
// of its queries, however long, while every other visits a window's. Where a sequence
// leaves the chunk of query rows (p.chunk, at least a window) that it starts in, that workgroup
// stops at limit() and the rest is split by chunk: task (chunk, block of sinks) sums over the
// queries of the sequence that spans the chunk's first row. Such keys' sums go to fp32 slots,
// which window_join_kernel adds in chunk order (at most one sequence spans into, and one out
// of, a chunk, so slots are by chunk).
//
// With few keys (p.parts > 1) several workgroups share a key block's query heads and write
// fp32 shares, which window_sum_kernel adds in head order.
__device__ __forceinline__ int limit(const WinP &p, int s, int kblk) {
  return max((kblk + 1) * p.krows - 1 + p.window, (s / p.chunk + 1) * p.chunk);
}
// a slot of [dk | dv], 2 HD floats: set 0 the owner's sums (by the chunk that the sequence
// starts in), set 1 a chunk's
template <int HD>
__device__ __forceinline__ float *slot(const WinP &p, int set, int c, int kvh, int part, int sink) {
  return p.slots +
         ((((((int64_t)set * p.chunks + c) * p.Hkv + kvh) * p.parts + part) * p.n_sink) + sink) * (2 * HD);
}

// fp16 inputs: 8 values of a dO row times its scale, as fp16. c: the scale as (e - 29) << 7 in both
// halves, e the exponent of the row's largest value in bf16's terms, so that exponents fall by
// e - 29 and the largest value's is 29, 2^14 in fp16. What falls below fp16's normal range (2^-28 of the
// row's largest value) is left as a mantissa of the exponent 0, off by less than that.
__device__ __forceinline__ f16x8_v scaled_row(bf16x8_v x, uint32_t c) {
  typedef __attribute__((ext_vector_type(2))) uint16_t u16x2_v;
  typedef __attribute__((ext_vector_type(4))) uint32_t u32x4_v;
  u32x4_v v = __builtin_bit_cast(u32x4_v, x);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const u16x2_v a = __builtin_elementwise_sub_sat(__builtin_bit_cast(u16x2_v, v[i] & 0x7FFF7FFFu),
                                                    __builtin_bit_cast(u16x2_v, c));
    v[i] = (v[i] & 0x80008000u) | __builtin_bit_cast(uint32_t, a << (uint16_t)3);
  }
  return __builtin_bit_cast(f16x8_v, v);
}

template <typename QE, int HD> constexpr int dkdv_stage() {
  return 2 * Tile<HD>::BYTES + (std::is_same<QE, __bf16>::value ? 512 : 768);
}
template <typename QE, int HD, int NP, int QG> constexpr int dkdv_smem() {
  constexpr int handoff = QG * NP * HD * 64 * 4, stages = QG * 2 * dkdv_stage<QE, HD>();
  return stages > handoff ? stages : handoff;
}

template <typename QE, int HD, int NP, int QG>
__global__ __launch_bounds__(128 * NP * QG, 2) void window_dkdv_kernel(WinP p) {
  typedef typename V8<QE>::type QV;
  typedef Tile<HD> TL;
  constexpr bool F16 = !std::is_same<QE, __bf16>::value;
  constexpr int NES = HD / 16, NI = HD / 32;
  constexpr int KROWS = 32 * NP, RPW = TL::NR / NP;  // keys; tile runs per wave
  constexpr int STAGE = dkdv_stage<QE, HD>();
  __shared__ __align__(256) char smem[dkdv_smem<QE, HD, NP, QG>()];
  __shared__ int keys[2][KROWS];  // lo and cnt (below) of every key
  // fp16 of head_dim 128 has no registers for the first of K's fragments: it is read again for every
  // block (8100 tokens in 9 sequences, 32/8 heads: 377 -> 333 us; see lane_again)
  constexpr bool KL = F16 && HD == 128 && NP == 2;
  __shared__ __align__(16) char first_k[KL ? NP * 1024 : 16];
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hf = lane >> 5;
  const int w8 = __builtin_amdgcn_readfirstlane(tid >> 6), w = w8 % (2 * NP), kg = w8 / (2 * NP);
  lds_t *const L = LDS_AS(char, smem) + kg * 2 * STAGE;
  const int pw = w % NP, hq = w / NP;  // key block of the pair, query half
  const bool splits = p.chunks > 1;

  // the task: keys kblk, queries [qa, qb) of sequence [s, e) (the one past the block's last key)
  const Sequences sq(p.off, p.S, p.T, p.B, lane);
  int kblk, kvh, part, c = -1, b, s, e, qa, qb;
  {
    int i = p.first + (int)blockIdx.x;
    const int pad = (p.nsplit + 7) & ~7;  // the long tasks first
    if (i < pad) {
      if (i >= p.nsplit) return;
      const int kbi = i % p.nkb;
      i /= p.nkb;
      part = i % p.parts;
      i /= p.parts;
      kvh = i % p.Hkv;
      c = 1 + i / p.Hkv;
      const int r = c * p.chunk;
      if (!sq.of_wave(r, lane, b, s, e) || s >= r) return;
      kblk = s / KROWS + kbi;
      if (kblk * KROWS >= min(s + p.n_sink, e)) return;
      qa = max(r, limit(p, s, kblk));
      qb = min(e, r + p.chunk);
      if (qa >= qb) return;
    } else {
      const int t = xcd_task(i - pad, p.nmain);
      if (t < 0) return;
      const int nb = (p.T + KROWS - 1) / KROWS;
      kblk = t % nb;
      kvh = t / nb % p.Hkv;
      part = t / nb / p.Hkv;
      const int k0 = kblk * KROWS, r1 = min(k0 + KROWS, sq.last) - 1;
      if (r1 < max(k0, sq.first) || !sq.of_wave(r1, lane, b, s, e)) return;
      qa = k0;
      qb = p.window < e - r1 ? r1 + p.window : e;
      if (p.n_sink > 0 && k0 - s < p.n_sink) qb = splits ? min(e, limit(p, s, kblk)) : e;
    }
  }
  // this lane's key: the queries [lo, lo + cnt) see it
  const int key = kblk * KROWS + pw * 32 + l32;
  int lo = key, cnt = 0, ks = s, ke = e;
  bool later = false;  // its sums are joined from slots
  if (c >= 0) {
    if (key >= s && key - s < p.n_sink && key < e) {
      lo = qa;
      cnt = qb - qa;
    }
  } else {
    bool ok = key < e;
    if (s > kblk * KROWS) ok = sq.of_lane(key, 0, ks, ke);  // (more than one sequence)
    if (ok) {
      const bool sink = key - ks < p.n_sink;
      int hi = sink || p.window >= ke - key ? ke : key + p.window;
      if (splits) {
        const int lim = limit(p, s, kblk);
        later = sink && key >= s && key - s < p.n_sink && e > lim;
        hi = min(hi, lim);
      }
      cnt = max(0, hi - key);
    }
  }
  constexpr int NONE = 0x7FFFFFFF;
  const int lo_min = wave_min32(cnt ? lo : NONE), lo_max = wave_max32(cnt ? lo : NONE);
  const int hi_max = wave_max32(cnt ? lo + cnt : -1), hi_min = wave_min32(lo + cnt);
  const int64_t krow = min(key, p.T - 1);
  if (w8 == pw && hf == 0) {
    keys[0][pw * 32 + l32] = lo;
    keys[1][pw * 32 + l32] = cnt;
  }
  const float sc = p.scale * LOG2E;

  // half of the waves bring Q, half dO, RPW runs each; the last one also -lse log2(e), D and the
  // inverses (64 floats each)
  const int tl = w / NP, sub = w % NP;
  const void *const src = tl == 0 ? p.q : static_cast<const void *>(p.dout);
  const int64_t ld = tl == 0 ? p.ld_q : p.ld_do;
  const uint32_t rowb = (uint32_t)(ld * 2);
  const int h0 = kvh * p.G + part * p.GP;
  auto load = [&](int g, int qbi, lds_t *st) {
    const int ln = lane_again<HD>(lane);
    const uint32_t vo = (uint32_t)TL::lane_row(ln) * rowb + 16 * TL::lane_chunk(ln);
    const i32x4_v rs = block_rsrc<HD>(src, ld, (h0 + g) * HD, qbi * KB, p.T);
#pragma unroll
    for (int t = 0; t < RPW; ++t) {
      const int run = RPW * sub + t;
      dma16(rs, st + tl * TL::BYTES + run * RUNB, vo + rowb * (uint32_t)TL::run_row(run));
    }
    if (w == 2 * NP - 1) {
      const int64_t at = (int64_t)(h0 + g) * p.T + qbi * KB;
      const uint32_t bytes = (uint32_t)min(KB, p.T - qbi * KB) * 4;
      dma4(make_rsrc(p.nl2 + at, bytes), st + 2 * TL::BYTES, ln * 4);
      dma4(make_rsrc(p.D + at, bytes), st + 2 * TL::BYTES + 256, ln * 4);
      if (F16) dma4(make_rsrc(p.inv + at, bytes), st + 2 * TL::BYTES + 512, ln * 4);
    }
  };
  const int qfirst = qa / KB, nqb = max(0, (qb + KB - 1) / KB - qfirst), nit = nqb * p.GP;
  // The walk over the blocks begins at the one that comes first in a clock of a window's blocks:
  // workgroups side by side, whose windows overlap a little further on each, are then at the same
  // block at the same time, so that it comes from the L2 once for all (4096 tokens x 32 heads, window
  // 1024: 201 -> 193 us, fp16 287 -> 272). Long windows, whose workgroups follow one another through
  // them anyway, lose by it (32768 tokens, 16/4 heads, window 4096: 2456 -> 2550 us).
  int turn = p.period > 0 ? (p.period - qfirst % p.period) % p.period : 0;
  if (turn >= nqb) turn = 0;
  f32x16_v dk[NI], dv[NI];
  auto pass = [&](auto pairs_) {
    constexpr bool pairs = decltype(pairs_)::value;
    // head and block of this group's unit; the walk's next one
    int g = 0, qi = turn;
    auto next = [&](int &gn, int &qn) {
      qn = qn + 1 < nqb ? qn + 1 : 0;
      if (qn == turn) ++gn;
    };
    if (kg == 1) next(g, qi);
    if (kg < nit) load(g, qfirst + qi, L);
    QV kf[NES], vf[NES];
#pragma unroll
    for (int es = 0; es < NES; ++es) {
      const int col = kvh * HD + es * 16 + hf * 8;
      kf[es] = *reinterpret_cast<const QV *>(static_cast<const QE *>(p.k) + krow * p.ld_k + col);
      vf[es] = *reinterpret_cast<const QV *>(static_cast<const QE *>(p.v) + krow * p.ld_v + col);
    }
    if (KL && hq == 0) *reinterpret_cast<QV *>(first_k + 1024 * pw + 16 * lane) = kf[0];
#pragma unroll
    for (int i = 0; i < NI; ++i) dk[i] = dv[i] = zero16();
    wait_vm0();
    __syncthreads();
    for (int it = kg, i0 = 0; i0 < nit; it += QG, i0 += QG) {  // (as many steps in every group)
      const lds_t *cur = L + (i0 / QG & 1) * STAGE;
      int gn = g, qn = qi;
#pragma unroll
      for (int u = 0; u < QG; ++u) next(gn, qn);
      if (it + QG < nit) load(gn, qfirst + qn, L + ((i0 / QG + 1) & 1) * STAGE);
      const int q0 = (qfirst + qi) * KB + 32 * hq;  // this wave's 32 queries
      if (it < nit && q0 + 31 >= lo_min && q0 < hi_max) {
        f32x16_v sv = zero16(), dp = zero16();
        // fragment rows of this wave's 32 queries: a per-lane base plus immediates
        const int ln = lane_again<HD>(lane), lh = ln >> 5;
        const lds_t *qrow = cur + TL::rows_lane(ln) + 512 * hq;
        // each fragment is read one product ahead of the product that uses it
        uint32_t rs = 0;  // this fragment row's scale
        if constexpr (F16) {
          // (the inverse of the scale has the exponent e - 14)
          rs = (frag_at<uint32_t>(cur + 2 * TL::BYTES + 512 + 128 * hq + 4 * (ln & 31)) >> 23) - 15;
          rs = rs << 7 | rs << 23;
        }
        auto scaled = [&](bf16x8_v x) -> QV {
          if constexpr (F16) return scaled_row(x, rs);
          else return x;
        };
        QV k0{};
        if (KL) k0 = frag_at<QV>(LDS_AS(char, first_k) + 1024 * pw + 16 * ln);
        QV qv = frag_at<QV>(qrow);
        bf16x8_v da = frag_at<bf16x8_v>(qrow + TL::BYTES);
#pragma unroll
        for (int es = 0; es < NES; ++es) {
          QV qx{};
          bf16x8_v dx{};
          if (es + 1 < NES) qx = frag_at<QV>(qrow + 32 * (es + 1));
          __builtin_amdgcn_sched_barrier(0);
          sv = mfma(qv, KL && es == 0 ? k0 : kf[es], sv);
          if (es + 1 < NES) dx = frag_at<bf16x8_v>(qrow + TL::BYTES + 32 * (es + 1));
          __builtin_amdgcn_sched_barrier(0);
          dp = mfma(scaled(da), vf[es], dp);
          __builtin_amdgcn_sched_barrier(0);
          qv = qx;
          da = dx;
        }
        const bool masked = !(q0 >= lo_max && q0 + 31 < hi_min);
        // four rows at a time: their -lse log2(e) and D are 4 consecutive floats each
        typedef __attribute__((ext_vector_type(4))) float f4_t;
        const lds_t *const st = cur + 2 * TL::BYTES + 128 * hq + 16 * lh;
#pragma unroll
        for (int gq = 0; gq < 4; ++gq) {
          const f4_t lc = frag_at<f4_t>(st + 32 * gq), dc = frag_at<f4_t>(st + 256 + 32 * gq);
          f4_t ic{};
          if (F16) ic = frag_at<f4_t>(st + 512 + 32 * gq);
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const int r = 4 * gq + x;  // out_row(r, hf) = 8 gq + 4 hf + x
            const float pv = ex2(__builtin_fmaf(sv[r], sc, lc[x]));
            sv[r] = pv;
            dp[r] = pv * (F16 ? ic[x] * (dp[r] - dc[x]) : dp[r] - dc[x]);
          }
        }
        if (masked) {
          const int at = pw * 32 + (ln & 31), d = q0 - keys[0][at] + 4 * lh;
          const uint32_t n = keys[1][at];
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (!((uint32_t)(d + out_row(r, 0)) < n)) sv[r] = dp[r] = 0.0f;
        }
        if (masked && pairs) {
          auto vis = [&](int n) { return (uint32_t)(q0 + n - lo) < (uint32_t)cnt; };
          const f32x16_v w1[1] = {sv}, w2[1] = {dp};
          add_pairs<__bf16, __bf16, HD, 1>(dv, w1, cur + TL::BYTES, 32 * hq, hf, vis);
          add_pairs<__bf16, QE, HD, 1>(dk, w2, cur, 32 * hq, hf, vis);
        } else {
          // P and dS rounded to bf16 before the gradient products, so that the
          // fp32 score registers are free while those run
          const bf16x8_v pf[2] = {pack8<__bf16>(sv, 0), pack8<__bf16>(sv, 8)};
          const bf16x8_v sf[2] = {pack8<__bf16>(dp, 0), pack8<__bf16>(dp, 8)};
          __builtin_amdgcn_sched_barrier(0);
          // dO^T and Q^T fragments: transposing reads of the dO and Q rows in P's query order
          const uint32_t aq = (uint32_t)(uintptr_t)cur + TL::cols_lane(lane_again<HD>(lane)) + 512 * hq, ao = aq + TL::BYTES;
          bf16x8_v fo[2];
          uint4 fq[2];
          fo[0] = frag_cols_x<bf16x8_v>(ao, 0, 0);
          fq[0] = frag_cols_x<uint4>(aq, 0, 0);
#pragma unroll
          for (int n = 0; n < 2 * NI; ++n) {
            const int t = n / NI, i = n % NI;
            if (n + 1 < 2 * NI) {
              const int i1 = (n + 1) % NI, k1 = 16 * ((n + 1) / NI);
              fo[(n + 1) & 1] = frag_cols_x<bf16x8_v>(ao, i1, k1);
              fq[(n + 1) & 1] = frag_cols_x<uint4>(aq, i1, k1);
            }
            __builtin_amdgcn_sched_barrier(0);
            dv[i] = mfma(fo[n & 1], pf[t], dv[i]);
            dk[i] = mfma(to_bf16x8<QE>(fq[n & 1]), sf[t], dk[i]);
            __builtin_amdgcn_sched_barrier(0);
          }
        }
      }
      g = gn;
      qi = qn;
      wait_vm0();
      __syncthreads();
    }
  };
  pass(std::false_type{});
  if (__syncthreads_or(not_finite(dk) || not_finite(dv))) pass(std::true_type{});
  // the second group hands its sums to the first, then the upper waves theirs to the lower ones (the
  // stages are free now)
  typedef __attribute__((address_space(3))) float lds_f;
  if constexpr (QG > 1) {
    lds_f *const red = reinterpret_cast<lds_f *>(LDS_AS(char, smem)) + w * (HD * 64) + lane;
    if (kg == 1) {
#pragma unroll
      for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          red[(i * 16 + r) * 64] = dk[i][r];
          red[(HD / 2 + i * 16 + r) * 64] = dv[i][r];
        }
    }
    __syncthreads();
    if (kg == 0) {
#pragma unroll
      for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          dk[i][r] += red[(i * 16 + r) * 64];
          dv[i][r] += red[(HD / 2 + i * 16 + r) * 64];
        }
    }
    __syncthreads();
  }
  lds_f *const red = reinterpret_cast<lds_f *>(LDS_AS(char, smem)) + pw * (HD * 64) + lane;
  if (hq == 1 && kg == 0) {
#pragma unroll
    for (int i = 0; i < NI; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        red[(i * 16 + r) * 64] = dk[i][r];
        red[(HD / 2 + i * 16 + r) * 64] = dv[i][r];
      }
  }
  __syncthreads();
  if (hq == 1 || kg == 1 || cnt == 0) return;
#pragma unroll
  for (int i = 0; i < NI; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      dk[i][r] = (dk[i][r] + red[(i * 16 + r) * 64]) * p.scale;
      dv[i][r] += red[(HD / 2 + i * 16 + r) * 64];
    }
  if (c >= 0 || (later && p.parts == 1)) {
    float *const to = slot<HD>(p, c >= 0, c >= 0 ? c : s / p.chunk, kvh, part, key - s);
    store_f32<HD>(to, dk, hf);
    store_f32<HD>(to + HD, dv, hf);
  } else if (p.parts > 1) {
    const int64_t at = ((int64_t)part * p.T + key) * p.Hkv + kvh, n = (int64_t)p.parts * p.T * p.Hkv;
    store_f32<HD>(p.share + at * HD, dk, hf);
    store_f32<HD>(p.share + (n + at) * HD, dv, hf);
  } else {
    store_bf16<HD>(p.dk + key * p.ld_dk + (int64_t)kvh * HD, dk, 1.0f, hf);
    store_bf16<HD>(p.dv + key * p.ld_dv + (int64_t)kvh * HD, dv, 1.0f, hf);
  }
}

// dk, dv of every key row = the sum of the parts' shares in order, 8 elements per thread
__global__ __launch_bounds__(256) void window_sum_kernel(WinP p, int width) {
  const int cpr = width / 8;
  const int64_t n = (int64_t)p.T * cpr, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const bool isv = i >= n;
  const int64_t at = isv ? i - n : i, row = at / cpr, col = 8 * (at % cpr);
  const Sequences sq(p.off, p.S, p.T, p.B, threadIdx.x & 63);
  if (i >= 2 * n || row < sq.first || row >= sq.last) return;
  const float *src = p.share + (isv ? (int64_t)p.parts * p.T * width : 0) + row * width + col;
  float a[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  for (int t = 0; t < p.parts; ++t, src += (int64_t)p.T * width) {
    const float4 x = *reinterpret_cast<const float4 *>(src), y = *reinterpret_cast<const float4 *>(src + 4);
    a[0] += x.x; a[1] += x.y; a[2] += x.z; a[3] += x.w;
    a[4] += y.x; a[5] += y.y; a[6] += y.z; a[7] += y.w;
  }
  store8_dt(isv ? p.dv + row * p.ld_dv : p.dk + row * p.ld_dk, col, LC_BF16, a);
}

// dk, dv of the sinks whose work was split: workgroup (chunk that the sequence starts in,
// key/value head, sink), one thread per element
template <int HD>
__global__ __launch_bounds__(2 * HD) void window_join_kernel(WinP p) {
  int i = (int)blockIdx.x;
  const int sink = i % p.n_sink;
  i /= p.n_sink;
  const int kvh = i % p.Hkv, c0 = i / p.Hkv, r = (c0 + 1) * p.chunk, el = threadIdx.x;
  int b, s, e;
  const Sequences sq(p.off, p.S, p.T, p.B, threadIdx.x & 63);
  if (!sq.of_wave(r, threadIdx.x & 63, b, s, e) || s >= r || s / p.chunk != c0) return;
  const int key = s + sink;
  const int lim = limit(p, s, key / p.krows);
  if (key >= e || e <= lim) return;
  float sum = 0.0f;
  for (int part = 0; part < p.parts; ++part) {
    if (p.parts > 1) {
      const int64_t at = ((int64_t)part * p.T + key) * p.Hkv + kvh, n = (int64_t)p.parts * p.T * p.Hkv;
      sum += p.share[((el >= HD ? n : 0) + at) * HD + el % HD];
    } else {
      sum += slot<HD>(p, 0, c0, kvh, 0, sink)[el];
    }
    for (int c = c0 + 1; c * p.chunk < e; ++c)
      if (max(c * p.chunk, lim) < min(e, (c + 1) * p.chunk)) sum += slot<HD>(p, 1, c, kvh, part, sink)[el];
  }
  __bf16 *const to = el >= HD ? p.dv + key * p.ld_dv : p.dk + key * p.ld_dk;
  to[(int64_t)kvh * HD + el % HD] = (__bf16)sum;
}

// ---------------------------------------------------------------- host
// Keys per dK/dV workgroup: 64, or 32 and two groups of waves where that leaves a compute unit to
// every two workgroups of 64 (1024 tokens in 4 sequences, 8 heads, window 256: 21 -> 16 us; one
// sequence of 1500, 4 heads, causal: 38 -> 27. With 160 of them, 300 tokens x 32 heads: 16 -> 21)
int key_rows(int64_t T, int H) { return (T + 63) / 64 * H <= 128 ? 32 : 64; }

int kv_of(const lc_window_attn_args &a) { return a.Hkv ? a.Hkv : a.H; }

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
    if (a.hd > 128 || a.hd % 2) return fail(LC_ERR_UNSUPPORTED, "window attention fp32: even head_dim <= 128");
  } else {
    return fail(LC_ERR_INVALID_ARG, "window attention: unknown dtype");
  }
  const int64_t most = (int64_t)1 << 24;  // (64 rows span less than 2^32 bytes)
  const int64_t qw = (int64_t)a.H * a.hd, kw = (int64_t)kv_of(a) * a.hd;
  if (qw > most) return fail(LC_ERR_UNSUPPORTED, "window attention: H * hd larger than 2^24");
  auto ld_bad = [&](int64_t ld, int64_t w) { return ld < w || ld > most || (a.dtype != LC_FP32 && ld % 8); };
  if (ld_bad(a.ld_q, qw) || ld_bad(a.ld_k, kw) || ld_bad(a.ld_v, kw) || ld_bad(a.ld_o, qw) ||
      (bwd && (ld_bad(a.ld_dout, qw) || ld_bad(a.ld_dq, qw) || ld_bad(a.ld_dk, kw) || ld_bad(a.ld_dv, kw))))
    return fail(LC_ERR_INVALID_ARG, "window attention: a leading dimension is smaller than heads * hd, larger "
                "than 2^24 or (16 bits) not a multiple of 8");
  if (a.T == 0) return LC_OK;
  auto bad = [](const void *x) { return !x || !aligned16(x); };
  if (bad(a.q) || bad(a.k) || bad(a.v) || bad(a.o) || bad(a.lse))
    return fail(LC_ERR_INVALID_ARG, "window attention: null or unaligned pointer");
  if (reinterpret_cast<uintptr_t>(a.seq_offsets) & 3)
    return fail(LC_ERR_INVALID_ARG, "window attention: unaligned seq_offsets");
  if (bwd) {
    if (bad(a.dout) || bad(a.dq) || bad(a.dk) || bad(a.dv))
      return fail(LC_ERR_INVALID_ARG, "window attention: null or unaligned gradient pointer");
    const WindowPlan w = window_plan(a.dtype, a.T, a.H, kv_of(a), a.hd, a.window, a.n_sink);
    if (bad(a.scratch) || a.scratch_bytes < (size_t)w.total)
      return fail(LC_ERR_WORKSPACE, "window attention: scratch smaller than "
                  "lc_window_attention_scratch_bytes (or unaligned)");
  }
  return LC_OK;
}

WinP params(const lc_window_attn_args &a, bool bwd) {
  WinP p{};
  p.q = a.q; p.k = a.k; p.v = a.v;
  p.o = static_cast<__bf16 *>(a.o);
  p.lse = a.lse;
  p.dout = static_cast<const __bf16 *>(a.dout);
  p.dq = static_cast<__bf16 *>(a.dq);
  p.dk = static_cast<__bf16 *>(a.dk);
  p.dv = static_cast<__bf16 *>(a.dv);
  p.off = a.seq_offsets;
  p.ld_q = a.ld_q; p.ld_k = a.ld_k; p.ld_v = a.ld_v; p.ld_o = a.ld_o;
  p.ld_do = a.ld_dout; p.ld_dq = a.ld_dq; p.ld_dk = a.ld_dk; p.ld_dv = a.ld_dv;
  p.T = (int)a.T;
  p.B = a.B;
  p.S = (int)(a.T / a.B);
  p.H = a.H;
  p.Hkv = kv_of(a);
  p.G = p.H / p.Hkv;
  p.window = a.window;
  p.n_sink = a.n_sink;
  p.scale = 1.0f / sqrtf((float)a.hd);
  if (!bwd) return p;
  const WindowPlan w = window_plan(a.dtype, a.T, p.H, p.Hkv, a.hd, a.window, a.n_sink);
  char *const sc = static_cast<char *>(a.scratch);
  p.D = reinterpret_cast<float *>(sc + w.D);
  p.nl2 = reinterpret_cast<float *>(sc + w.nl2);
  p.inv = reinterpret_cast<float *>(sc + w.inv);
  p.share = reinterpret_cast<float *>(sc + w.share);
  p.slots = reinterpret_cast<float *>(sc + w.slots);
  p.parts = w.parts;
  p.GP = p.G / w.parts;
  p.chunk = w.chunk;
  p.chunks = w.chunks;
  p.krows = w.krows;
  p.period = p.window <= 2048 ? (p.window + p.krows - 1 + KB - 1) / KB : 0;
  p.nkb = p.chunks > 1 ? (p.n_sink + p.krows - 2) / p.krows + 1 : 0;
  return p;
}

// Forward and dQ: 32 QW rows (of one head) per workgroup and KG groups of waves, by the number of
// workgroups that 128 rows each would make.
// Up to 64: 32 rows and four groups, so that four times as many compute units share the work and a
// chain of blocks is a quarter as long (1024 tokens in 4 sequences, 8 heads, window 256: forward 17.0 ->
// 13.2 us, dQ 21.3 -> 15.4; one sequence of 1500, 4 heads, causal: 41 -> 23 and 51 -> 25). With 96
// workgroups the chip is full (300 tokens, 32 heads: 12.8 -> 18.5).
// Up to 256, one per compute unit, and chains of 8 blocks or more: two groups (3000 tokens, 10 heads,
// window 1000: 33.3 -> 28.6 and 41.2 -> 37.0; with chains of up to 5 blocks 12.8 -> 13.1, 16.1 -> 18.4).
struct Shape { int QW, KG; };
Shape row_shape(const WinP &p) {
  const int64_t n = (p.T + 127ll) / 128 * p.H;
  if (n <= 64) return {1, 4};
  return n <= 256 && p.window >= 512 && p.T / p.B >= 512 ? Shape{4, 2} : Shape{4, 1};
}

// Forward and dQ grids. gh heads of a group (as many of 1, 2, 4 as divide it, at most one per wave) share
// a workgroup's keys, so that it spans fewer rows and with them fewer keys.
lc_status row_grid(WinP &p, int QW, unsigned &grid) {
  p.gh = 1;
  while (2 * p.gh <= QW && p.G % (2 * p.gh) == 0) p.gh *= 2;
  const int qrows = 32 * QW / p.gh;
  p.nq = (p.T + qrows - 1) / qrows;
  const int64_t n = (int64_t)p.nq * (p.H / p.gh);
  if (n > 1 << 30) return fail(LC_ERR_UNSUPPORTED, "window attention: more than 2^30 blocks of rows and heads");
  grid = (unsigned)((n + 7) / 8 * 8);
  return LC_OK;
}

// A launch of `kernel` with n workgroups, in parts
lc_status launch(void (*kernel)(WinP), WinP p, unsigned n, unsigned threads, hipStream_t s, const char *what) {
  launch_parts(n, [&](uint32_t first, uint32_t count) {
    p.first = (int)first;
    hipLaunchKernelGGL(kernel, dim3(count), dim3(threads), 0, s, p);
  });
  return check_launch(what);
}

template <typename QE, int HD>
lc_status fwd(const lc_window_attn_args &a, hipStream_t s) {
  WinP p = params(a, false);
  const Shape sh = row_shape(p);
  unsigned grid = 0;
  LC_TRY(row_grid(p, sh.QW, grid));
  if (sh.QW == 1) return launch(window_fwd_kernel<QE, HD, 1, 4>, p, grid, 256, s, "window_fwd_kernel");
  if (sh.KG == 2) return launch(window_fwd_kernel<QE, HD, 4, 2>, p, grid, 512, s, "window_fwd_kernel");
  return launch(window_fwd_kernel<QE, HD, 4, 1>, p, grid, 256, s, "window_fwd_kernel");
}

template <typename QE, int HD>
lc_status bwd(const lc_window_attn_args &a, hipStream_t s) {
  WinP p = params(a, true);
  const Shape sh = row_shape(p);
  unsigned grid = 0;
  LC_TRY(row_grid(p, sh.QW, grid));
  const int64_t nmain = ((int64_t)p.T + p.krows - 1) / p.krows * p.Hkv * p.parts;
  const int64_t nsplit = (int64_t)(p.chunks - 1) * p.Hkv * p.parts * p.nkb;
  const int64_t n = ((nsplit + 7) / 8 + (nmain + 7) / 8) * 8;
  p.nmain = (int)nmain;
  p.nsplit = (int)nsplit;
  if (n > 1 << 30) return fail(LC_ERR_UNSUPPORTED, "window attention: more than 2^30 blocks of keys and heads");
  const int width = p.Hkv * HD;
  if (sh.QW == 1) LC_TRY(launch(window_dq_kernel<QE, HD, 1, 4>, p, grid, 256, s, "window_dq_kernel"));
  else if (sh.KG == 2) LC_TRY(launch(window_dq_kernel<QE, HD, 4, 2>, p, grid, 512, s, "window_dq_kernel"));
  else LC_TRY(launch(window_dq_kernel<QE, HD, 4, 1>, p, grid, 256, s, "window_dq_kernel"));
  if (p.krows == 32) LC_TRY(launch(window_dkdv_kernel<QE, HD, 1, 2>, p, (unsigned)n, 256, s, "window_dkdv_kernel"));
  else LC_TRY(launch(window_dkdv_kernel<QE, HD, 2, 1>, p, (unsigned)n, 256, s, "window_dkdv_kernel"));
  if (p.parts > 1) {
    // (fewer than 384 blocks of keys and heads: window_plan)
    hipLaunchKernelGGL(window_sum_kernel, dim3(ceil_div(2 * (size_t)p.T * width / 8, 256)), dim3(256), 0, s, p, width);
    LC_TRY(check_launch("window_sum_kernel"));
  }
  if (p.chunks > 1) {
    hipLaunchKernelGGL((window_join_kernel<HD>), dim3((unsigned)((p.chunks - 1) * p.Hkv * p.n_sink)), dim3(2 * HD),
                       0, s, p);
    LC_TRY(check_launch("window_join_kernel"));
  }
  return LC_OK;
}

lc_status forward(const lc_window_attn_args &a, hipStream_t s) {
  LC_TRY(check(a, false));
  if (a.T == 0) return LC_OK;
  if (a.dtype == LC_FP32) return window_f32_fwd_launch(a, s);
  if (a.dtype == LC_FP16) return a.hd == 64 ? fwd<_Float16, 64>(a, s) : fwd<_Float16, 128>(a, s);
  return a.hd == 64 ? fwd<__bf16, 64>(a, s) : fwd<__bf16, 128>(a, s);
}

lc_status backward(const lc_window_attn_args &a, hipStream_t s) {
  LC_TRY(check(a, true));
  if (a.T == 0) return LC_OK;
  if (a.dtype == LC_FP32) return window_f32_bwd_launch(a, s);
  if (a.dtype == LC_FP16) return a.hd == 64 ? bwd<_Float16, 64>(a, s) : bwd<_Float16, 128>(a, s);
  return a.hd == 64 ? bwd<__bf16, 64>(a, s) : bwd<__bf16, 128>(a, s);
}

}  // namespace

WindowPlan window_plan(int dtype, int64_t T, int H, int Hkv, int hd, int window, int n_sink) {
  WindowPlan w{};
  int64_t at = 0;
  auto take = [&](int64_t bytes) {
    const int64_t x = at;
    at += (bytes + 255) / 256 * 256;
    return x;
  };
  w.parts = w.chunks = 1;
  w.D = take(T * H * 4);
  w.nl2 = w.inv = w.share = w.slots = 0;
  if (dtype != LC_FP32) {
    w.nl2 = take(T * H * 4);
    if (dtype == LC_FP16) w.inv = take(T * H * 4);
    const int G = H / Hkv;
    w.krows = key_rows(T, H);
    const int64_t tasks = (T + w.krows - 1) / w.krows * Hkv;
    for (int n = 1; n <= G; ++n)
      if (G % n == 0) {
        w.parts = n;
        if (tasks * n >= 384) break;
      }
    if (w.parts > 1) w.share = take(2 * w.parts * T * Hkv * hd * 4);
    int64_t chunk = 1024;
    while (chunk < (int64_t)window + w.krows) chunk *= 2;
    const int64_t joins = (T + chunk - 1) / chunk * Hkv * n_sink;  // (workgroups of window_join_kernel)
    if (n_sink > 0 && n_sink <= MAXSINK && chunk < T && joins <= 1 << 23) {
      w.chunk = (int)chunk;
      w.chunks = (int)((T + chunk - 1) / chunk);
      w.slots = take(2ll * w.chunks * Hkv * w.parts * n_sink * 2 * hd * 4);
    } else {
      w.chunk = 1 << 30;
    }
  }
  w.total = at;
  return w;
}

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
  if (T <= 0 || T >= (int64_t)1 << 30 || H < 1 || Hkv < 0 || hd < 1 || hd > 128 || window < 1 || n_sink < 0 ||
      (Hkv > 0 && H % Hkv) || (int64_t)H * hd > 1 << 24)
    return 0;
  return (size_t)lc::window_plan(dtype, T, H, Hkv ? Hkv : H, hd, window, n_sink).total;
}

}  // extern "C"
