// 8-bit products of many rows and columns: square tiles through LDS (gfx950).
//
// Tile BT x BT per workgroup of WM x WN waves; a wave owns FM x FN blocks of 16 x 16. A
// stage is one block of 128 k: BT rows of 128 bytes of each operand and a scale per row.
// Two stages lie in LDS; stage st + 2 streams into st's place from st's barrier on.
//
// Operands go from global memory straight into LDS, 1 KiB per wave instruction: run q
// (of NR = BT / 8) holds tile rows q + NR p (p = 0 .. 7), 128 bytes each, and runs sit
// 1056 bytes apart, so a fragment (16 rows; lane l reads bytes 16 (l / 16) .. and 64 + 16
// (l / 16) .. of row l % 16) is two conflict-free ds_read_b128. Which 32 of a row's 128
// values a lane holds does not matter to the sum, as both operands choose alike and a
// block has one scale. Scale bytes come as dwords (buffer_load_ubyte ... lds), placed so
// that a lane's FM (FN) rows of a wave's fragments lie side by side.
//
// A stage is multiplied in four steps, halves of A's fragments by halves of B's: (0, 0),
// (0, 1), (1, 1), (1, 0), in the next stage (0, 1), (0, 0), (1, 0), (1, 1): each step
// changes one half, which is read into the registers that the step before has freed, so
// every fragment is read once per stage and none is held twice. The stage's barrier sits
// in the middle: its own reads are done, the next stage's may begin.
//
// Bound: the matrix cores, under the chip's power. 4096 x 11008 x 4096, bf16 out: 142 us,
// 2.60 PFLOP/s (a loop of these instructions alone reaches 4.4). 2048 of k are 16 stages beside a
// tile's start and end, and the last round of tiles is not full: 8187 rows of eight experts x 2816 x
// 2048 55 us (1023 or 1026 rows each), 57 (100 to 2000), 54 (two with 5102 and 3085, six with none),
// 1.66 to 1.74 PFLOP/s; their weight gradients 59, 57 and 55.
#include "gemm_fp8.hpp"

namespace lc {
namespace {

constexpr int RUN = 1024 + 32;
constexpr uint32_t OOB = 0x80000000u;

// 1 byte per lane, zero-extended to 4, into lds + 4 * lane
__device__ __forceinline__ void dma1(i32x4_v rs, lds_t *lds, uint32_t off) {
  const uint32_t m0 = __builtin_amdgcn_readfirstlane((uint32_t) reinterpret_cast<uintptr_t>(lds));
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_ubyte %0, %1, 0 offen lds"
               :
               : "v"(off), "s"(rs), "s"(m0)
               : "memory", "m0");
}

typedef __attribute__((address_space(3))) i32x4_v lds_i4;

// N scales (dwords) of a lane's rows
template <int N>
__device__ __forceinline__ void fp8_read_scales(const lds_t *q, int *e) {
  static_assert(N == 1 || N == 2 || N == 4, "one LDS read");
  typedef __attribute__((ext_vector_type(N))) int vec;
  const vec v = *reinterpret_cast<const __attribute__((address_space(3))) vec *>(q);
#pragma unroll
  for (int i = 0; i < N; ++i) e[i] = v[i];
}

// At most LEFT of this wave's loads in flight and its LDS reads done, then the workgroup's
// barrier
template <int LEFT>
__device__ __forceinline__ void fp8_wait_barrier() {
  if constexpr (LEFT == 0) {  // (known to the compiler, which then adds no waits of its own)
    __builtin_amdgcn_s_waitcnt(0x0070);
    __syncthreads();
    return;
  }
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" : : "n"(LEFT) : "memory");
}

// What a wave of a BT x BT tile loads: the first half of the NW waves stream A, the others
// B, each RPW of the operand's runs and the scales of 64 * SPW rows.
template <int BT, int NW, int FM, int FN, int D>
struct Fp8Stream {
  static constexpr int NR = BT / 8, RPW = NR / (NW / 2), SPW = BT / 64 / (NW / 2);
  static constexpr int OPND = NR * RUN, SCALES = BT * 4, STAGE = 2 * (OPND + SCALES);
  static constexpr int LOADS = RPW + SPW;
  static_assert(NR % 16 == 0 && SPW >= 1 && SPW * 64 * (NW / 2) == BT, "whole loads per wave");

  lds_t *R0;
  i32x4_v rs, rb;  // values, scales
  uint32_t vo, so[SPW];
  uint32_t ld, lds;
  int opnd, w, kspan, ns, kl;

  __device__ __forceinline__ void init(const Fp8P &p, const Fp8Tile &t, lds_t *ring, int wave, int lane) {
    R0 = ring;
    opnd = wave / (NW / 2);
    w = wave % (NW / 2);
    ns = t.kb1 - t.kb0;
    kspan = t.span();
    kl = 16 * (lane & 7);
    const bool a = opnd == 0;
    const int row0 = a ? t.m0 : t.n0, rows = min((a ? t.m_lim : p.N) - row0, BT);
    const int64_t ld64 = a ? p.lda : p.ldb, lds64 = a ? p.ldsa : p.ldsb;
    ld = (uint32_t)ld64;
    lds = (uint32_t)lds64;
    // offsets past the last row's end read zero; a tile's rows start below 2^30
    rs = make_rsrc((a ? p.A : t.B) + row0 * ld64 + (int64_t)t.kb0 * KB, (uint32_t)((rows - 1) * ld64 + kspan));
    vo = (uint32_t)(w * RPW + NR * (lane >> 3)) * ld + kl;
    const int sh = a ? p.ash : p.bsh, F = a ? FM : FN;
    rb = make_rsrc((a ? p.sa : t.sb) + (row0 >> sh) + t.kb0 * lds64, 0x7FFFFFFFu);
    // scale at position `at`: row (at % F) * 16 + at / F of its wave's part
#pragma unroll
    for (int u = 0; u < SPW; ++u) {
      const int at = 64 * (w * SPW + u) + lane, part = at / (16 * F), in = at % (16 * F);
      const int r = min(part * 16 * F + (in % F) * 16 + in / F, rows - 1);
      so[u] = (uint32_t)(((row0 + r) >> sh) - (row0 >> sh));
    }
  }
  // Load r of stage st (a run; from RPW on the scales); zeros behind a row's end and in
  // stages past the last. No branch: in a loop of one basic block the products stay
  // between the reads, where they are sunk past a branch.
  __device__ __forceinline__ void load(int st, int r) const {
    lds_t *const d = R0 + st % D * STAGE;
    if (r < RPW) {
      const uint32_t o = st * KB + kl < kspan ? vo + (uint32_t)st * KB : OOB;
      dma16(rs, d + opnd * OPND + (w * RPW + r) * RUN, o + (uint32_t)r * ld);
    } else {
      const int u = r - RPW;
      dma1(rb, d + 2 * OPND + opnd * SCALES + (w * SPW + u) * 256, st < ns ? so[u] + (uint32_t)st * lds : OOB);
    }
  }
  // The first D stages on their way, the first one there
  __device__ __forceinline__ void start() const {
#pragma unroll
    for (int st = 0; st < D; ++st) load_part(st, 0, 1);
    fp8_wait_barrier<(D - 1) * LOADS>();
  }
  // part k of n of a stage's loads
  __device__ __forceinline__ void load_part(int st, int k, int n) const {
#pragma unroll
    for (int r = k * LOADS / n; r < (k + 1) * LOADS / n; ++r) load(st, r);
  }
};

// The epilogue of a wave's FM x FN blocks at rows m0 .., columns n0 ..: 32 rows at a time
// through E, the wave's own 2 KiB * FN of LDS, so that stores cover whole lines: written as
// the products leave them (chunk of 4 columns c of row r at c ^ (r % 16)), read by rows.
template <int FM, int FN>
__device__ __forceinline__ void fp8_epilogue(const Fp8P &p, const Fp8Tile &t, int m0, int n0, lds_t *E, int lane,
                                             const f32x4_v (&acc)[FM][FN]) {
  constexpr int CH = 4 * FN;  // chunks of a row
  typedef __attribute__((address_space(3))) f32x4_v lds_f4;
  const int i16 = lane & 15, g = lane >> 4;
#pragma unroll
  for (int h = 0; h < FM / 2; ++h) {
#pragma unroll
    for (int f = 0; f < 2; ++f)
#pragma unroll
      for (int j = 0; j < FN; ++j) {
        const int r = 16 * f + i16, c = 4 * j + g;
        *reinterpret_cast<lds_f4 *>(E + r * (64 * FN) + ((c ^ i16) << 4)) = acc[2 * h + f][j];
      }
    const int m = m0 + 32 * h;
    auto chunk = [&](int r, int c) { return *reinterpret_cast<const lds_f4 *>(E + r * (64 * FN) + ((c ^ (r & 15)) << 4)); };
    if (p.store16) {  // 8 columns at a time
#pragma unroll
      for (int u = 0; u < 16 * CH / 64; ++u) {
        const int at = u * 64 + lane, r = at / (CH / 2), c = at % (CH / 2) * 2, n = n0 + 4 * c;
        const f32x4_v x = chunk(r, c), y = chunk(r, c + 1);
        if (m + r >= t.m_lim || n >= p.N) continue;
        if (n + 8 <= p.N) {
          const int64_t to = t.c_off + (int64_t)(m + r) * p.ldc + n;
          if (p.c_dt == LC_BF16) {
            const bf16x8_v o = {(__bf16)x[0], (__bf16)x[1], (__bf16)x[2], (__bf16)x[3],
                                (__bf16)y[0], (__bf16)y[1], (__bf16)y[2], (__bf16)y[3]};
            fp8_stream_store(static_cast<__bf16 *>(p.C) + to, o);
          } else {
            const f16x8_v o = {(_Float16)x[0], (_Float16)x[1], (_Float16)x[2], (_Float16)x[3],
                               (_Float16)y[0], (_Float16)y[1], (_Float16)y[2], (_Float16)y[3]};
            fp8_stream_store(static_cast<_Float16 *>(p.C) + to, o);
          }
        } else {
          fp8_store4(p, t.c_off, m + r, n, x[0], x[1], x[2], x[3]);
          if (n + 4 < p.N) fp8_store4(p, t.c_off, m + r, n + 4, y[0], y[1], y[2], y[3]);
        }
      }
    } else {
#pragma unroll 1
      for (int u = 0; u < 32 * CH / 64; ++u) {
        const int at = u * 64 + lane, r = at / CH, c = at % CH, n = n0 + 4 * c;
        const f32x4_v v = chunk(r, c);
        if (m + r < t.m_lim && n < p.N) fp8_store4(p, t.c_off, m + r, n, v[0], v[1], v[2], v[3]);
      }
    }
  }
}

template <int FA, int FB, int BT, int WM, int WN, int D>
__global__ __launch_bounds__(64 * WM * WN) void fp8_tile_kernel(Fp8P p, uint32_t first) {
  constexpr int NW = WM * WN, FM = BT / 16 / WM, FN = BT / 16 / WN;
  typedef Fp8Stream<BT, NW, FM, FN, D> Stream;
  constexpr int NR = Stream::NR, OPND = Stream::OPND, SCALES = Stream::SCALES, STAGE = Stream::STAGE;
  constexpr int EPI = NW * 2048 * FN;
  __shared__ __align__(16) char ring[D * STAGE > EPI ? D * STAGE : EPI];

  const int lane = threadIdx.x & 63, i16 = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave % WM, wn = wave / WM;
  Fp8Tile t;
  if (!fp8_tile<BT, BT, true>(p, first + blockIdx.x, t)) return;  // before any barrier

  f32x4_v acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) acc[i][j] = f32x4_v{0.0f, 0.0f, 0.0f, 0.0f};

  lds_t *const R0 = LDS_AS(char, ring);
  Stream in;
  in.init(p, t, R0, wave, lane);
  const int ns = in.ns;

  i32x8_v fa[FM], fb[FN];
  int ea[FM], eb[FN];
  // This lane's place in the stage that is read, as LDS byte offsets: A's and B's values,
  // their scales. One register each, moved to the next stage at the barrier.
  uint32_t qa = i16 * RUN + g * 16 + (wm * FM * 16) / NR * 128 + (wm * FM * 16) % NR * RUN;
  uint32_t qb = OPND + i16 * RUN + g * 16 + (wn * FN * 16) / NR * 128 + (wn * FN * 16) % NR * RUN;
  uint32_t qea = 2 * OPND + (wm * 16 + i16) * FM * 4, qeb = 2 * OPND + SCALES + (wn * 16 + i16) * FN * 4;
  const uint32_t ta = 2 * qa + STAGE, tb = 2 * qb + STAGE, tea = 2 * qea + STAGE, teb = 2 * qeb + STAGE;
  auto next_stage = [&](int st) {  // from st's
    if constexpr (D == 2) {
      qa = ta - qa;
      qb = tb - qb;
      qea = tea - qea;
      qeb = teb - qeb;
    } else {
      const uint32_t by = st % D == D - 1 ? (uint32_t)(1 - D) * STAGE : STAGE;
      qa += by;
      qb += by;
      qea += by;
      qeb += by;
    }
  };
  auto frag = [&](uint32_t q, int f) -> i32x8_v {  // fragment f of the wave's
    const lds_t *const at = R0 + q + (16 * f) % NR * RUN + (16 * f) / NR * 128;
    const i32x4_v lo = *reinterpret_cast<const lds_i4 *>(at), hi = *reinterpret_cast<const lds_i4 *>(at + 64);
    return i32x8_v{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
  };
  // fragment f, and before a half's first one the half's scales
  auto read_a = [&](int f) {
    if (f % (FM / 2) == 0) fp8_read_scales<FM / 2>(R0 + qea + 4 * f, &ea[f]);
    fa[f] = frag(qa, f);
  };
  auto read_b = [&](int f) {
    if (f % (FN / 2) == 0) fp8_read_scales<FN / 2>(R0 + qeb + 4 * f, &eb[f]);
    fb[f] = frag(qb, f);
  };
  // Half HA of A's fragments by half HB of B's, in FN / 2 parts of FM / 2 products: B's
  // fragments are used in the order in which they were read. Part j first reads (rd) and
  // loads (ld) its share.
  auto step = [&](auto ha, auto hb, auto rd, auto ldr) {
    constexpr int I0 = decltype(ha)::value * FM / 2, J0 = decltype(hb)::value * FN / 2;
#pragma unroll
    for (int j = 0; j < FN / 2; ++j) {
      rd(j);
      ldr(j);
#pragma unroll
      for (int i = 0; i < FM / 2; ++i)
        acc[I0 + i][J0 + j] = fp8_mul<FA, FB>(fa[I0 + i], fb[J0 + j], ea[I0 + i], eb[J0 + j], acc[I0 + i][J0 + j]);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  auto none = [](int) {};
  auto rd_a = [&](int h) { return [=, &read_a](int j) { if (j < FM / 2) read_a(h * FM / 2 + j); }; };
  auto rd_b = [&](int h) { return [=, &read_b](int j) { read_b(h * FN / 2 + j); }; };
  auto ld_of = [&](int st, int h) {  // a part's share of the stage's loads, in the two steps after the barrier
    return [=, &in](int j) { in.load_part(st, h * FN / 2 + j, FN); };
  };
  typedef std::integral_constant<int, 0> H0;
  typedef std::integral_constant<int, 1> H1;
  auto stage = [&](int st, auto b0, auto b1) {
    step(H0{}, b0, rd_b(b1), none);
    step(H0{}, b1, rd_a(1), none);
    fp8_wait_barrier<(D - 2) * Stream::LOADS>();
    next_stage(st);
    // (after the last stage this reads another place's old values, unused)
    step(H1{}, b1, rd_a(0), ld_of(st + D, 0));
    step(H1{}, b0, rd_b(b1), ld_of(st + D, 1));
  };
  in.start();
  if (ns > 0) {
#pragma unroll
    for (int i = 0; i < FM / 2; ++i) read_a(i);
#pragma unroll
    for (int j = 0; j < FN / 2; ++j) read_b(j);
    int st = 0;
    for (; st + 1 < ns; st += 2) {
      stage(st, H0{}, H1{});
      stage(st + 1, H1{}, H0{});
    }
    if (st < ns) stage(st, H0{}, H1{});
  }

  fp8_wait_barrier<0>();  // every wave's reads are done, and the zeros of stages past the last have landed
  fp8_epilogue<FM, FN>(p, t, t.m0 + wm * FM * 16, t.n0 + wn * FN * 16, R0 + wave * (2048 * FN), lane, acc);
}

// Results of fp16 and fp32: the same stages, the values converted to bf16 with their scales on the
// way to the bf16 instruction. A lane's 32 values of a row's 128 are two pieces of 16; a
// stage is multiplied in two steps, the pieces at 0 and at 64, and while one multiplies the
// other's are read. A step is two products of 32 k: 8 values of each lane. Bound: the
// conversions, two (of two values each) beside every product, which then takes 30 cycles
// instead of 16: 3001 x 1155 x 1872 22.5 us, 0.58 PFLOP/s; 4096 x 11008 x 4096 297 us, 1.24, in fp16
// 287, accumulated 363 (C, 180 MB, is read too; the bf16 product of lc_gemm accumulates in 334);
// the eight experts' weight gradients (1023 or 1026 rows each) 103, accumulated 175 (lc_gemm 146).
template <int FA, int FB, int D>
__global__ __launch_bounds__(256) void fp8_wide_kernel(Fp8P p, uint32_t first) {
  constexpr int BT = 128, FM = 4, FN = 4;
  typedef Fp8Stream<BT, 4, FM, FN, D> Stream;
  constexpr int NR = Stream::NR, OPND = Stream::OPND, SCALES = Stream::SCALES, STAGE = Stream::STAGE;
  __shared__ __align__(16) char ring[D * STAGE];
  static_assert(D * STAGE >= 4 * 2048 * FN, "epilogue");

  const int lane = threadIdx.x & 63, i16 = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave & 1, wn = wave >> 1;
  Fp8Tile t;
  if (!fp8_tile<BT, BT, true>(p, first + blockIdx.x, t)) return;  // before any barrier

  f32x4_v acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) acc[i][j] = f32x4_v{0.0f, 0.0f, 0.0f, 0.0f};

  lds_t *const R0 = LDS_AS(char, ring);
  Stream in;
  in.init(p, t, R0, wave, lane);
  const int ns = in.ns;
  uint32_t qa = i16 * RUN + g * 16 + wm * FM * 128, qb = OPND + i16 * RUN + g * 16 + wn * FN * 128;
  static_assert(NR == 16, "fragment f: position f of the runs");
  uint32_t qea = 2 * OPND + (wm * 16 + i16) * FM * 4, qeb = 2 * OPND + SCALES + (wn * 16 + i16) * FN * 4;

  i32x4_v ra[2][FM], rb[2][FN];  // pieces 0, 1
  int ea[FM], eb[FN];
  auto read = [&](int h, int f) {  // fragment f of A (below FM) or B
    if (f < FM) ra[h][f] = *reinterpret_cast<const lds_i4 *>(R0 + qa + f * 128 + h * 64);
    else rb[h][f - FM] = *reinterpret_cast<const lds_i4 *>(R0 + qb + (f - FM) * 128 + h * 64);
  };
  float ga[FM], gb[FN];
  auto scales = [&]() {
    fp8_read_scales<FM>(R0 + qea, ea);
    fp8_read_scales<FN>(R0 + qeb, eb);
  };
  auto step = [&](int h, auto each) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      bf16x8_v ca[FM];
#pragma unroll
      for (int i = 0; i < FM; ++i) ca[i] = fp8_to_bf16<FA>(ra[h][i][2 * u], ra[h][i][2 * u + 1], ga[i]);
#pragma unroll
      for (int j = 0; j < FN; ++j) {
        each(u * FN + j);
        const bf16x8_v cb = fp8_to_bf16<FB>(rb[h][j][2 * u], rb[h][j][2 * u + 1], gb[j]);
#pragma unroll
        for (int i = 0; i < FM; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(cb, ca[i], acc[i][j], 0, 0, 0);
      }
    }
  };
  in.start();
  if (ns > 0) {
    scales();
#pragma unroll
    for (int f = 0; f < FM + FN; ++f) read(0, f);
    for (int st = 0; st < ns; ++st) {
#pragma unroll
      for (int i = 0; i < FM; ++i) ga[i] = fp8_scale(ea[i]);
#pragma unroll
      for (int j = 0; j < FN; ++j) gb[j] = fp8_scale(eb[j]);
      step(0, [&](int j) { read(1, j); });
      fp8_wait_barrier<(D - 2) * Stream::LOADS>();
      const uint32_t by = st % D == D - 1 ? (uint32_t)(1 - D) * STAGE : STAGE;
      qa += by;
      qb += by;
      qea += by;
      qeb += by;
      scales();
      step(1, [&](int j) {
        read(0, j);
        in.load_part(st + D, j, 2 * FN);
      });
    }
  }
  fp8_wait_barrier<0>();
  fp8_epilogue<FM, FN>(p, t, t.m0 + wm * FM * 16, t.n0 + wn * FN * 16, R0 + wave * (2048 * FN), lane, acc);
}

// Small tiles, k split over the waves: each of W waves takes every W-th block of k for the
// whole T x T tile and streams it into two stages of its own in LDS, with no barrier but
// its own wait; the waves' sums are added through LDS in order. For grids of few tiles,
// where a tile's chain of blocks, each a load's latency long, is the time: 1 x 4096 x 4096
// 6.2 us (an operand of 16.8 MB at 2.7 TB/s); 64 rows 6.7, by tiles of 128 15.
// Stage: rows of 128 bytes, 16-byte piece c of row r at c ^ (r / 2 % 8), which keeps
// fragment reads (16 rows, four pieces) free of bank conflicts without padding.
template <int FA, int FB, bool F32, int T, int W>
__global__ __launch_bounds__(64 * W) void fp8_split_kernel(Fp8P p, uint32_t first) {
  constexpr int F = T / 16, RUNS = T / 8;          // 1 KiB loads of an operand
  constexpr int OPND = T * 128, STAGE = 2 * OPND + 512, LOADS = 2 * RUNS + 2;
  constexpr int OUT = W * T * T * 4;
  __shared__ __align__(16) char ring[2 * W * STAGE > OUT ? 2 * W * STAGE : OUT];
  const int lane = threadIdx.x & 63, i16 = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  Fp8Tile t;
  if (!fp8_tile<T, T, true>(p, first + blockIdx.x, t)) return;  // before any barrier

  lds_t *const R = LDS_AS(char, ring), *const mine = R + wave * 2 * STAGE;
  const int kspan = t.span(), nb = t.kb1 - t.kb0;
  const int n = (nb - wave + W - 1) / W;  // this wave's blocks
  i32x4_v rs[2], rb[2];
  uint32_t vo[2], so[2];
  const int pos = lane >> 3, kl = 16 * ((lane & 7) ^ (pos >> 1));  // runs of an even row: r / 2 % 8 = 4 (run % 2) + pos / 2
#pragma unroll
  for (int o = 0; o < 2; ++o) {
    const int row0 = o == 0 ? t.m0 : t.n0, rows = min((o == 0 ? t.m_lim : p.N) - row0, T);
    const int64_t ld = o == 0 ? p.lda : p.ldb, lds = o == 0 ? p.ldsa : p.ldsb;
    const int sh = o == 0 ? p.ash : p.bsh;
    rs[o] = make_rsrc((o == 0 ? p.A : t.B) + row0 * ld + (int64_t)t.kb0 * KB, (uint32_t)((rows - 1) * ld + kspan));
    vo[o] = (uint32_t)pos * (uint32_t)ld;
    rb[o] = make_rsrc((o == 0 ? p.sa : t.sb) + (row0 >> sh) + t.kb0 * lds, 0x7FFFFFFFu);
    const int r = min(lane % F * 16 + lane / F, rows - 1);  // scale at position `lane`: row lane / F of fragment lane % F
    so[o] = (uint32_t)(((row0 + r) >> sh) - (row0 >> sh));
  }
  auto load = [&](int i) {  // this wave's i-th block (past the last: zeros)
    const int b = wave + i * W;
    lds_t *const d = mine + (i & 1) * STAGE;
#pragma unroll
    for (int o = 0; o < 2; ++o) {
      const uint32_t ld = (uint32_t)(o == 0 ? p.lda : p.ldb), lds = (uint32_t)(o == 0 ? p.ldsa : p.ldsb);
#pragma unroll
      for (int r = 0; r < RUNS; ++r) {
        const int k = kl ^ (64 * (r & 1));
        const uint32_t at = b * KB + k < kspan ? vo[o] + (uint32_t)r * 8 * ld + (uint32_t)(b * KB + k) : OOB;
        dma16(rs[o], d + o * OPND + r * 1024, at);
      }
      dma1(rb[o], d + 2 * OPND + o * 256, b < nb && lane < T ? so[o] + (uint32_t)b * lds : OOB);
    }
  };
  f32x4_v acc[F][F];
#pragma unroll
  for (int i = 0; i < F; ++i)
#pragma unroll
    for (int j = 0; j < F; ++j) acc[i][j] = f32x4_v{0.0f, 0.0f, 0.0f, 0.0f};
  const uint32_t q = i16 * 128 + ((g ^ (i16 >> 1)) << 4);
  load(0);
  load(1);
  for (int s = 0; s < n; ++s) {
    asm volatile("s_waitcnt vmcnt(%0)" : : "n"(LOADS) : "memory");
    const lds_t *const d = mine + (s & 1) * STAGE;
    i32x8_v fa[F], fb[F];
    int ea[F], eb[F];
    auto frag = [&](const lds_t *at) -> i32x8_v {
      const i32x4_v lo = *reinterpret_cast<const lds_i4 *>(at + q), hi = *reinterpret_cast<const lds_i4 *>(at + (q ^ 64));
      return i32x8_v{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    };
    fp8_read_scales<F>(d + 2 * OPND + i16 * F * 4, ea);
    fp8_read_scales<F>(d + 2 * OPND + 256 + i16 * F * 4, eb);
#pragma unroll
    for (int i = 0; i < F; ++i) {
      fa[i] = frag(d + i * 2048);
      fb[i] = frag(d + OPND + i * 2048);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");  // read: the stage may be overwritten
    load(s + 2);
    if constexpr (F32) {
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        bf16x8_v ca[F];
#pragma unroll
        for (int i = 0; i < F; ++i) ca[i] = fp8_to_bf16<FA>(fa[i][2 * h], fa[i][2 * h + 1], fp8_scale(ea[i]));
#pragma unroll
        for (int j = 0; j < F; ++j) {
          const bf16x8_v cb = fp8_to_bf16<FB>(fb[j][2 * h], fb[j][2 * h + 1], fp8_scale(eb[j]));
#pragma unroll
          for (int i = 0; i < F; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(cb, ca[i], acc[i][j], 0, 0, 0);
        }
      }
    } else {
#pragma unroll
      for (int j = 0; j < F; ++j)
#pragma unroll
        for (int i = 0; i < F; ++i) acc[i][j] = fp8_mul<FA, FB>(fa[i], fb[j], ea[i], eb[j], acc[i][j]);
    }
  }
  // every load has landed before the stages become sums
  fp8_wait_barrier<0>();
  constexpr int CH = T / 4, SW = CH - 1;  // chunks of 4 columns of a row; chunk c of row r at c ^ (r % CH)
  typedef __attribute__((address_space(3))) f32x4_v lds_f4;
  auto place = [&](int w, int r, int c) { return reinterpret_cast<lds_f4 *>(R + ((w * T + r) * CH + (c ^ (r & SW))) * 16); };
#pragma unroll
  for (int i = 0; i < F; ++i)
#pragma unroll
    for (int j = 0; j < F; ++j) *place(wave, 16 * i + i16, 4 * j + g) = acc[i][j];
  fp8_wait_barrier<0>();
#pragma unroll
  for (int at = threadIdx.x; at < T * CH; at += 64 * W) {
    const int r = at / CH, c = at % CH;
    f32x4_v v = *place(0, r, c);
#pragma unroll
    for (int w = 1; w < W; ++w) v += *place(w, r, c);
    const int m = t.m0 + r, col = t.n0 + 4 * c;
    if (m < t.m_lim && col < p.N) fp8_store4(p, t.c_off, m, col, v[0], v[1], v[2], v[3]);
  }
}

// GO(kernel with FA, FB in scope), over the grid of BT x BT tiles
#define FP8_LAUNCH(BT, THREADS, ...)                                                                   \
  do {                                                                                                 \
    uint32_t grid;                                                                                     \
    LC_TRY((fp8_grid<BT, BT>(p, &grid)));                                                              \
    launch_parts(grid, [&](uint32_t first, uint32_t count) {                                           \
      fp8_with_formats(a, [&](auto fa, auto fb) {                                                      \
        constexpr int FA = decltype(fa)::value, FB = decltype(fb)::value;                              \
        hipLaunchKernelGGL((__VA_ARGS__), dim3(count), dim3(THREADS), 0, s, p, first);                 \
      });                                                                                              \
    });                                                                                                \
    return check_launch("fp8 product");                                                                \
  } while (0)

}  // namespace

lc_status gemm_fp8_tile_launch(Fp8P p, const lc_gemm_fp8_args &a, int tile, bool deep, bool f32, hipStream_t s) {
  if (f32) {
    if (tile == 32) FP8_LAUNCH(32, 512, fp8_split_kernel<FA, FB, true, 32, 8>);
    if (tile == 64) FP8_LAUNCH(64, 256, fp8_split_kernel<FA, FB, true, 64, 4>);
    if (deep) FP8_LAUNCH(128, 256, fp8_wide_kernel<FA, FB, 4>);
    FP8_LAUNCH(128, 256, fp8_wide_kernel<FA, FB, 2>);
  }
  if (tile == 32) FP8_LAUNCH(32, 512, fp8_split_kernel<FA, FB, false, 32, 8>);
  if (tile == 64) FP8_LAUNCH(64, 256, fp8_split_kernel<FA, FB, false, 64, 4>);
  if (tile == 256) FP8_LAUNCH(256, 512, fp8_tile_kernel<FA, FB, 256, 4, 2, 2>);
  if (deep) FP8_LAUNCH(128, 256, fp8_tile_kernel<FA, FB, 128, 2, 2, 4>);
  FP8_LAUNCH(128, 256, fp8_tile_kernel<FA, FB, 128, 2, 2, 2>);
}

}  // namespace lc
