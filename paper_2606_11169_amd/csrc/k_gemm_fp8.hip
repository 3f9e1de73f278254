// Products of 8-bit operands with a power-of-two scale per block of 128 (gfx950):
//
//   C(m, n) = sum_b 2^(sa(m, b) + sb(n, b) - 254) sum_{k in block b} A(m, k) B(n, k)
//
// Results of bf16 are summed by v_mfma_scale_f32_16x16x128_f8f6f4, which takes the
// scales as they are, one byte per row and 32 k. Of each 8 neighbouring products it cuts off,
// towards zero, what lies below 2^(E - 13), 2^E the largest's factors' powers of two (2^16 + 8
// is exact, 2^16 + 7 is 2^16, and so are 448^2 + 7 and 448^2), and adds the rest, and the sums
// of eights, in fp32: 1.5e-5 of the result on random signs; at most 7 * 2^-13 of sum |a b|,
// whatever K, where all have one sign: 0.22 of bf16's half step, 2^-8, but 1.75 of fp16's.
// So results of fp16 and fp32 are summed by v_mfma_f32_16x16x32_bf16 on the same values.
#include "gemm_fp8.hpp"

namespace lc {
namespace {

// Tiles of 16 x 16, fragments straight from global memory: 8 waves take the k blocks in
// turn, a block's loads under way while the one before is multiplied, and their sums are
// added in LDS in order. For products of few rows or a short k, where a tile's time is a
// few latencies: 14 x 3616, K 7856 7.9 us, by tiles of 32 8.2.
template <int FA, int FB, bool F32>
__global__ __launch_bounds__(512) void fp8_direct_kernel(Fp8P p, uint32_t first) {
  constexpr int T = 16, W = 8;
  Fp8Tile t;
  if (!fp8_tile<T, T>(p, first + blockIdx.x, t)) return;  // before any barrier
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int i16 = lane & 15, g = lane >> 4;

  // (rows past the end: the last one's values, unused)
  const int64_t ra = min(t.m0 + i16, t.m_lim - 1), rb = min(t.n0 + i16, p.N - 1);
  const uint8_t *const pa = p.A + ra * p.lda + 16 * g, *const pb = t.B + rb * p.ldb + 16 * g;
  const uint8_t *const qa = p.sa + (ra >> p.ash), *const qb = t.sb + (rb >> p.bsh);

  auto frag = [&](const uint8_t *q, int k) -> i32x8_v {  // k: the lane's first of the block
    typedef __attribute__((ext_vector_type(4))) int i4;
    i4 lo = i4{0, 0, 0, 0}, hi = i4{0, 0, 0, 0};
    if (k < t.kend) lo = *reinterpret_cast<const i4 *>(q);
    if (k + 64 < t.kend) hi = *reinterpret_cast<const i4 *>(q + 64);
    return i32x8_v{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
  };
  struct Block {
    i32x8_v a, b;
    int ea, eb;
  };
  auto fetch = [&](Block &x, int kb) {  // (a block past the last: zeros)
    const bool in = kb < t.kb1;
    const int64_t at = in ? kb : t.kb0;
    const int k = in ? kb * KB + 16 * g : t.kend;
    x.a = frag(pa + at * KB, k);
    x.ea = qa[at * p.ldsa];
    x.b = frag(pb + at * KB, k);
    x.eb = qb[at * p.ldsb];
  };
  f32x4_v acc = f32x4_v{0.0f, 0.0f, 0.0f, 0.0f};
  auto multiply = [&](const Block &x) {
    if constexpr (F32) {
#pragma unroll
      for (int h = 0; h < 4; ++h)
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fp8_to_bf16<FB>(x.b[2 * h], x.b[2 * h + 1], fp8_scale(x.eb)),
                                                      fp8_to_bf16<FA>(x.a[2 * h], x.a[2 * h + 1], fp8_scale(x.ea)),
                                                      acc, 0, 0, 0);
    } else {
      acc = fp8_mul<FA, FB>(x.a, x.b, x.ea, x.eb, acc);
    }
  };
  if (t.kb0 + wave < t.kb1) {
    Block x, y;
    fetch(x, t.kb0 + wave);
    for (int kb = t.kb0 + wave; kb < t.kb1; kb += 2 * W) {
      fetch(y, kb + W);
      multiply(x);
      if (kb + W >= t.kb1) break;
      fetch(x, kb + 2 * W);
      multiply(y);
    }
  }
  __shared__ __align__(16) float part[W - 1][256];
  if (wave > 0) *reinterpret_cast<f32x4_v *>(&part[wave - 1][4 * lane]) = acc;
  __syncthreads();
  if (wave > 0) return;
#pragma unroll
  for (int s = 0; s < W - 1; ++s) acc += *reinterpret_cast<const f32x4_v *>(&part[s][4 * lane]);
  const int m = t.m0 + i16, n = t.n0 + 4 * g;
  if (m < t.m_lim && n < p.N) fp8_store4(p, t.c_off, m, n, acc[0], acc[1], acc[2], acc[3]);
}

static lc_status direct_launch(Fp8P p, const lc_gemm_fp8_args &a, bool f32, hipStream_t s) {
  uint32_t grid;
  LC_TRY((fp8_grid<16, 16>(p, &grid)));
  launch_parts(grid, [&](uint32_t first, uint32_t count) {
    fp8_with_formats(a, [&](auto fa, auto fb) {
      constexpr int FA = decltype(fa)::value, FB = decltype(fb)::value;
      if (f32) hipLaunchKernelGGL((fp8_direct_kernel<FA, FB, true>), dim3(count), dim3(512), 0, s, p, first);
      else hipLaunchKernelGGL((fp8_direct_kernel<FA, FB, false>), dim3(count), dim3(512), 0, s, p, first);
    });
  });
  return check_launch("fp8_direct_kernel");
}

}  // namespace

static lc_status check_gemm_fp8(const lc_gemm_fp8_args &a) {
  if (a.M < 0 || a.N <= 0 || a.K <= 0) return fail(LC_ERR_INVALID_ARG, "gemm fp8: need M >= 0, N > 0, K > 0");
  if (a.M >= (1 << 30) || a.N >= (1 << 30) || a.K >= (1 << 30))
    return fail(LC_ERR_UNSUPPORTED, "gemm fp8: dimension too large");
  if ((a.a_dtype != LC_FP8_E4M3 && a.a_dtype != LC_FP8_E5M2) || (a.b_dtype != LC_FP8_E4M3 && a.b_dtype != LC_FP8_E5M2))
    return fail(LC_ERR_INVALID_ARG, "gemm fp8: operands must be e4m3 or e5m2");
  if ((a.a_block_rows != 1 && a.a_block_rows != 128) || (a.b_block_rows != 1 && a.b_block_rows != 128))
    return fail(LC_ERR_INVALID_ARG, "gemm fp8: block rows must be 1 or 128");
  if (a.epilogue < LC_EPI_STORE || a.epilogue > LC_EPI_SWIGLU_BWD)
    return fail(LC_ERR_INVALID_ARG, "gemm fp8: unknown epilogue %d", a.epilogue);
  if (a.epilogue > LC_EPI_RESIDUAL)
    return fail(LC_ERR_UNSUPPORTED, "gemm fp8: epilogues are STORE, STORE_F32, ACCUM_F32 and RESIDUAL");
  const bool typed = a.epilogue == LC_EPI_STORE || a.epilogue == LC_EPI_RESIDUAL;
  if (typed && !valid_dtype(a.c_dtype)) return fail(LC_ERR_INVALID_ARG, "gemm fp8: unknown c_dtype");
  const int64_t MOST = (int64_t)1 << 30;
  if (a.M > 0 && (!a.A || !a.B || !a.a_scale || !a.b_scale || !a.C || !aligned16(a.A) || !aligned16(a.B) ||
                  !aligned16(a.a_scale) || !aligned16(a.b_scale) || !aligned16(a.C)))
    return fail(LC_ERR_INVALID_ARG, "gemm fp8: null or unaligned pointer");
  if (a.K % 16 || a.lda % 16 || a.ldb % 16 || a.ld_a_scale % 4 || a.ld_b_scale % 4)
    return fail(LC_ERR_INVALID_ARG, "gemm fp8: K, lda, ldb must be multiples of 16, ld_a_scale, ld_b_scale of 4");
  if (a.lda < a.K || a.ldb < a.K || a.ld_a_scale < (a.M + a.a_block_rows - 1) / a.a_block_rows ||
      a.ld_b_scale < (a.N + a.b_block_rows - 1) / a.b_block_rows || a.ldc < a.N)
    return fail(LC_ERR_INVALID_ARG, "gemm fp8: leading dimension too small");
  if (a.lda > (1 << 22) || a.ldb > (1 << 22) || a.ld_a_scale > MOST || a.ld_b_scale > MOST || a.ldc > MOST)
    return fail(LC_ERR_UNSUPPORTED, "gemm fp8: leading dimension too large");
  const int64_t lines = (a.K + 127) / 128;  // (offsets of scales within a tile are 32 bits)
  if (lines * a.ld_a_scale > INT32_MAX || lines * a.ld_b_scale > INT32_MAX)
    return fail(LC_ERR_UNSUPPORTED, "gemm fp8: scales of 2^31 bytes or more");
  if (a.epilogue == LC_EPI_RESIDUAL) {
    if (a.M > 0 && (!a.R || !aligned16(a.R))) return fail(LC_ERR_INVALID_ARG, "gemm fp8: null or unaligned residual");
    if (!valid_dtype(a.r_dtype) || a.ldr < a.N || a.ldr > MOST)
      return fail(LC_ERR_INVALID_ARG, "gemm fp8: bad residual operand");
  }
  if (a.group_mode != LC_GROUP_NONE) {
    if (a.group_mode != LC_GROUP_ROWS && a.group_mode != LC_GROUP_K)
      return fail(LC_ERR_INVALID_ARG, "gemm fp8: unknown group mode %d", a.group_mode);
    if (a.n_groups < 1 || a.n_groups > 64) return fail(LC_ERR_INVALID_ARG, "gemm fp8: n_groups must be 1..64");
    if (!a.group_offsets || (reinterpret_cast<uintptr_t>(a.group_offsets) & 3))
      return fail(LC_ERR_INVALID_ARG, "gemm fp8: group offsets must be a 4-byte aligned device array");
    if (a.epilogue == LC_EPI_RESIDUAL)
      return fail(LC_ERR_UNSUPPORTED, "gemm fp8: grouped products take STORE, STORE_F32 or ACCUM_F32");
    const int64_t FAR = (int64_t)1 << 50;
    if (a.group_mode == LC_GROUP_ROWS) {
      if (a.a_block_rows != 1) return fail(LC_ERR_UNSUPPORTED, "gemm fp8: LC_GROUP_ROWS needs a_block_rows 1");
      if (a.group_stride_b < 0 || a.group_stride_b % 16 || a.group_stride_b_scale < 0 ||
          a.group_stride_b > FAR || a.group_stride_b_scale > FAR)
        return fail(LC_ERR_INVALID_ARG, "gemm fp8: bad group stride of B or its scales");
    } else if (a.group_stride_c < 0 || a.group_stride_c > FAR) {
      return fail(LC_ERR_INVALID_ARG, "gemm fp8: bad group_stride_c");
    } else if (a.group_stride_c < (a.M - 1) * a.ldc + a.N) {
      // groups not one behind the other: rows of two, `far` elements apart, must not meet
      for (int64_t g = 1; g < a.n_groups; ++g) {
        const int64_t far = g * a.group_stride_c, rows = far / a.ldc, rest = far % a.ldc;
        if ((rows < a.M && rest < a.N) || (rows + 1 < a.M && a.ldc - rest < a.N))
          return fail(LC_ERR_INVALID_ARG, "gemm fp8: the groups' results overlap (group_stride_c)");
      }
    }
  }
  return LC_OK;
}

// How a product may be tiled, and its expected time in ns:
//   base + max(fix + chain * its, tiles / slots * (fix + rate * its))
// with whole rounds of tiles / slots above one. its: a tile's blocks of 128 k, for each of
// the waves that share them; slots: workgroups that run at once. `chain` is a block's
// latency where few workgroups run, `rate` its share of the chip's throughput. Tile 16 has
// many workgroups per compute unit and rate counts its blocks alone. Fitted to 100 products
// of 1 to 11680 x 16 to 14000 outputs at K = 64 to 16256, of bf16 and of fp32 each (the
// times are 7 to 25% off); the choice costs 0.7% (bf16) and 1% (fp32) over the fastest
// on the mean, 27% at most. Both sides at a few sizes, us (M x N, K): 4096 x 4096, 4096:
// 256 53, 128 64, 64 150; 1024 x 4096, 4096: deep 128 19.4, 128 24.7, 64 38, 256 42; 256 x
// 4096, 4096: 64 10.5, 128 15.9, 32 20.5; 64 x 4096, 4096: 32 6.7, 64 10, 16 17.9; 14 x 3616,
// 7856: 16 7.9, 32 8.2, deep 128 26.
struct Fp8Tiling {
  int tile;
  bool deep;
  int waves, slots;
  int base, fix, chain, rate;
};
static const Fp8Tiling kTilingsBf16[] = {
    {256, false, 1, 256, 3200, 7000, 980, 1350}, {128, false, 1, 512, 2670, 3030, 465, 930},
    {128, true, 1, 256, 2440, 3680, 356, 442},   {64, false, 4, 256, 2130, 2890, 655, 856},
    {32, false, 8, 256, 2180, 1590, 545, 780},   {16, false, 8, 0, 2630, 180, 660, 110},
};
static const Fp8Tiling kTilingsF32[] = {
    {128, false, 1, 512, 4420, 3140, 833, 1634}, {128, true, 1, 256, 1750, 5620, 806, 894},
    {64, false, 4, 256, 1970, 3200, 1016, 1121}, {32, false, 8, 256, 2220, 1570, 696, 935},
    {16, false, 8, 0, 2740, 1320, 667, 115},
};

static const Fp8Tiling *pick(const lc_gemm_fp8_args &a, bool f32) {
  const Fp8Tiling *const first = f32 ? kTilingsF32 : kTilingsBf16;
  const int n = f32 ? (int)(sizeof(kTilingsF32) / sizeof(*first)) : (int)(sizeof(kTilingsBf16) / sizeof(*first));
  const Fp8Tiling *best = first;
  double least = 0.0;
  for (int i = 0; i < n; ++i) {
    const Fp8Tiling &v = first[i];
    int64_t tm = (a.M + v.tile - 1) / v.tile;
    const int64_t tn = (a.N + v.tile - 1) / v.tile;
    // grouped rows: about half a partial row of tiles per group besides
    if (a.group_mode == LC_GROUP_ROWS) tm += (a.n_groups + 1) / 2;
    const int64_t groups = a.group_mode == LC_GROUP_K ? a.n_groups : 1;
    const int64_t most = (tm + (a.group_mode == LC_GROUP_ROWS ? a.n_groups : 0)) * tn * groups;
    if (i > 0 && most > INT32_MAX - 8 * 64) continue;
    // Grouped: every workgroup first reads the offsets and looks its tile up. In ns per 256
    // tiles of 16, per further round of the others; fitted with 940 grouped products of up to 32
    // groups, the first and the last with rows and those between empty, where the choice then costs
    // 4% over the fastest on the mean (without 8 and 17%: 52 rows x 12634, K 320, 32 groups 41 us by
    // 16, 9 by 128). Groups that all have rows were not in the fit: 8187 rows x 2816 x 2048 of eight
    // take 128, where 256 is faster: 1023 or 1026 rows each 55.8 us, 52.1; 100 to 2000 56.9, 52.1.
    double look = 0.0;
    if (a.group_mode != LC_GROUP_NONE) {
      const double rounds = (double)most / (v.tile == 16 ? 256 : v.slots);
      look = v.tile == 16 ? 900.0 * rounds : rounds > 1.0 ? 500.0 * (rounds - 1.0) : 0.0;
    }
    auto time = [&](double tiles, int64_t blocks) -> double {
      const double its = (double)((blocks + v.waves - 1) / v.waves);
      double one = v.fix + v.chain * its, full;
      if (v.tile == 16) {
        full = tiles / 256.0 * v.rate * (double)blocks;
      } else {
        const double rounds = tiles / v.slots;
        full = (rounds > 1.0 ? (double)(int64_t)(rounds + 0.999999) : rounds) * (v.fix + v.rate * its);
        if (rounds > 1.0) one = 0.0;
      }
      return v.base + look + (one > full ? one : full);
    };
    // Grouped k, lengths unknown: between groups of one length and a quarter of them with
    // all of it. 2816 x 2048 of 8187 rows in 8 groups, us: even 57 by 256, 69 by 128; two
    // groups 54, 61; a single one 77, 61. 1024 x 1024 of 4096: 14.6, 11.0; 29, 19; 42, 26.
    double t = time((double)(tm * tn * groups), (a.K / groups + 127) / 128);
    if (groups > 1) {
      const int64_t few = groups / 4 > 1 ? groups / 4 : 1;
      t += time((double)(tm * tn * few), (a.K / few + 127) / 128);
    }
    if (i == 0 || t < least) {
      least = t;
      best = &v;
    }
  }
  return best;
}

static lc_status gemm_fp8_launch(const lc_gemm_fp8_args &a, hipStream_t s) {
  LC_TRY(check_gemm_fp8(a));
  if (a.M == 0) return LC_OK;
  const bool typed = a.epilogue == LC_EPI_STORE || a.epilogue == LC_EPI_RESIDUAL;
  Fp8P p{};
  p.A = static_cast<const uint8_t *>(a.A);
  p.B = static_cast<const uint8_t *>(a.B);
  p.sa = a.a_scale;
  p.sb = a.b_scale;
  p.C = a.C;
  p.R = a.R;
  p.goff = a.group_offsets;
  p.lda = a.lda;
  p.ldb = a.ldb;
  p.ldsa = a.ld_a_scale;
  p.ldsb = a.ld_b_scale;
  p.ldc = a.ldc;
  p.ldr = a.ldr;
  p.gstride_b = a.group_mode == LC_GROUP_ROWS ? a.group_stride_b : 0;
  p.gstride_sb = a.group_mode == LC_GROUP_ROWS ? a.group_stride_b_scale : 0;
  p.gstride_c = a.group_mode == LC_GROUP_K ? a.group_stride_c : 0;
  p.M = (int)a.M;
  p.N = (int)a.N;
  p.K = (int)a.K;
  p.ash = a.a_block_rows == 128 ? 7 : 0;
  p.bsh = a.b_block_rows == 128 ? 7 : 0;
  p.gmode = a.group_mode;
  p.ngroups = a.group_mode == LC_GROUP_NONE ? 1 : a.n_groups;
  p.goff_max = a.group_mode == LC_GROUP_ROWS ? p.M : p.K;
  p.epi = a.epilogue;
  p.c_dt = typed ? a.c_dtype : LC_FP32;
  p.r_dt = a.r_dtype;
  const bool f32 = p.c_dt != LC_BF16;  // summed by the bf16 instructions
  p.store16 = p.c_dt != LC_FP32 && a.epilogue == LC_EPI_STORE;
  const Fp8Tiling *v = pick(a, f32);
  if (v->tile == 16) return direct_launch(p, a, f32, s);
  return gemm_fp8_tile_launch(p, a, v->tile, v->deep, f32, s);
}

}  // namespace lc

extern "C" lc_status lc_gemm_fp8(const lc_gemm_fp8_args *args, void *stream) {
  if (!args) return lc::fail(LC_ERR_INVALID_ARG, "gemm fp8: null args");
  return lc::gemm_fp8_launch(*args, static_cast<hipStream_t>(stream));
}
