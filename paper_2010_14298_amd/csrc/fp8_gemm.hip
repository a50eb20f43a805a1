// Products of 8-bit floating point operands with a power-of-two scale for
// each row and block of 128 along the contraction:
//
//   C[m, n] = sum over blocks b, k in b of A[m, k] 2^EA[m, b] B[n, k] 2^EB[n, b]
//
// The codes are converted to bfloat16 with their scale
// (v_cvt_scalef32_pk_bf16_fp8, exact) and go through v_mfma_f32_32x32x16_bf16,
// whose sums are float32: 2e-8 to 1.5e-7 of the result (2-norm).  The output is
// rounded once.  The matrix instructions that take the codes as they are
// (v_mfma_scale_f32_32x32x64_f8f6f4 and the plain ones) run at twice the rate,
// but they drop the part of a product that lies more than 13 bits below the
// largest product summed with it: 65536 - 65536 + 4 gives 0.  That loses 1.5e-5
// (normal data) to 7e-5 (one large element a block) of the result, and all of
// one that is left over from large products that cancel, so no output takes
// them: 8192 x 4096 x 1024 with bfloat16 outputs was 43 us with them, 66 without.
//
// Back to back on changing operands, us (PFLOP/s), M x N x K, and a library
// product of bfloat16 operands and outputs (no scales) in the same run:
//                        bfloat16 outputs   float32 outputs   library
//   8192 x 8192 x 8192      758 (1.45)         782 (1.41)        695
//   8192 x 4096 x 1024       64 (1.07)          78 (0.88)         64
//   8192 x 1024 x 4096       63 (1.08)          61 (1.14)         61
//   4096 x 1024 x 8192       68 (1.00)          62 (1.11)         67
// 8192 x 4096 x 1024 waits for the stores of its last tiles, which all units issue
// at the same time.  In 4096 x 1024 x 8192 (float32) matrix instructions fill 57 %
// of the cycles at a clock of 1.8 GHz; without the conversions it is no faster.
#include "fp8_loops.h"

namespace fqt {

// The parts of a split product added in order, with the product's epilogue.
template <class T>
__device__ __forceinline__ void split_sum(const Fp8GemmParams& p, int splits, uint32_t block) {
  const int64_t quads = (p.N + 3) / 4, i = (int64_t)block * 256 + threadIdx.x;
  if (i >= p.M * quads) return;
  const int64_t row = i / quads, col = i % quads * 4, n = p.N - col;
  float o[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
  for (int s = 0; s < splits; ++s) {
    float v[4];
    load_part<float, 4>(p.part + (s * p.M + row) * p.N + col, n, v);
#pragma unroll
    for (int j = 0; j < 4; ++j) o[j] += v[j];
  }
  if (p.relu) {
#pragma unroll
    for (int j = 0; j < 4; ++j) o[j] = o[j] < 0.0f ? 0.0f : o[j];
  }
  if (p.mask) {
    float m[4];
    load_part<T, 4>(static_cast<const T*>(p.mask) + row * p.ldmask + col, n, m);
#pragma unroll
    for (int j = 0; j < 4; ++j) o[j] = m[j] > 0.0f ? o[j] : 0.0f;
  }
  store_part<T, 4>(static_cast<T*>(p.C) + row * p.ldc + col, n, o);
}
template <class T>
__global__ __launch_bounds__(256) void fp8_split_sum_kernel(Fp8GemmParams p, int splits) {
  split_sum<T>(p, splits, blockIdx.x);
}

// Two products that do not depend on each other, a with float32 outputs and b, tile
// by tile in one launch: the units that one of them leaves idle work on the other.
// Half of K a wave whatever the type: the sums' order is the float32 products'.
template <class T, bool NT>
__global__ __launch_bounds__(512) void fp8_two_tiles_kernel(Fp8GemmParams a, Fp8GemmParams b, int nk_a, int nk_b,
                                                            uint32_t first, int second_is_b) {
  const bool early = blockIdx.x < first, is_b = early != (second_is_b != 0);
  const Fp8GemmParams p = is_b ? b : a;
  pipe_tile<float, SmallTile, false, NT, Fp8GemmParams, T>(p, is_b ? nk_b : nk_a, early ? blockIdx.x : blockIdx.x - first, 0, is_b);
}
// Their parts, and the sums of these, in one launch each.
__global__ __launch_bounds__(512) void fp8_two_parts_kernel(Fp8GemmParams a, Fp8GemmParams b, int chunk_a, int chunk_b,
                                                            uint32_t tiles_a, uint32_t blocks_a, uint32_t tiles_b) {
  const bool first = blockIdx.x < blocks_a;
  const uint32_t id = first ? blockIdx.x : blockIdx.x - blocks_a, tiles = first ? tiles_a : tiles_b;
  const Fp8GemmParams p = first ? a : b;
  pipe_tile<float, SmallTile, true, false, Fp8GemmParams>(p, first ? chunk_a : chunk_b, id % tiles, id / tiles);
}
template <class T>
__global__ __launch_bounds__(256) void fp8_two_sums_kernel(Fp8GemmParams a, Fp8GemmParams b, int splits_a, int splits_b,
                                                           uint32_t blocks_a) {
  if (blockIdx.x < blocks_a)
    split_sum<float>(a, splits_a, blockIdx.x);
  else
    split_sum<T>(b, splits_b, blockIdx.x - blocks_a);
}

// ---------------------------------------------------------------------------
// launches
// ---------------------------------------------------------------------------
// Which tile, and for small tiles into how many parts along K the product is
// split: the least estimated time of turns x (stages x c + t0), turns the
// tiles (times parts) over 256 units of one block each, plus the pass that adds
// the parts.  Measured on one product a turn (us a stage of 128): small 0.94
// (4096 x 1024 x 8192), mid 1.77 (8192 x 1024 x 4096), large 3.3 (4096 x 4096 x
// 4096).
// Every product with each tile, us, large / mid / small, the choice first:
//   8192 x 4096 x 1024 bfloat16  large 64     (67 / 83 / 101)
//   8192 x 1024 x 4096 bfloat16  mid   63     (83 / 63 / 76)
//   4096 x 1024 x 8192 float32   small 65     (145 / 87 / 64)
//   3001 x 1024 x 4096 float32   small 32     (78 / 46 / 32)
//   250 x 1001 x 2048 float32    split 13.4   (45.6 / 25.8 / 16.6)
//   130 x 260 x 8192 float32     split 15.6   (142 / 82 / 48.7)
Fp8Plan fp8_plan(int64_t M, int64_t N, int64_t K, double pass) {
  using Plan = Fp8Plan;
  const int64_t nk = fp8_blocks(K);
  const double c[3] = {0.94, 1.77, 3.3}, t0[3] = {4.0, 5.0, 8.0};
  auto turns = [](int64_t blocks) { return (double)((blocks + 255) / 256); };
  const int64_t small = tiles_of(M, N, SmallTile::BM, SmallTile::BN);
  Plan best{Plan::LARGE, 1, (int)nk};
  double least = turns(tiles_of(M, N, LargeTile::BM, LargeTile::BN)) * ((double)nk * c[2] + t0[2]);
  const double mid = turns(tiles_of(M, N, MidTile::BM, MidTile::BN)) * ((double)nk * c[1] + t0[1]);
  if (mid < least) {
    least = mid;
    best.tile = Plan::MID;
  }
  for (int s : {1, 2, 3, 4, 6, 8, 12, 16}) {
    const int64_t chunk = (nk + s - 1) / s, parts = (nk + chunk - 1) / chunk;
    if (parts != s) continue;
    double t = turns(small * s) * ((double)chunk * c[0] + t0[0]);
    if (s > 1) t += pass + (double)(M * N) * 8.0 * s / 4.0e6;  // written and read at about 4 TB/s
    if (t < least) {
      least = t;
      best = Plan{Plan::SMALL, s, (int)chunk};
    }
  }
  return best;
}

// Up to 64 rows stream the weights (fp8_rows_kernel): 17 x 4096 x 1024 bfloat16
// 3.6 us, in small tiles 10.5; 64 x 4096 x 1024 5.1, 11.1; 64 x 1024 x 4096 float32
// 12.2, 14.1.  Up to 16 rows are quantized there as well: 1024 -> 4096 bfloat16, one
// row 4.0 us, 7.1 with a quantizer's launch before it, 16 rows 4.7, 8.5; 16 rows
// of 4096 -> 1024 11.2, 11.4.
constexpr int64_t ROWS_MAX = 64, ROWS_RAW_MAX = 16;
bool fp8_rows_raw(int64_t M) { return M <= ROWS_RAW_MAX; }

// Blocks of the large tile that stay for several: more whole tiles of columns
// than units, an even number of stages, no mask, outputs in whole lines.
static bool several_tiles(const Fp8Plan& plan, int64_t M, int64_t N, bool masked, bool lines) {
  return plan.tile == Fp8Plan::LARGE && lines && !masked && tiles_of(M, N, LargeTile::BM, LargeTile::BN) > 256 &&
         N % LargeTile::BN == 0 && plan.chunk % 2 == 0 && plan.chunk >= 4;
}

fqt_fp8_form fp8_gemm_form(int64_t M, int64_t N, int64_t K, bool masked, bool lines) {
  if (M <= ROWS_MAX) return FQT_FP8_ROWS;
  const Fp8Plan plan = fp8_plan(M, N, K);
  switch (plan.tile) {
    case Fp8Plan::SMALL: return plan.splits > 1 ? FQT_FP8_PARTS : FQT_FP8_SMALL;
    case Fp8Plan::MID: return FQT_FP8_MIDDLE;
    case Fp8Plan::LARGE: break;
  }
  return several_tiles(plan, M, N, masked, lines) ? FQT_FP8_SEVERAL : FQT_FP8_LARGE;
}

int64_t fp8_gemm_partials(int64_t M, int64_t N, int64_t K) {
  if (M <= ROWS_MAX) return 0;
  const int64_t s = fp8_plan(M, N, K).splits;
  return s > 1 ? s * M * N : 0;
}

hipError_t launch_fp8_rows(fqt_dtype type, const Fp8GemmParams& p, const void* x, int64_t ldx, hipStream_t s) {
  return with_type(type, [&](auto e) {
    using T = decltype(e);
    const int64_t blocks = (p.N + 15) / 16;
    if (p.M > (x ? ROWS_RAW_MAX : ROWS_MAX)) return hipErrorInvalidValue;
    auto go = [&](auto kernel) {
      hipLaunchKernelGGL(kernel, grid_of(blocks, 64 * ROW_WAVES), dim3(64 * ROW_WAVES), 0, s, p, x, ldx);
      return hipGetLastError();
    };
    if (x) return go(fp8_rows_kernel<T, T, 1>);
    if (p.M <= 16) return go(fp8_rows_kernel<T, void, 1>);
    return p.M <= 32 ? go(fp8_rows_kernel<T, void, 2>) : go(fp8_rows_kernel<T, void, 4>);
  });
}

hipError_t launch_fp8_parts(const Fp8GemmParams& p, const Fp8Plan& plan, hipStream_t s) {
  const int64_t blocks = tiles_of(p.M, p.N, SmallTile::BM, SmallTile::BN);
  if (blocks > 0x7FFFFF) return hipErrorInvalidValue;
  hipLaunchKernelGGL((fp8_gemm_pipe_kernel<float, SmallTile, true, false>), dim3((unsigned)blocks, (unsigned)plan.splits),
                     dim3(512), 0, s, p, plan.chunk);
  return hipGetLastError();
}

hipError_t launch_fp8_gemm(fqt_dtype type, const Fp8GemmParams& p, hipStream_t s) {
  if (p.M <= ROWS_MAX) return launch_fp8_rows(type, p, nullptr, 0, s);
  return with_type(type, [&](auto e) {
    using T = decltype(e);
    // Whole lines of outputs of one tile a block go past the caches.  Ordinary /
    // nontemporal, with the pass that reads them next, us: bfloat16 and a quantizer
    // 8192 x 1024 x 4096 74.4 / 74.4, 2048 x 4096 x 1024 33.0 / 31.7; float32 and a norm
    // 4096 x 1024 x 8192 76.8 / 74.8, 3001 x 4096 x 4096 119 / 115, 3001 x 4096 x 1024
    // 51.1 / 47.9.
    const bool nt = (p.ldc * sizeof(T)) % 128 == 0 && ((uintptr_t)p.C & 127) == 0;
    const Fp8Plan plan = fp8_plan(p.M, p.N, p.K);
    auto tiles = [&](auto c) {
      using C = decltype(c);
      return tiles_of(p.M, p.N, C::BM, C::BN);
    };
    const int64_t blocks = plan.tile == Fp8Plan::LARGE ? tiles(LargeTile{}) : plan.tile == Fp8Plan::MID ? tiles(MidTile{}) : tiles(SmallTile{});
    if (blocks > 0x7FFFFF) return hipErrorInvalidValue;  // 2^32 threads, 2^37 outputs
    int64_t grid = blocks;
    auto go = [&](auto kernel, auto... more) {
      hipLaunchKernelGGL(kernel, dim3((unsigned)grid, (unsigned)plan.splits), dim3(512), 0, s, p, more...);
      return hipGetLastError();
    };
    if (plan.tile == Fp8Plan::LARGE) {
      if (several_tiles(plan, p.M, p.N, p.mask != nullptr, nt)) {
        grid = 256;  // one block a unit
        return go(fp8_gemm_large_kernel<T, true, true>);
      }
      return nt ? go(fp8_gemm_large_kernel<T, true, false>) : go(fp8_gemm_large_kernel<T, false, false>);
    }
    if (plan.tile == Fp8Plan::MID)
      return nt ? go(fp8_gemm_pipe_kernel<T, MidTile, false, true>, plan.chunk)
                : go(fp8_gemm_pipe_kernel<T, MidTile, false, false>, plan.chunk);
    using Small = std::conditional_t<sizeof(T) == 2, SmallTile16, SmallTile>;
    if (plan.splits == 1)
      return nt ? go(fp8_gemm_pipe_kernel<T, Small, false, true>, plan.chunk)
                : go(fp8_gemm_pipe_kernel<T, Small, false, false>, plan.chunk);
    const hipError_t err = launch_fp8_parts(p, plan, s);
    if (err != hipSuccess) return err;
    const int64_t quads = p.M * ((p.N + 3) / 4);
    hipLaunchKernelGGL((fp8_split_sum_kernel<T>), dim3((unsigned)((quads + 255) / 256)), dim3(256), 0, s, p, plan.splits);
    return hipGetLastError();
  });
}

bool fp8_two_at_once(int64_t Ma, int64_t Na, int64_t Ka, int64_t Mb, int64_t Nb, int64_t Kb) {
  return Ma > ROWS_MAX && Mb > ROWS_MAX && fp8_plan(Ma, Na, Ka).splits > 1 && fp8_plan(Mb, Nb, Kb).splits > 1;
}

double fp8_plan_time(int64_t M, int64_t N, const Fp8Plan& plan, double pass) {
  const bool large = plan.tile == Fp8Plan::LARGE, mid = plan.tile == Fp8Plan::MID;
  const double c = large ? 3.3 : mid ? 1.77 : 0.94, t0 = large ? 8.0 : mid ? 5.0 : 4.0;
  const int64_t tiles = tiles_of(M, N, mid || large ? 256 : 128, large ? 256 : 128) * plan.splits;
  return (double)((tiles + 255) / 256) * (plan.chunk * c + t0) +
         (plan.splits > 1 ? pass + (double)(M * N) * 8.0 * plan.splits / 4.0e6 : 0.0);
}

hipError_t launch_fp8_two(fqt_dtype type, const Fp8GemmParams& a, const Fp8GemmParams& b, bool any_order, hipStream_t s) {
  if (!fp8_two_at_once(a.M, a.N, a.K, b.M, b.N, b.K)) {
    if (any_order && a.M > ROWS_MAX && b.M > ROWS_MAX) {
      // The tiles of the longer contraction first, and half of one of the shorter
      // behind the last of them.  Together / apart, whole backward, us: bfloat16 2048,
      // 1024 -> 1024 32 / 47.5, 700, 2048 -> 1500 42 / 50, 3001, 1024 -> 2730 112 / 121
      // (float32 103 / 110), 2048, 1024 -> 4096 101 / 100; where one of the longer tiles
      // takes as long as all the rest, apart: 1024, 1024 -> 4096 70 / 63.
      const int nk_a = (int)fp8_blocks(a.K), nk_b = (int)fp8_blocks(b.K);
      const int64_t ta = tiles_of(a.M, a.N, SmallTile::BM, SmallTile::BN), tb = tiles_of(b.M, b.N, SmallTile::BM, SmallTile::BN);
      const double one_a = nk_a * 0.94 + 4.0, one_b = nk_b * 0.94 + 4.0;
      const double shorter = one_a < one_b ? one_a : one_b, longer = one_a < one_b ? one_b : one_a;
      double both = ((double)ta * one_a + (double)tb * one_b) / 256.0 + 0.5 * shorter;
      if (both < longer + 4.0) both = longer + 4.0;
      const double apart = fp8_plan_time(a.M, a.N, fp8_plan(a.M, a.N, a.K)) + fp8_plan_time(b.M, b.N, fp8_plan(b.M, b.N, b.K));
      if (both < apart && ta + tb <= 0x7FFFFF) {
        const bool b_first = nk_b >= nk_a;
        return with_type(type, [&](auto e) {
          using T = decltype(e);
          const bool nt = ((uintptr_t)a.C & 127) == 0 && ((uintptr_t)b.C & 127) == 0 && a.ldc * 4 % 128 == 0 &&
                          b.ldc * sizeof(T) % 128 == 0;
          auto go = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, dim3((unsigned)(ta + tb)), dim3(512), 0, s, a, b, nk_a, nk_b,
                               (uint32_t)(b_first ? tb : ta), (int)!b_first);
            return hipGetLastError();
          };
          return nt ? go(fp8_two_tiles_kernel<T, true>) : go(fp8_two_tiles_kernel<T, false>);
        });
      }
    }
    const hipError_t err = launch_fp8_gemm(FQT_F32, a, s);
    return err == hipSuccess ? launch_fp8_gemm(type, b, s) : err;
  }
  const Fp8Plan pa = fp8_plan(a.M, a.N, a.K), pb = fp8_plan(b.M, b.N, b.K);
  const int64_t ta = tiles_of(a.M, a.N, SmallTile::BM, SmallTile::BN), tb = tiles_of(b.M, b.N, SmallTile::BM, SmallTile::BN);
  const int64_t blocks = ta * pa.splits + tb * pb.splits;
  const int64_t qa = (a.M * ((a.N + 3) / 4) + 255) / 256, qb = (b.M * ((b.N + 3) / 4) + 255) / 256;
  if (blocks > 0x7FFFFF || qa + qb > 0xFFFFFF) return hipErrorInvalidValue;
  hipLaunchKernelGGL(fp8_two_parts_kernel, dim3((unsigned)blocks), dim3(512), 0, s, a, b, pa.chunk, pb.chunk, (uint32_t)ta,
                     (uint32_t)(ta * pa.splits), (uint32_t)tb);
  hipError_t err = hipGetLastError();
  if (err != hipSuccess) return err;
  return with_type(type, [&](auto e) {
    hipLaunchKernelGGL((fp8_two_sums_kernel<decltype(e)>), dim3((unsigned)(qa + qb)), dim3(256), 0, s, a, b, pa.splits,
                       pb.splits, (uint32_t)qa);
    return hipGetLastError();
  });
}

}  // namespace fqt
