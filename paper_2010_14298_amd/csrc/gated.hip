// Gated layer in 8-bit floating point, forward:
//
//   a = Q(X) W_gate^T,  b = Q(X) W_up^T,  H = act(a) b
//   d_gate = Q8(b act'(a)),  d_up = Q8(act(a))    (kept for the backward)
//
// The products' loops of fp8_loops.h over both halves of the weights at once;
// a and b stay in registers, so that of them nothing goes to memory but H and two
// bytes a hidden unit.
//
// 8192, 1024 -> 4096 bfloat16 with checkpoints (137 GFLOP, 168 MB): the call 145 us by
// itself, where a library product of the same size with bfloat16 operands and outputs,
// without codes, scales and activation, takes 127 - 130 in the same run.  In a trace of
// 90 calls one after another, under which the clock falls, quantizer 10.3 and product
// 154 on average (0.89 PFLOP/s), 135 at least (1.02).  Matrix instructions fill 47 % of the
// cycles, at a clock below 2 GHz; what is left between them is
// the conversions of the codes and each block's activations and stores.
// Serving: one token of 1024 -> 4096 (8.4 MB of weights) 4.6 us, 1.8 TB/s, 48 of
// 2048 -> 1001 float16 7.6 us: a launch, and the chain of load, quantize, multiply and
// the join of the waves' sums.
#include "fp8_loops.h"

namespace fqt {

template <bool SAVE>
struct GatedGemm : GatedGemmParams {
  static constexpr bool KEEP = SAVE;
};

// H and the checkpoints from parts of a and b in memory, [splits][M][2 hidden]: a
// thread four columns, eight threads a block of a checkpoint.
template <class T>
__global__ __launch_bounds__(256) void gated_finish_kernel(GatedGemmParams p, int splits) {
  const int64_t quads = kept_pitch(p.hidden) / 4, i = block_id() * 256 + threadIdx.x;
  if (i >= p.M * quads) return;  // eight threads of a block leave together
  const int64_t row = i / quads, col = (i - row * quads) * 4, n = p.hidden - col;
  float a[4] = {0.0f, 0.0f, 0.0f, 0.0f}, b[4] = {0.0f, 0.0f, 0.0f, 0.0f}, h[4], dg[4], du[4];
#pragma unroll 4
  for (int s = 0; s < splits; ++s) {
    const float* const at = p.part + (s * p.M + row) * p.N + col;
    float va[4], vb[4];
    load_part<float, 4>(at, n, va);
    load_part<float, 4>(at + p.hidden, n, vb);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      a[j] += va[j];
      b[j] += vb[j];
    }
  }
  with_act(p.act, [&](auto act) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float slope;
      activate<decltype(act)::value>(a[j], du[j], slope);
      h[j] = du[j] * b[j];
      dg[j] = slope * b[j];
      if (j >= n) dg[j] = du[j] = 0.0f;
    }
  });
  store_part<T, 4>(static_cast<T*>(p.C) + row * p.ldc + col, n, h);
  auto keep = [&](const Kept& k, const float (&v)[4]) {
    if (!k.q) return;
    uint32_t key = 0u;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t m = __float_as_uint(v[j]) & 0x7fffffffu;
      key = key > m ? key : m;
    }
    auto larger = [](uint32_t x, uint32_t y) { return x > y ? x : y; };
    key = larger(key, dpp<0xB1>(key));
    key = larger(key, dpp<0x4E>(key));
    key = Quad<float>::key(larger(key, dpp<0x141>(key)));
    const uint32_t byte = scale_bytes(key) & 0xffffu;
    const Quad<float> x{{v[0], v[1], v[2], v[3]}};
    const int64_t o = row * quads * 4 + col;
    *reinterpret_cast<uint32_t*>(k.q + o) = key >= NAN_KEY ? 0x7f7f7f7fu : x.row_codes(scale_up(byte));
    if (col % KEPT_BLOCK == 0) k.e[o / KEPT_BLOCK] = stored_byte(key, byte);
  };
  keep(p.gate, dg);
  keep(p.up, du);
}

// ---------------------------------------------------------------------------
// launches
// ---------------------------------------------------------------------------
// Few rows that keep nothing (serving) are read as they are, 16 a block, each of
// which quantizes them for itself and walks all of K; with more blocks or a longer K a
// quantizer in front and the tiles, in parts along K, are faster.  us in a graph,
// bfloat16, as they are / tiles: 1024 -> 4096 one row 3.9, 16 rows 4.5, 64 10.8 / 16.1,
// 96 15.6 / 16.0, 128 20 / 15; 2048 -> 1001 48 rows 7.0 / 20, 128 12.4 / 18.8; 4096 ->
// 4096 17 rows 18.9 / 24.5, 48 31 / 24; 48 rows -> 2048, two turns of the units, 4096 20.9 /
// 23.5, 6144 29.7 / 26.4, 8192 37.9 / 28.7; 48 rows -> 512 8192 19.8 / 25.2, 12288 28.1 /
// 26.8, 32768 69 / 37.  One row and 16, whose tiles wait for the weights of many hidden
// units: -> 256 12288 19.0 / 22.1 and 27.4 / 25.0, 16384 23.6 / 23.3 and 35.6 / 27.1, 32768
// 42.6 / 29.9 and 69 / 33; -> 1024 16384 24.8 / 25.9 and 36.4 / 31.6, 32768 44 / 34 and 69 /
// 38; -> 2048 20480 30.6 / 34.0 and 44.8 / 37.6, 32768 45 / 46 and 70 / 48; -> 4096 32768
// 53 / 73 and 72 / 78, 65536 110 / 155 and 144 / 156.  (float32 16 rows: -> 256 12288 36 / 26,
// 16384 47 / 27, -> 4096 32768 93 / 75; the workspace is asked for without a type.)
bool gated_rows_raw(int64_t M, int64_t hidden, int64_t K) {
  const int64_t nk = fp8_blocks(K), blocks = (hidden + 15) / 16, turns = ((M + 15) / 16 * blocks + 255) / 256;
  if (M <= 16) return nk <= 96 + blocks || blocks >= 192;
  return M <= 128 && turns * nk < 40 + nk + nk / 2 && turns * nk <= 96;
}
// The tiles of both halves of B, as if they were columns.  A pass over the parts
// gates them too, and the call's host time pays for its launch.  Where the small
// tiles leave half of the units without one they are halved, 64 rows each, 0.63 us a
// stage of 128; whole / half, in a graph with checkpoints, us: 250, 2048 -> 1001
// float32 23.9 / 19.4 (in two parts 22.8), 256, 1024 -> 2048 float16 18.1 / 15.2, 2048,
// 256 -> 512 bfloat16 13.3 / 12.1; in parts / half 250, 2944 -> 1024
// bfloat16 25.1 / 22.3.  Longer ones stay in parts.
// The order of a row's sums is the form's: a wave holds both projections of 32 hidden
// units, 64 columns, so that these tiles, for every type, divide K between two groups
// of four waves (the plain layer's of 16-bit outputs, 32 columns a wave, need not).
typedef PipeTile<64, 128, 32, 64, 2, 4> HalfTile;
static bool halves(const Fp8Plan& plan, int64_t M, int64_t hidden) {
  return plan.tile == Fp8Plan::SMALL && plan.splits == 1 && tiles_of(M, hidden, SmallTile::BM, SmallTile::BN / 2) <= 128;
}
static Fp8Plan gated_plan(int64_t M, int64_t hidden, int64_t K) {
  const int64_t nk = fp8_blocks(K);
  const Fp8Plan plan = fp8_plan(M, 2 * hidden, K, 8.0), whole{Fp8Plan::SMALL, 1, (int)nk};
  return halves(whole, M, hidden) && (double)nk * 0.63 + 4.0 < fp8_plan_time(M, 2 * hidden, plan, 8.0) ? whole : plan;
}
int64_t gated_partials(int64_t M, int64_t hidden, int64_t K) {
  const int64_t s = gated_plan(M, hidden, K).splits;
  return s > 1 ? s * M * 2 * hidden : 0;
}

template <class T, bool SAVE>
static hipError_t gated_tiles(const GatedGemm<SAVE>& p, const Fp8Plan& plan, hipStream_t s) {
  auto tiles = [&](auto c) {
    using C = decltype(c);
    return tiles_of(p.M, p.hidden, C::BM, C::BN / 2);
  };
  const int64_t blocks = plan.tile == Fp8Plan::LARGE ? tiles(LargeTile{}) : plan.tile == Fp8Plan::MID ? tiles(MidTile{}) : tiles(SmallTile{});
  if (blocks > 0x3FFFFF) return hipErrorInvalidValue;  // and twice as many of two a unit
  auto go = [&](auto kernel, int64_t grid, auto... more) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(512), 0, s, p, more...);
    return hipGetLastError();
  };
  if (plan.tile == Fp8Plan::LARGE) {
    // us, 8192 tokens, 4096 hidden units, bfloat16, two blocks a unit / 256 x 256, with checkpoints (without): 512 wide
    // 90 / 98 (70 / 74), 1024 139 / 142 (119 / 119), 2048 238 / 230 (217 / 202), 8192 863 / 798 (826 / 758)
    if (plan.chunk <= 8) {
      hipLaunchKernelGGL((fp8_gemm_pair_kernel<T, GatedGemm<SAVE>>), dim3((unsigned)tiles(PairTile{})),
                         dim3(PairTile::THREADS), 0, s, p);
      return hipGetLastError();
    }
    return go(fp8_gemm_large_kernel<T, false, false, GatedGemm<SAVE>>, blocks);
  }
  if (halves(plan, p.M, p.hidden))
    return go(fp8_gemm_pipe_kernel<T, HalfTile, false, false, GatedGemm<SAVE>>, tiles(HalfTile{}), plan.chunk);
  if (plan.tile == Fp8Plan::MID)
    return go(fp8_gemm_pipe_kernel<T, MidTile, false, false, GatedGemm<SAVE>>, blocks, plan.chunk);
  return go(fp8_gemm_pipe_kernel<T, SmallTile, false, false, GatedGemm<SAVE>>, blocks, plan.chunk);
}

hipError_t launch_gated_gemm(fqt_dtype type, const GatedGemmParams& params, const void* x, int64_t ldx, hipStream_t s) {
  return with_type(type, [&](auto e) {
    using T = decltype(e);
    if (!params.gate.q && !params.up.q && gated_rows_raw(params.M, params.hidden, params.K)) {
      dim3 grid = grid_of((params.hidden + 15) / 16, 64 * 16);
      grid.z = (unsigned)((params.M + 15) / 16);
      const T* const rows = static_cast<const T*>(x);
      if constexpr (sizeof(T) == 2) {  // float32 rows do not fit the registers of sixteen waves
        if (fp8_blocks(params.K) > 8) {
          hipLaunchKernelGGL((gated_rows_kernel<T, 16>), grid, dim3(64 * 16), 0, s, params, rows, ldx);
          return hipGetLastError();
        }
      }
      hipLaunchKernelGGL((gated_rows_kernel<T, 8>), grid, dim3(64 * 8), 0, s, params, rows, ldx);
      return hipGetLastError();
    }
    const Fp8Plan plan = gated_plan(params.M, params.hidden, params.K);
    if (plan.splits > 1) {
      const hipError_t err = launch_fp8_parts(params, plan, s);
      if (err != hipSuccess) return err;
      const int64_t threads = params.M * (kept_pitch(params.hidden) / 4);
      hipLaunchKernelGGL((gated_finish_kernel<T>), grid_of((threads + 255) / 256, 256), dim3(256), 0, s, params, plan.splits);
      return hipGetLastError();
    }
    return params.gate.q || params.up.q ? gated_tiles<T, true>(GatedGemm<true>{params}, plan, s)
                                        : gated_tiles<T, false>(GatedGemm<false>{params}, plan, s);
  });
}

}  // namespace fqt
