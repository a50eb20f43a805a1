// Products of 8-bit floating point operands with a power-of-two scale for
// each row and block of 128 along the contraction:
//
//   C[m, n] = sum over blocks b, k in b of A[m, k] 2^EA[m, b] B[n, k] 2^EB[n, b]
//
// Two ways through the matrix cores, by the output's type:
//   16-bit outputs  v_mfma_scale_f32_32x32x64_f8f6f4 on the codes as they are;
//     it applies both scales itself.  It drops the part of a product that lies
//     more than 13 bits below the largest product summed with it: 1.5e-5 to
//     7e-5 of the result (2-norm) against the output's own rounding of 1.7e-3.
//   float32 outputs  the codes are converted to bfloat16 with their scale
//     (v_cvt_scalef32_pk_bf16_fp8, exact) and go through
//     v_mfma_f32_32x32x16_bf16 at half the rate, which sums to 1.5e-7.
// The output is rounded once.
#include "train_kernels.h"

namespace fqt {

typedef float v16f __attribute__((ext_vector_type(16)));
typedef int v8i __attribute__((ext_vector_type(8)));
typedef int v4i __attribute__((ext_vector_type(4)));
typedef __bf16 v2b __attribute__((ext_vector_type(2)));
typedef __bf16 v8b __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(1))) void gmem_void;
typedef __attribute__((address_space(3))) void lmem_void;

// Block tile BM x BN, wave tile WM x WN, NS stages of 128 along K in LDS.
template <int BM_, int BN_, int WM_, int WN_, int NS_>
struct Fp8Tile {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, NS = NS_;
  static constexpr int WAVES_N = BN / WN, WAVES = (BM / WM) * WAVES_N, THREADS = WAVES * 64;
  static constexpr int IT = WM / 32, JT = WN / 32;
  static constexpr int CODES = (BM + BN) * FP8_BLOCK;       // a stage's codes, A then B
  static constexpr int STAGE = CODES + (BM + BN) * 4;       // and one word of scales a row
  static constexpr int A_INS = BM / 8 / WAVES, B_INS = BN / 8 / WAVES;  // 1 KB loads of a wave
  static constexpr int E_SEGS = (BM + BN) / 64;             // 64-row runs of scale words
  static constexpr int E_INS = (E_SEGS + WAVES - 1) / WAVES;
  static constexpr int OUT_LD = WN + 8;                     // float row of the output staging
  static constexpr int OUT = WAVES * 32 * OUT_LD * 4;
  static constexpr int LDS = NS * STAGE > OUT ? NS * STAGE : OUT;
  static_assert(A_INS * 8 * WAVES == BM && B_INS * 8 * WAVES == BN, "whole 1 KB blocks per wave");
};

// 16-byte slot of (row r, chunk c): rows of 128 bytes, chunk index XOR-ed with
// (r / 2) mod 8, so that 16 rows read at one chunk fall on distinct banks.
__device__ __forceinline__ int fslot(int r, int c) { return 8 * r + (c ^ ((r >> 1) & 7)); }

// Output tile of a block: each XCD (block id mod 8) takes a contiguous run of
// tiles, in groups of four tile rows.
__device__ __forceinline__ void block_tile(int64_t id, int64_t tm, int64_t tn, int64_t& m, int64_t& n) {
  const uint32_t tiles = (uint32_t)(tm * tn), q = tiles / 8;
  uint32_t t = (uint32_t)id;
  if (t < q * 8) t = (t % 8) * q + t / 8;
  const uint32_t per = 4 * (uint32_t)tn, first = t / per * 4, rem = t - first * (uint32_t)tn;
  const uint32_t left = (uint32_t)tm - first, rows = left < 4 ? left : 4;
  n = rem / rows;
  m = first + (rem - (uint32_t)n * rows);
}

// Stores a wave's 32-row strip of outputs that lies in LDS as float32.
template <class T, class C>
__device__ __forceinline__ void store_strip(const Fp8GemmParams& p, const float* strip, int64_t row0, int64_t col0) {
  constexpr int V = 16 / (int)sizeof(T), LANES = C::WN / V, ROWS = 64 / LANES;
  const int lane = threadIdx.x & 63, lr = lane / LANES, lc = (lane % LANES) * V;
#pragma unroll
  for (int r = 0; r < 32; r += ROWS) {
    const int64_t row = row0 + r + lr, col = col0 + lc;
    if (row >= p.M || col >= p.N) continue;
    float o[V];
#pragma unroll
    for (int i = 0; i < V; ++i) o[i] = strip[(r + lr) * C::OUT_LD + lc + i];
    if (p.relu) {
#pragma unroll
      for (int i = 0; i < V; ++i) o[i] = o[i] < 0.0f ? 0.0f : o[i];
    }
    if (p.mask) {
      float m[V];
      load_part<T, V>(static_cast<const T*>(p.mask) + row * p.ldmask + col, p.N - col, m);
#pragma unroll
      for (int i = 0; i < V; ++i) o[i] = m[i] > 0.0f ? o[i] : 0.0f;
    }
    store_part<T, V>(static_cast<T*>(p.C) + row * p.ldc + col, p.N - col, o);
  }
}

// Eight codes (two words) as bfloat16 times `scale`, a power of two: exact
// where the result is at least 2^-126, the smallest normal number.
__device__ __forceinline__ v8b widen(int w0, int w1, float scale) {
  const v2b a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, scale, false);
  const v2b b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, scale, true);
  const v2b c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, scale, false);
  const v2b d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, scale, true);
  return v8b{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
// 2^E of the scale byte `sh` bits up in w (byte 0: 2^-127, a subnormal).
__device__ __forceinline__ float scale_of(int w, int sh) {
  const uint32_t b = ((uint32_t)w >> sh) & 255u;
  return __uint_as_float(b ? b << 23 : 0x400000u);
}

template <class T, class C>
__global__ __launch_bounds__(C::THREADS) void fp8_gemm_kernel(Fp8GemmParams p) {
  __shared__ __attribute__((aligned(16))) uint8_t lds[C::LDS];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / C::WAVES_N, wn = wave % C::WAVES_N;
  int64_t tm, tn;
  block_tile(blockIdx.x, (p.M + C::BM - 1) / C::BM, (p.N + C::BN - 1) / C::BN, tm, tn);
  const int64_t m0 = tm * C::BM, n0 = tn * C::BN;
  const int64_t pitch = fp8_pitch(p.K), nk = fp8_blocks(p.K);
  // sources of this lane; rows past the edge read the last row, never stored
  const uint8_t* src[C::A_INS + C::B_INS];
#pragma unroll
  for (int i = 0; i < C::A_INS + C::B_INS; ++i) {
    const bool a = i < C::A_INS;
    const int r = 8 * (a ? wave * C::A_INS + i : wave * C::B_INS + i - C::A_INS) + (lane >> 3);
    const int64_t at = (a ? m0 : n0) + r, last = (a ? p.M : p.N) - 1;
    src[i] = (a ? p.A : p.B) + (at < last ? at : last) * pitch + 16 * ((lane & 7) ^ ((r >> 1) & 7));
  }
  const uint8_t* esrc[C::E_INS];
  int64_t estep[C::E_INS];
  int eseg[C::E_INS];
#pragma unroll
  for (int i = 0; i < C::E_INS; ++i) {
    eseg[i] = (wave + i * C::WAVES) % C::E_SEGS;  // fewer runs than waves: some load one twice
    const bool a = eseg[i] * 64 < C::BM;
    const int64_t at = (a ? m0 : n0 - C::BM) + eseg[i] * 64 + lane, last = (a ? p.M : p.N) - 1;
    esrc[i] = (a ? p.eA : p.eB) + (at < last ? at : last) * 4;
    estep[i] = (a ? p.M : p.N) * 4;
  }
  auto load = [&](int64_t t) __attribute__((always_inline)) {
    uint8_t* st = lds + (t % C::NS) * C::STAGE;
#pragma unroll
    for (int i = 0; i < C::A_INS + C::B_INS; ++i) {
      uint8_t* d = st + (i < C::A_INS ? (wave * C::A_INS + i) * 1024
                                      : C::BM * FP8_BLOCK + (wave * C::B_INS + i - C::A_INS) * 1024);
      __builtin_amdgcn_global_load_lds((gmem_void*)(src[i] + t * FP8_BLOCK), (lmem_void*)d, 16, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < C::E_INS; ++i)
      __builtin_amdgcn_global_load_lds((gmem_void*)(esrc[i] + (t >> 2) * estep[i]),
                                       (lmem_void*)(st + C::CODES + eseg[i] * 256), 4, 0, 0);
  };
  v16f acc[C::IT][C::JT];
#pragma unroll
  for (int i = 0; i < C::IT; ++i)
#pragma unroll
    for (int j = 0; j < C::JT; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;
  const int lrow = lane & 31, half = lane >> 5;
  load(0);
  for (int64_t t = 0; t < nk; ++t) {
    __syncthreads();  // waits for this wave's loads; and everyone is done with the other buffer
    if (t + 1 < nk) load(t + 1);
    const uint8_t* st = lds + (t % C::NS) * C::STAGE;
    const int* ea = reinterpret_cast<const int*>(st + C::CODES);
    int sa[C::IT], sb[C::JT];
#pragma unroll
    for (int i = 0; i < C::IT; ++i) sa[i] = ea[wm * C::WM + i * 32 + lrow] >> (8 * (t & 3));
#pragma unroll
    for (int j = 0; j < C::JT; ++j) sb[j] = ea[C::BM + wn * C::WN + j * 32 + lrow] >> (8 * (t & 3));
    float fa[C::IT], fb[C::JT];
#pragma unroll
    for (int i = 0; i < C::IT; ++i) fa[i] = scale_of(sa[i], 0);
#pragma unroll
    for (int j = 0; j < C::JT; ++j) fb[j] = scale_of(sb[j], 0);
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      v8i a[C::IT], b[C::JT];
      auto frag = [&](const uint8_t* base, int r) __attribute__((always_inline)) {
        const int c = 4 * kk + 2 * half;
        const v4i x = *reinterpret_cast<const v4i*>(base + 16 * fslot(r, c));
        const v4i y = *reinterpret_cast<const v4i*>(base + 16 * fslot(r, c + 1));
        return v8i{x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
      };
#pragma unroll
      for (int i = 0; i < C::IT; ++i) a[i] = frag(st, wm * C::WM + i * 32 + lrow);
#pragma unroll
      for (int j = 0; j < C::JT; ++j) b[j] = frag(st + C::BM * FP8_BLOCK, wn * C::WN + j * 32 + lrow);
      if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int i = 0; i < C::IT; ++i)
#pragma unroll
          for (int j = 0; j < C::JT; ++j)
            acc[i][j] =
                __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a[i], b[j], acc[i][j], 0, 0, 0, sa[i], 0, sb[j]);
      } else {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          v8b wa[C::IT], wb[C::JT];
#pragma unroll
          for (int i = 0; i < C::IT; ++i) wa[i] = widen(a[i][2 * q], a[i][2 * q + 1], fa[i]);
#pragma unroll
          for (int j = 0; j < C::JT; ++j) wb[j] = widen(b[j][2 * q], b[j][2 * q + 1], fb[j]);
#pragma unroll
          for (int i = 0; i < C::IT; ++i)
#pragma unroll
            for (int j = 0; j < C::JT; ++j)
              acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wa[i], wb[j], acc[i][j], 0, 0, 0);
        }
      }
    }
  }
  __syncthreads();
  // a strip of 32 rows at a time through this wave's part of LDS, so that the
  // stores are whole lines
  float* strip = reinterpret_cast<float*>(lds) + wave * 32 * C::OUT_LD;
#pragma unroll
  for (int i = 0; i < C::IT; ++i) {
#pragma unroll
    for (int j = 0; j < C::JT; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        strip[(8 * (r >> 2) + 4 * half + (r & 3)) * C::OUT_LD + j * 32 + lrow] = acc[i][j][r];
    __builtin_amdgcn_wave_barrier();
    store_strip<T, C>(p, strip, m0 + wm * C::WM + i * 32, n0 + wn * C::WN);
    __builtin_amdgcn_wave_barrier();
  }
}

using Fp8Small = Fp8Tile<128, 128, 64, 64, 2>;

int64_t fp8_gemm_partials(int64_t, int64_t, int64_t) { return 0; }

hipError_t launch_fp8_gemm(fqt_dtype type, const Fp8GemmParams& p, hipStream_t s) {
  return with_type(type, [&](auto e) {
    using T = decltype(e);
    using C = Fp8Small;
    const int64_t tiles = ((p.M + C::BM - 1) / C::BM) * ((p.N + C::BN - 1) / C::BN);
    if (tiles > 0x3FFFFFFF) return hipErrorInvalidValue;
    hipLaunchKernelGGL((fp8_gemm_kernel<T, C>), dim3((unsigned)tiles), dim3(C::THREADS), 0, s, p);
    return hipGetLastError();
  });
}

}  // namespace fqt
