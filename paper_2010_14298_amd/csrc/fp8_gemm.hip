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

// Block tile BM x BN in eight waves of WM x WN.
template <int BM_, int BN_, int WM_, int WN_>
struct Fp8Tile {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_;
  static constexpr int WAVES_N = BN / WN, WAVES = (BM / WM) * WAVES_N, THREADS = WAVES * 64;
  static constexpr int IT = WM / 32, JT = WN / 32;
  static constexpr int HALF = (BM + BN) * 64;               // half a stage (64 along K) of codes, A then B
  static constexpr int A_INS = BM / 16 / WAVES, B_INS = BN / 16 / WAVES;  // 1 KB loads of a wave and half stage
  static constexpr int INS = A_INS + B_INS;
  static constexpr int E_SEGS = (BM + BN) / 64;             // 64-row runs of a stage's scale words
  static constexpr int E_INS = (E_SEGS + WAVES - 1) / WAVES;
  static constexpr int OUT_LD = WN + 8;                     // float row of the output staging
  static_assert(WAVES == 8 && A_INS * 16 * WAVES == BM && B_INS * 16 * WAVES == BN, "whole 1 KB blocks per wave");
  static_assert(32 * OUT_LD * 4 <= HALF / 2, "two waves' output strips in a half stage's LDS");
};

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
template <class T, class C, bool NT>
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
    T* const at = static_cast<T*>(p.C) + row * p.ldc + col;
    if (NT && col + V <= p.N) {
      typedef T vec __attribute__((ext_vector_type(V)));
      vec v;
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] = (T)o[i];
      __builtin_nontemporal_store(v, reinterpret_cast<vec*>(at));
    } else {
      store_part<T, V>(at, p.N - col, o);
    }
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

// A run of memory that waves load straight to LDS, at a 32-bit offset of the
// lane plus one of the wave.
struct Rows {
  __amdgpu_buffer_rsrc_t r;
  __device__ __forceinline__ explicit Rows(const uint8_t* base)
      : r(__builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(base), 0, -1, 0x00027000)) {}
  __device__ __forceinline__ void to_lds16(uint8_t* lds, int lane_off, int wave_off) const {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lmem_void*)lds, 16, lane_off, wave_off, 0, 0);
  }
  __device__ __forceinline__ void to_lds4(int* lds, int lane_off) const {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lmem_void*)lds, 4, lane_off, 0, 0, 0);
  }
};

// Waits until at most N of this wave's loads to LDS are under way, and until
// its LDS reads are done; then a block barrier.
template <int N>
__device__ __forceinline__ void wait_loads() {
  __builtin_amdgcn_s_waitcnt(0x3F70 | (N & 15) | ((N >> 4) << 14));
}
__device__ __forceinline__ void meet() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("" ::: "memory");
}

// The K loop works in half stages of 64 along K, each with a buffer of its
// own (two stages, four buffers), filled by direct loads to LDS.  Rows of 64
// bytes, the 16-byte chunk index XOR-ed with (r / 4) mod 4, so that the 16
// rows that are read at one chunk fall on distinct banks.
//
// Two waves share each SIMD.  One half of the waves runs a segment behind
// the other: while one wave of a SIMD feeds the matrix cores from registers,
// the other reads its next half stage from LDS and issues loads, and barriers
// keep them in step.  With segments s, s+1, .. the waves in front do
//   s: read (t, 0)   s+1: multiply (t, 0)   s+2: read (t, 1)   s+3: multiply (t, 1)
// and those behind the same one segment later.  A buffer is free when the
// waves behind have read it: half (t, 0) from s+2 on, where read (t, 1) issues
// the loads of (t + 2, 0); read (t + 1, 0) issues those of (t + 2, 1).  Loads
// have to be complete before the waves in front read them, so every wave
// waits for the half stage after next at the end of its read segment.
template <class T, class C, bool NT>
__global__ __launch_bounds__(C::THREADS) void fp8_gemm_kernel(Fp8GemmParams p) {
  // separate arrays, so that a pending load into one does not hold up reads of another
  __shared__ __attribute__((aligned(16))) uint8_t h00[C::HALF], h01[C::HALF], h10[C::HALF], h11[C::HALF];
  __shared__ int e0[C::BM + C::BN], e1[C::BM + C::BN];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / C::WAVES_N, wn = wave % C::WAVES_N;
  int64_t tm, tn;
  block_tile(blockIdx.x, (p.M + C::BM - 1) / C::BM, (p.N + C::BN - 1) / C::BN, tm, tn);
  const int64_t m0 = tm * C::BM, n0 = tn * C::BN;
  const int64_t pitch = fp8_pitch(p.K);
  const int nk = (int)fp8_blocks(p.K);
  // sources of this lane, as 32-bit offsets from the tile's first row; rows
  // past the edge read the last row, their outputs are never stored
  const Rows rowsA(p.A + m0 * pitch), rowsB(p.B + n0 * pitch);
  const int lastA = p.M - 1 - m0 < C::BM - 1 ? (int)(p.M - 1 - m0) : C::BM - 1;
  const int lastB = p.N - 1 - n0 < C::BN - 1 ? (int)(p.N - 1 - n0) : C::BN - 1;
  int src[C::INS];
#pragma unroll
  for (int i = 0; i < C::INS; ++i) {
    const bool a = i < C::A_INS;
    const int r = 16 * (a ? wave * C::A_INS + i : wave * C::B_INS + i - C::A_INS) + (lane >> 2);
    const int last = a ? lastA : lastB;
    src[i] = (r < last ? r : last) * (int)pitch + 16 * ((lane & 3) ^ ((r >> 2) & 3));
  }
  const uint8_t* ebase[C::E_INS];
  int64_t estep[C::E_INS];
  int esrc[C::E_INS], eseg[C::E_INS];
#pragma unroll
  for (int i = 0; i < C::E_INS; ++i) {
    eseg[i] = (wave + i * C::WAVES) % C::E_SEGS;  // fewer runs than waves: some load one twice
    const bool a = eseg[i] * 64 < C::BM;
    const int r = eseg[i] * 64 - (a ? 0 : C::BM) + lane, last = a ? lastA : lastB;
    ebase[i] = a ? p.eA + m0 * 4 : p.eB + n0 * 4;
    esrc[i] = 4 * (r < last ? r : last);
    estep[i] = (a ? p.M : p.N) * 4;
  }
  auto load_half = [&](uint8_t* d, int t, int kk) __attribute__((always_inline)) {
    const int ko = t * FP8_BLOCK + 64 * kk;
#pragma unroll
    for (int i = 0; i < C::INS; ++i) {
      const bool a = i < C::A_INS;
      uint8_t* const to = d + (a ? (wave * C::A_INS + i) * 1024 : C::BM * 64 + (wave * C::B_INS + i - C::A_INS) * 1024);
      (a ? rowsA : rowsB).to_lds16(to, src[i], ko);
    }
  };
  auto load_scales = [&](int* e, int t) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < C::E_INS; ++i)
      Rows(ebase[i] + (t >> 2) * estep[i]).to_lds4(e + eseg[i] * 64, esrc[i]);
  };
  v16f acc[C::IT][C::JT];
#pragma unroll
  for (int i = 0; i < C::IT; ++i)
#pragma unroll
    for (int j = 0; j < C::JT; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;
  const int lrow = lane & 31, half = lane >> 5;
  const int sw = (lrow >> 2) & 3;
  const int offA = (wm * C::WM + lrow) * 64, offB = C::BM * 64 + (wn * C::WN + lrow) * 64;
  const int c0 = 16 * ((2 * half) ^ sw), c1 = 16 * ((2 * half + 1) ^ sw);
  v8i a[C::IT], b[C::JT];
  int sa[C::IT], sb[C::JT];
  constexpr int N0 = C::INS + C::E_INS, N1 = C::INS;  // loads of a first and a second half stage
  auto read = [&](const uint8_t* st) __attribute__((always_inline)) {
    auto frag = [&](const uint8_t* q) __attribute__((always_inline)) {
      const v4i x = *reinterpret_cast<const v4i*>(q + c0);
      const v4i y = *reinterpret_cast<const v4i*>(q + c1);
      return v8i{x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
    };
#pragma unroll
    for (int i = 0; i < C::IT; ++i) a[i] = frag(st + offA + i * 32 * 64);
#pragma unroll
    for (int j = 0; j < C::JT; ++j) b[j] = frag(st + offB + j * 32 * 64);
  };
  auto multiply = [&]() __attribute__((always_inline)) {
    __builtin_amdgcn_s_setprio(1);
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int i = 0; i < C::IT; ++i)
#pragma unroll
        for (int j = 0; j < C::JT; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a[i], b[j], acc[i][j], 0, 0, 0, sa[i], 0, sb[j]);
    } else {
      float fa[C::IT], fb[C::JT];
#pragma unroll
      for (int i = 0; i < C::IT; ++i) fa[i] = scale_of(sa[i], 0);
#pragma unroll
      for (int j = 0; j < C::JT; ++j) fb[j] = scale_of(sb[j], 0);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        v8b wa[C::IT], wb[C::JT];
#pragma unroll
        for (int j = 0; j < C::JT; ++j) wb[j] = widen(b[j][2 * q], b[j][2 * q + 1], fb[j]);
#pragma unroll
        for (int i = 0; i < C::IT; ++i) wa[i] = widen(a[i][2 * q], a[i][2 * q + 1], fa[i]);
#pragma unroll
        for (int i = 0; i < C::IT; ++i)
#pragma unroll
          for (int j = 0; j < C::JT; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wa[i], wb[j], acc[i][j], 0, 0, 0);
      }
    }
    __builtin_amdgcn_s_setprio(0);
    // the products belong to this segment: keep the compiler from moving them past the barrier
#pragma unroll
    for (int i = 0; i < C::IT; ++i)
#pragma unroll
      for (int j = 0; j < C::JT; ++j) asm volatile("" : "+v"(acc[i][j]));
  };
  // `inner`: stages t + 1 and t + 2 exist (a constant: a load behind a branch
  // would make the compiler wait for all loads at the loop's head)
  auto stage = [&](auto inner, int t, const uint8_t* r0, const uint8_t* r1, const int* e, uint8_t* w0, uint8_t* w1,
                   int* we) __attribute__((always_inline)) {
    // read (t, 0): the buffer of (t + 1, 1) is free
    read(r0);
#pragma unroll
    for (int i = 0; i < C::IT; ++i) sa[i] = e[wm * C::WM + i * 32 + lrow] >> (8 * (t & 3));
#pragma unroll
    for (int j = 0; j < C::JT; ++j) sb[j] = e[C::BM + wn * C::WN + j * 32 + lrow] >> (8 * (t & 3));
    if (inner || t + 1 < nk) {
      load_half(w1, t + 1, 1);
      wait_loads<N0 + N1>();  // (t, 1) is there
    } else {
      wait_loads<0>();
    }
    __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
    meet();
    multiply();
    meet();
    // read (t, 1): the buffer of (t + 2, 0), this stage's first, is free
    read(r1);
    if (inner || t + 2 < nk) {
      load_half(w0, t + 2, 0);
      load_scales(we, t + 2);
      wait_loads<N0 + N1>();  // (t + 1, 0) is there
    } else {
      wait_loads<N1>();
    }
    __builtin_amdgcn_s_waitcnt(0xC07F);
    meet();
    multiply();
    meet();
  };
  load_half(h00, 0, 0);
  load_scales(e0, 0);
  load_half(h01, 0, 1);
  if (nk > 1) {
    load_half(h10, 1, 0);
    load_scales(e1, 1);
    wait_loads<N0 + N1>();
  } else {
    wait_loads<N1>();
  }
  meet();
  const bool behind = wave >= C::WAVES / 2;
  if (behind) meet();
  constexpr std::true_type inner{};
  constexpr std::false_type last{};
  int t = 0;
  for (; t + 3 < nk; t += 2) {
    stage(inner, t, h00, h01, e0, h00, h11, e0);
    stage(inner, t + 1, h10, h11, e1, h10, h01, e1);
  }
  stage(last, t, h00, h01, e0, h00, h11, e0);
  if (t + 1 < nk) stage(last, t + 1, h10, h11, e1, h10, h01, e1);
  if (t + 2 < nk) stage(last, t + 2, h00, h01, e0, h00, h11, e0);
  if (!behind) meet();
  __syncthreads();
  // a strip of 32 rows at a time through this wave's part of LDS, so that the
  // stores are whole lines
  uint8_t* const own = (wave < 4 ? (wave < 2 ? h00 : h01) : (wave < 6 ? h10 : h11)) + (wave & 1) * (C::HALF / 2);
  float* strip = reinterpret_cast<float*>(own);
#pragma unroll
  for (int i = 0; i < C::IT; ++i) {
#pragma unroll
    for (int j = 0; j < C::JT; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        strip[(8 * (r >> 2) + 4 * half + (r & 3)) * C::OUT_LD + j * 32 + lrow] = acc[i][j][r];
    __builtin_amdgcn_wave_barrier();
    store_strip<T, C, NT>(p, strip, m0 + wm * C::WM + i * 32, n0 + wn * C::WN);
    __builtin_amdgcn_wave_barrier();
  }
}

using Fp8Large = Fp8Tile<256, 256, 128, 64>;
using Fp8Mid = Fp8Tile<256, 128, 64, 64>;
using Fp8Small = Fp8Tile<128, 128, 64, 32>;

int64_t fp8_gemm_partials(int64_t, int64_t, int64_t) { return 0; }

template <class C>
static int64_t tiles_of(int64_t M, int64_t N) {
  return ((M + C::BM - 1) / C::BM) * ((N + C::BN - 1) / C::BN);
}

hipError_t launch_fp8_gemm(fqt_dtype type, const Fp8GemmParams& p, hipStream_t s) {
  return with_type(type, [&](auto e) {
    using T = decltype(e);
    auto go = [&](auto c) {
      using C = decltype(c);
      const int64_t tiles = tiles_of<C>(p.M, p.N);
      if (tiles > 0x3FFFFFFF) return hipErrorInvalidValue;
      // whole lines of outputs go past the caches (8192 x 4096 x 1024, bfloat16:
      // 46.8 us ordinary, 43.5 nontemporal; float32: 76.8, 72.0)
      const bool nt = (p.ldc * sizeof(T)) % 128 == 0 && ((uintptr_t)p.C & 127) == 0;
      if (nt)
        hipLaunchKernelGGL((fp8_gemm_kernel<T, C, true>), dim3((unsigned)tiles), dim3(C::THREADS), 0, s, p);
      else
        hipLaunchKernelGGL((fp8_gemm_kernel<T, C, false>), dim3((unsigned)tiles), dim3(C::THREADS), 0, s, p);
      return hipGetLastError();
    };
    if (tiles_of<Fp8Large>(p.M, p.N) >= 256) return go(Fp8Large{});
    return tiles_of<Fp8Mid>(p.M, p.N) >= 256 ? go(Fp8Mid{}) : go(Fp8Small{});
  });
}

}  // namespace fqt
