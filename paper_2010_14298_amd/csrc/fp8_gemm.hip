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
#include "fp8_codes.h"

namespace fqt {

typedef float v16f __attribute__((ext_vector_type(16)));
typedef int v8i __attribute__((ext_vector_type(8)));
typedef int v4i __attribute__((ext_vector_type(4)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef __bf16 v2b __attribute__((ext_vector_type(2)));
typedef __bf16 v8b __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(1))) void gmem_void;
typedef __attribute__((address_space(3))) void lmem_void;

// The large tile: 256 x 256 in eight waves of 128 x 64.
struct LargeTile {
  static constexpr int BM = 256, BN = 256, WM = 128, WN = 64;
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

// The mask of a wave's 32-row strip of outputs, as it lies in memory.  Inside C
// all its loads are under way at once, ahead of the strip's way through LDS
// (8192 x 4096 x 1024 float32 103 us, 117 with the loads one by one as at the edges).
template <class T, int WN>
struct StripMask {
  static constexpr int V = 16 / (int)sizeof(T), LANES = WN / V, ROWS = 64 / LANES;
  typename Packed<T, V>::type v[32 / ROWS];
  bool whole;
  __device__ __forceinline__ StripMask(const Fp8GemmParams& p, int64_t row0, int64_t col0)
      : whole(p.mask && row0 + 32 <= p.M && col0 + WN <= p.N) {
    if (!whole) return;
    const int lane = threadIdx.x & 63;
    const T* at = static_cast<const T*>(p.mask) + (row0 + lane / LANES) * p.ldmask + col0 + lane % LANES * V;
#pragma unroll
    for (int i = 0; i < 32 / ROWS; ++i) v[i] = *reinterpret_cast<const typename Packed<T, V>::type*>(at + i * ROWS * p.ldmask);
  }
};

// Stores a wave's 32-row strip of outputs that lies in LDS as float32.
template <class T, int WN, int OUT_LD, bool NT>
__device__ __forceinline__ void store_strip(const Fp8GemmParams& p, const float* strip, const StripMask<T, WN>& mask,
                                            int64_t row0, int64_t col0) {
  constexpr int V = 16 / (int)sizeof(T), LANES = WN / V, ROWS = 64 / LANES;
  const int lane = threadIdx.x & 63, lr = lane / LANES, lc = (lane % LANES) * V;
#pragma unroll
  for (int r = 0; r < 32; r += ROWS) {
    const int64_t row = row0 + r + lr, col = col0 + lc;
    if (row >= p.M || col >= p.N) continue;
    float o[V];
#pragma unroll
    for (int i = 0; i < V; ++i) o[i] = strip[(r + lr) * OUT_LD + lc + i];
    if (p.relu) {
#pragma unroll
      for (int i = 0; i < V; ++i) o[i] = o[i] < 0.0f ? 0.0f : o[i];
    }
    if (p.mask) {
      float m[V];
      if (mask.whole) {
#pragma unroll
        for (int i = 0; i < V; ++i) m[i] = (float)mask.v[r / ROWS][i];
      } else {
        load_part<T, V>(static_cast<const T*>(p.mask) + row * p.ldmask + col, p.N - col, m);
      }
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

// Eight codes (two words) as bfloat16 times `scale`, a power of two: exact for
// scales from 2^-124 on; below, codes become multiples of 2^-133, bfloat16's
// smallest step.
__device__ __forceinline__ v8b widen(int w0, int w1, float scale) {
  const v2b a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, scale, false);
  const v2b b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, scale, true);
  const v2b c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, scale, false);
  const v2b d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, scale, true);
  return v8b{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
// 2^E of the scale byte in w's low bits (byte 0: 2^-127, a subnormal).
__device__ __forceinline__ float scale_of(int w) {
  const uint32_t b = (uint32_t)w & 255u;
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

// Instruction order of a widened multiply segment: QS steps of MF matrix
// instructions, whose operands take CV conversions each.  The first step's
// conversions go in front, the next step's between the matrix instructions,
// in the 32 cycles that each of those keeps the matrix cores busy.
template <int QS, int MF, int CV>
__device__ __forceinline__ void interleave() {
  __builtin_amdgcn_sched_group_barrier(0x2, CV, 0);  // VALU
#pragma unroll
  for (int q = 0; q < QS; ++q)
#pragma unroll
    for (int m = 0; m < MF; ++m) {
      __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);  // MFMA
      if (q + 1 < QS) __builtin_amdgcn_sched_group_barrier(0x2, CV / MF, 0);
    }
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
//
// RUN: blocks stay for several tiles (no mask, whole tiles of columns, an even
// number of stages, at least four).  The next tile's first two stages
// are on their way before this one's outputs are stored, and loads behind the
// stores are first waited for four segments later.  The load counter counts
// stores as well, in the order of issue, so until then the waits allow for
// STORES of them (another access in between only makes them stricter).  One block a
// tile / several, with the pass that reads the outputs next, us: bfloat16 8192 x
// 4096 x 1024 98 / 88, 8000 x 4096 x 1024 97 / 87, 16384 x 4096 x 512 144 / 123,
// 5120 x 5120 x 1024 86 / 74, 8192 x 8192 x 8192 840 / 813, 6144 x 4096 x 1024
// (one and a half tiles a unit) 84 / 83; float32 8192 x 4096 x 1024 108 / 104, 4096 x
// 8192 x 1024 120 / 104.  The product alone 70 / 64, 67 / 61, 86 / 78, 62 / 54, 781 /
// 762, 61 / 61; 74 / 78 (slower: its ordinary stores), 82 / 78.
template <class T, bool NT, bool RUN>
__global__ __launch_bounds__(LargeTile::THREADS) void fp8_gemm_large_kernel(Fp8GemmParams p) {
  using C = LargeTile;
  // separate arrays, so that a pending load into one does not hold up reads of another
  __shared__ __attribute__((aligned(16))) uint8_t h00[C::HALF], h01[C::HALF], h10[C::HALF], h11[C::HALF];
  __shared__ int e0[C::BM + C::BN], e1[C::BM + C::BN];
  // RUN: strips of outputs, 2 KB and padding a wave
  constexpr int V = 16 / (int)sizeof(T), STRIP = 2 * V, STRIP_LD = C::WN + V;
  __shared__ __attribute__((aligned(16))) T out[RUN ? C::WAVES : 1][RUN ? STRIP * STRIP_LD : 1];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / C::WAVES_N, wn = wave % C::WAVES_N;
  const int64_t pitch = fp8_pitch(p.K);
  const int nk = (int)fp8_blocks(p.K);
  // the tile, and the sources of this lane as 32-bit offsets from its first
  // row; rows past the edge read the last row, their outputs are never stored
  int64_t m0, n0;
  Rows rowsA(p.A), rowsB(p.B);
  int src[C::INS];
  const uint8_t* ebase[C::E_INS];
  int64_t estep[C::E_INS];
  int esrc[C::E_INS], eseg[C::E_INS];
  auto aim = [&](int64_t id) __attribute__((always_inline)) {
    int64_t tm, tn;
    block_tile(id, (p.M + C::BM - 1) / C::BM, (p.N + C::BN - 1) / C::BN, tm, tn);
    m0 = tm * C::BM;
    n0 = tn * C::BN;
    rowsA = Rows(p.A + m0 * pitch);
    rowsB = Rows(p.B + n0 * pitch);
    const int lastA = p.M - 1 - m0 < C::BM - 1 ? (int)(p.M - 1 - m0) : C::BM - 1;
    const int lastB = p.N - 1 - n0 < C::BN - 1 ? (int)(p.N - 1 - n0) : C::BN - 1;
#pragma unroll
    for (int i = 0; i < C::INS; ++i) {
      const bool a = i < C::A_INS;
      const int r = 16 * (a ? wave * C::A_INS + i : wave * C::B_INS + i - C::A_INS) + (lane >> 2);
      const int last = a ? lastA : lastB;
      src[i] = (r < last ? r : last) * (int)pitch + 16 * ((lane & 3) ^ ((r >> 2) & 3));
    }
#pragma unroll
    for (int i = 0; i < C::E_INS; ++i) {
      eseg[i] = (wave + i * C::WAVES) % C::E_SEGS;  // fewer runs than waves: some load one twice
      const bool a = eseg[i] * 64 < C::BM;
      const int r = eseg[i] * 64 - (a ? 0 : C::BM) + lane, last = a ? lastA : lastB;
      ebase[i] = a ? p.eA + m0 * 4 : p.eB + n0 * 4;
      esrc[i] = 4 * (r < last ? r : last);
      estep[i] = (a ? p.M : p.N) * 4;
    }
  };
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
  auto clear = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < C::IT; ++i)
#pragma unroll
      for (int j = 0; j < C::JT; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;
  };
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
    float fa[C::IT], fb[C::JT];
#pragma unroll
    for (int i = 0; i < C::IT; ++i) fa[i] = scale_of(sa[i]);
#pragma unroll
    for (int j = 0; j < C::JT; ++j) fb[j] = scale_of(sb[j]);
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
    interleave<4, C::IT * C::JT, 4 * (C::IT + C::JT)>();
    __builtin_amdgcn_s_setprio(0);
    // the products belong to this segment: keep the compiler from moving them past the barrier
#pragma unroll
    for (int i = 0; i < C::IT; ++i)
#pragma unroll
      for (int j = 0; j < C::JT; ++j) asm volatile("" : "+v"(acc[i][j]));
  };
  // `inner`: stages t + 1 and t + 2 exist (a constant: a load behind a branch
  // would make the compiler wait for all loads at the loop's head).  `more`:
  // stores under way in front of the loads that the two waits leave out;
  // `held`: the loads of (t + 1, 1) are under way already.
  auto stage = [&](auto inner, auto more0, auto more1, auto held, int t, const uint8_t* r0, const uint8_t* r1, const int* e,
                   uint8_t* w0, uint8_t* w1, int* we) __attribute__((always_inline)) {
    // read (t, 0): the buffer of (t + 1, 1) is free
    read(r0);
#pragma unroll
    for (int i = 0; i < C::IT; ++i) sa[i] = e[wm * C::WM + i * 32 + lrow] >> (8 * (t & 3));
#pragma unroll
    for (int j = 0; j < C::JT; ++j) sb[j] = e[C::BM + wn * C::WN + j * 32 + lrow] >> (8 * (t & 3));
    if (inner || t + 1 < nk) {
      if constexpr (!held) load_half(w1, t + 1, 1);
      wait_loads<N0 + N1 + more0>();  // (t, 1) is there
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
      wait_loads<N0 + N1 + more1>();  // (t + 1, 0) is there
    } else {
      wait_loads<N1>();
    }
    __builtin_amdgcn_s_waitcnt(0xC07F);
    meet();
    multiply();
    meet();
  };
  constexpr std::true_type yes{};
  constexpr std::false_type no{};
  constexpr std::integral_constant<int, 0> none{};
  const bool behind = wave >= C::WAVES / 2;
  auto stages_from = [&](int t) __attribute__((always_inline)) {
    for (; t + 3 < nk; t += 2) {
      stage(yes, none, none, no, t, h00, h01, e0, h00, h11, e0);
      stage(yes, none, none, no, t + 1, h10, h11, e1, h10, h01, e1);
    }
    stage(no, none, none, no, t, h00, h01, e0, h00, h11, e0);
    if (RUN || t + 1 < nk) stage(no, none, none, no, t + 1, h10, h11, e1, h10, h01, e1);
    if (!RUN && t + 2 < nk) stage(no, none, none, no, t + 2, h00, h01, e0, h00, h11, e0);
    if (!behind) meet();
  };
  auto store_all = [&](int64_t row0, int64_t col0) __attribute__((always_inline)) {
    if constexpr (RUN) {
      // STRIP rows at a time through LDS of their own, whole lines out of it;
      // rows past the edge hold what the last row does and store it there again.
      // Ordinary stores: nontemporal / ordinary with the pass that reads the
      // outputs next, us: bfloat16 8192 x 4096 x 1024 93 / 88, 16384 x 4096 x 512
      // 134 / 124, float32 8192 x 4096 x 1024 110 / 104, 8192 x 8192 x 1024 208 / 190;
      // the product alone 63 / 63, 74 / 78, 75 / 77, 134 / 149.  An output that is
      // read only much later, as a weight gradient may be, loses by them.
      T* const strip = out[wave];
      const float least = p.relu ? 0.0f : -__builtin_huge_valf();
      const int lr = lane / (C::WN / V), lc = lane % (C::WN / V) * V;
      T* const to = static_cast<T*>(p.C) + row0 * p.ldc + col0 + wn * C::WN + lc;
      const int last = p.M - 1 - row0 < C::BM - 1 ? (int)(p.M - 1 - row0) : C::BM - 1;
#pragma unroll
      for (int i = 0; i < C::WM / STRIP; ++i) {
#pragma unroll
        for (int j = 0; j < C::JT; ++j)
#pragma unroll
          for (int r = 0; r < STRIP / 2; ++r) {
            const float o = acc[i * STRIP / 32][j][i * STRIP % 32 / 2 + r];
            strip[(8 * (r >> 2) + 4 * half + (r & 3)) * STRIP_LD + j * 32 + lrow] = (T)(o < least ? least : o);
          }
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          typedef T vec __attribute__((ext_vector_type(V)));
          const vec v = *reinterpret_cast<const vec*>(strip + (V * h + lr) * STRIP_LD + lc);
          const int r = wm * C::WM + STRIP * i + V * h + lr;
          *reinterpret_cast<vec*>(to + (r < last ? r : last) * p.ldc) = v;
        }
        __builtin_amdgcn_wave_barrier();
      }
    } else {
      __syncthreads();
      // a strip of 32 rows at a time through this wave's part of LDS, so that the
      // stores are whole lines
      uint8_t* const own = (wave < 4 ? (wave < 2 ? h00 : h01) : (wave < 6 ? h10 : h11)) + (wave & 1) * (C::HALF / 2);
      float* strip = reinterpret_cast<float*>(own);
#pragma unroll
      for (int i = 0; i < C::IT; ++i) {
        const StripMask<T, C::WN> mask(p, row0 + wm * C::WM + i * 32, col0 + wn * C::WN);
#pragma unroll
        for (int j = 0; j < C::JT; ++j)
#pragma unroll
          for (int r = 0; r < 16; ++r)
            strip[(8 * (r >> 2) + 4 * half + (r & 3)) * C::OUT_LD + j * 32 + lrow] = acc[i][j][r];
        __builtin_amdgcn_wave_barrier();
        store_strip<T, C::WN, C::OUT_LD, NT>(p, strip, mask, row0 + wm * C::WM + i * 32, col0 + wn * C::WN);
        __builtin_amdgcn_wave_barrier();
      }
    }
  };
  int64_t id = blockIdx.x;
  aim(id);
  clear();
  load_half(h00, 0, 0);
  load_scales(e0, 0);
  load_half(h01, 0, 1);
  if constexpr (!RUN) {
    if (nk > 1) {
      load_half(h10, 1, 0);
      load_scales(e1, 1);
      wait_loads<N0 + N1>();
    } else {
      wait_loads<N1>();
    }
    meet();
    if (behind) meet();
    stages_from(0);
    store_all(m0, n0);
  } else {
    constexpr std::integral_constant<int, C::WM / STRIP * 2> STORES{};
    // the first two stages, behind `more` stores
    auto begin = [&](auto more) __attribute__((always_inline)) {
      wait_loads<N1 + N0 + N1 + more>();  // (0, 0) is there
      meet();
      if (behind) meet();
      stage(yes, more, more, yes, 0, h00, h01, e0, h00, h11, e0);
      stage(yes, more, none, no, 1, h10, h11, e1, h10, h01, e1);
    };
    auto rest_of_start = [&]() __attribute__((always_inline)) {
      load_half(h10, 1, 0);
      load_scales(e1, 1);
      load_half(h11, 1, 1);
    };
    rest_of_start();
    begin(none);
    const int64_t tiles = ((p.M + C::BM - 1) / C::BM) * (p.N / C::BN);
    for (;;) {
      stages_from(2);
      const int64_t row0 = m0, col0 = n0;
      id += gridDim.x;
      const bool more = id < tiles;
      if (more) {
        aim(id);
        load_half(h00, 0, 0);
        load_scales(e0, 0);
        load_half(h01, 0, 1);
        rest_of_start();
      }
      asm volatile("" ::: "memory");  // the loads go first
      __builtin_amdgcn_sched_barrier(0);
      store_all(row0, col0);
      if (!more) return;
      asm volatile("" ::: "memory");
      __builtin_amdgcn_sched_barrier(0);
      clear();
      begin(STORES);
    }
  }
}

// ---------------------------------------------------------------------------
// The pipelined loop: every wave reads the next step's operands from LDS while
// it multiplies the current ones; one barrier a stage of 128 along K.  KG = 2:
// half of the waves take the first half of each stage along K, half the
// second, and their sums meet in LDS at the end, so that a wave's tile is
// twice as large and reads (and widens) less for each product.  NS whole
// stages of 128-byte rows in LDS, the 16-byte chunk index XOR-ed with (r / 2)
// mod 8.  SPLIT: blockIdx.y takes `chunk` stages and leaves float32 sums in
// p.part.  256 x 256 tiles do not fit this loop: their accumulators and a second
// set of operands spill.
// ---------------------------------------------------------------------------
template <int BM_, int BN_, int WM_, int WN_, int KG_, int NS_>
struct PipeTile {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, KG = KG_, NS = NS_;
  static constexpr int WAVES_N = BN / WN, PLANE = (BM / WM) * WAVES_N;  // waves over the output
  static constexpr int IT = WM / 32, JT = WN / 32, STEPS = 2 / KG;      // steps of 64 along K a stage and wave
  static constexpr int CODES = (BM + BN) * FP8_BLOCK;
  static constexpr int INS = (BM + BN) / 64;                            // 1 KB loads of a wave and stage, eight rows each
  static constexpr int E_SEGS = (BM + BN) / 64;
  static constexpr int OUT_LD = WN + 8;
  static_assert(PLANE * KG == 8 && E_SEGS <= 8, "eight waves");
  static_assert(NS == 4 || (NS == 3 && KG == 1), "an even number of steps a turn");
};

// T: the stored type (SPLIT: float).
template <class T, class C, bool SPLIT, bool NT>
__global__ __launch_bounds__(512) void fp8_gemm_pipe_kernel(Fp8GemmParams p, int chunk) {
  __shared__ __attribute__((aligned(16))) uint8_t q0[C::CODES], q1[C::CODES], q2[C::CODES], q3[C::NS > 3 ? C::CODES : 16];
  __shared__ int x0[C::BM + C::BN], x1[C::BM + C::BN], x2[C::BM + C::BN], x3[C::NS > 3 ? C::BM + C::BN : 4];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kg = wave / C::PLANE, wm = wave % C::PLANE / C::WAVES_N, wn = wave % C::WAVES_N;
  int64_t tm, tn;
  block_tile(blockIdx.x, (p.M + C::BM - 1) / C::BM, (p.N + C::BN - 1) / C::BN, tm, tn);
  const int64_t m0 = tm * C::BM, n0 = tn * C::BN;
  const int64_t pitch = fp8_pitch(p.K);
  const int all = (int)fp8_blocks(p.K), first = SPLIT ? (int)blockIdx.y * chunk : 0;
  const int nk = SPLIT && first + chunk < all ? chunk : all - first;
  const int lastA = p.M - 1 - m0 < C::BM - 1 ? (int)(p.M - 1 - m0) : C::BM - 1;
  const int lastB = p.N - 1 - n0 < C::BN - 1 ? (int)(p.N - 1 - n0) : C::BN - 1;
  const Rows rowsA(p.A + m0 * pitch + (int64_t)first * FP8_BLOCK), rowsB(p.B + n0 * pitch + (int64_t)first * FP8_BLOCK);
  // this wave's 1 KB loads, eight rows each: of A, then of B
  int src[C::INS];
#pragma unroll
  for (int i = 0; i < C::INS; ++i) {
    const int at = 8 * (wave * C::INS + i), r = at + (lane >> 3);
    const bool a = at < C::BM;
    const int row = a ? r : r - C::BM, last = a ? lastA : lastB;
    src[i] = (row < last ? row : last) * (int)pitch + 16 * ((lane & 7) ^ ((r >> 1) & 7));
  }
  // scale words: a run of 64 rows a wave (fewer runs than waves: some twice)
  const int seg = wave % C::E_SEGS;
  const bool eA = seg * 64 < C::BM;
  const int er = seg * 64 - (eA ? 0 : C::BM) + lane, elast = eA ? lastA : lastB;
  const uint8_t* const ebase = eA ? p.eA + m0 * 4 : p.eB + n0 * 4;
  const int64_t estep = (eA ? p.M : p.N) * 4;
  const int esrc = 4 * (er < elast ? er : elast);
  auto load = [&](uint8_t* d, int* e, int t) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < C::INS; ++i)
      (8 * (wave * C::INS + i) < C::BM ? rowsA : rowsB).to_lds16(d + (wave * C::INS + i) * 1024, src[i], t * FP8_BLOCK);
    Rows(ebase + ((first + t) >> 2) * estep).to_lds4(e + seg * 64, esrc);
  };
  constexpr int PER = C::INS + 1;  // loads of a stage and wave
  v16f acc[C::IT][C::JT];
#pragma unroll
  for (int i = 0; i < C::IT; ++i)
#pragma unroll
    for (int j = 0; j < C::JT; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;
  const int lrow = lane & 31, half = lane >> 5, sw = (lrow >> 1) & 7;
  const int offA = (wm * C::WM + lrow) * FP8_BLOCK, offB = (C::BM + wn * C::WN + lrow) * FP8_BLOCK;
  struct Operands {
    v8i a[C::IT], b[C::JT];
    int sa[C::IT], sb[C::JT];
  } set0, set1;
  // the operands of one step: codes 64 kk .. + 63 of the stage, and its scales
  auto read = [&](Operands& o, const uint8_t* st, const int* e, int t, int kk) __attribute__((always_inline)) {
    const int c0 = 16 * ((4 * kk + 2 * half) ^ sw), c1 = 16 * ((4 * kk + 2 * half + 1) ^ sw);
    const int sh = 8 * ((first + t) & 3);
    auto frag = [&](const uint8_t* q) __attribute__((always_inline)) {
      const v4i x = *reinterpret_cast<const v4i*>(q + c0);
      const v4i y = *reinterpret_cast<const v4i*>(q + c1);
      return v8i{x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
    };
#pragma unroll
    for (int i = 0; i < C::IT; ++i) {
      o.a[i] = frag(st + offA + i * 32 * FP8_BLOCK);
      o.sa[i] = e[wm * C::WM + i * 32 + lrow] >> sh;
    }
#pragma unroll
    for (int j = 0; j < C::JT; ++j) {
      o.b[j] = frag(st + offB + j * 32 * FP8_BLOCK);
      o.sb[j] = e[C::BM + wn * C::WN + j * 32 + lrow] >> sh;
    }
  };
  auto multiply = [&](const Operands& o) __attribute__((always_inline)) {
    float fa[C::IT], fb[C::JT];
#pragma unroll
    for (int i = 0; i < C::IT; ++i) fa[i] = scale_of(o.sa[i]);
#pragma unroll
    for (int j = 0; j < C::JT; ++j) fb[j] = scale_of(o.sb[j]);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      v8b wa[C::IT], wb[C::JT];
#pragma unroll
      for (int j = 0; j < C::JT; ++j) wb[j] = widen(o.b[j][2 * q], o.b[j][2 * q + 1], fb[j]);
#pragma unroll
      for (int i = 0; i < C::IT; ++i) wa[i] = widen(o.a[i][2 * q], o.a[i][2 * q + 1], fa[i]);
#pragma unroll
      for (int i = 0; i < C::IT; ++i)
#pragma unroll
        for (int j = 0; j < C::JT; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wa[i], wb[j], acc[i][j], 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < C::IT; ++i)
#pragma unroll
      for (int j = 0; j < C::JT; ++j) asm volatile("" : "+v"(acc[i][j]));
  };
  // Stage t, whose first step's operands are in `cur`; q, e: its buffer, qn, en:
  // the next one's.  The barrier says that stage t + 1 has landed and that
  // everyone has read stage t, whose buffer then takes stage t + NS.
  auto stage = [&](auto inner, int t, Operands& cur, Operands& nxt, uint8_t* q, int* e, const uint8_t* qn,
                   const int* en) __attribute__((always_inline)) {
    if constexpr (C::STEPS == 2) {
      read(nxt, q, e, t, 1);
      multiply(cur);
    }
    if (inner) {
      wait_loads<(C::NS - 2) * PER>();
    } else if (t + 1 < nk) {
      const int later = nk - t - 2;  // stages behind t + 1 that are under way
      if (C::NS > 3 && later >= 2)
        wait_loads<2 * PER>();
      else if (later >= 1)
        wait_loads<PER>();
      else
        wait_loads<0>();
    }
    __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
    meet();
    if (inner || t + 1 < nk) read(C::STEPS == 2 ? cur : nxt, qn, en, t + 1, C::STEPS == 2 ? 0 : kg);
    if (inner || t + C::NS < nk) load(q, e, t + C::NS);
    multiply(C::STEPS == 2 ? nxt : cur);
  };
  load(q0, x0, 0);
  if (nk > 1) load(q1, x1, 1);
  if (nk > 2) load(q2, x2, 2);
  if (C::NS > 3 && nk > 3) load(q3, x3, 3);
  if (nk >= C::NS)
    wait_loads<(C::NS - 1) * PER>();
  else
    wait_loads<0>();
  meet();
  read(set0, q0, x0, 0, C::STEPS == 2 ? 0 : kg);
  constexpr std::true_type inner{};
  constexpr std::false_type last{};
  // with one step a stage the operand sets swap every stage, with two they end as they began
  Operands& odd = C::STEPS == 2 ? set0 : set1;
  Operands& even = C::STEPS == 2 ? set1 : set0;
  int t = 0;
  auto turn = [&](auto in) __attribute__((always_inline)) {
    auto go = [&](int k, Operands& c, Operands& n, uint8_t* q, int* e, const uint8_t* qn, const int* en)
                  __attribute__((always_inline)) {
      if (in || t + k < nk) stage(in, t + k, c, n, q, e, qn, en);
    };
    go(0, set0, set1, q0, x0, q1, x1);
    go(1, odd, even, q1, x1, q2, x2);
    if constexpr (C::NS == 3) {
      go(2, set0, set1, q2, x2, q0, x0);
    } else {
      go(2, set0, set1, q2, x2, q3, x3);
      go(3, odd, even, q3, x3, q0, x0);
    }
  };
  for (; t + 2 * C::NS - 1 < nk; t += C::NS) turn(inner);
  for (; t < nk; t += C::NS) turn(last);
  __syncthreads();
  if constexpr (C::KG == 2) {
    // the two halves of K: each wave hands half of its rows to its partner
    constexpr int HI = C::IT / 2, BYTES = HI * C::JT * 4096, FIT = C::CODES / BYTES;
    static_assert(FIT * C::NS >= 8, "the exchange fits the stage buffers");
    auto room = [&](int w) __attribute__((always_inline)) {
      uint8_t* const b = w / FIT == 0 ? q0 : (w / FIT == 1 ? q1 : (w / FIT == 2 ? q2 : q3));
      return reinterpret_cast<float4*>(b + w % FIT * BYTES) + lane;
    };
    float4* const give = room(wave);
#pragma unroll
    for (int i = 0; i < HI; ++i)
#pragma unroll
      for (int j = 0; j < C::JT; ++j) {
        const v16f lo = acc[i][j], hi = acc[HI + i][j], v = kg ? lo : hi;
#pragma unroll
        for (int r = 0; r < 4; ++r)
          give[((i * C::JT + j) * 4 + r) * 64] = make_float4(v[4 * r], v[4 * r + 1], v[4 * r + 2], v[4 * r + 3]);
      }
    __syncthreads();
    const float4* const take = room(wave ^ 4);
#pragma unroll
    for (int i = 0; i < HI; ++i)
#pragma unroll
      for (int j = 0; j < C::JT; ++j) {
        const v16f lo = acc[i][j], hi = acc[HI + i][j];
        v16f v = kg ? hi : lo;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float4 o = take[((i * C::JT + j) * 4 + r) * 64];
          v[4 * r] += o.x;
          v[4 * r + 1] += o.y;
          v[4 * r + 2] += o.z;
          v[4 * r + 3] += o.w;
        }
        acc[i][j] = v;
      }
    __syncthreads();
  }
  constexpr int STRIPS = C::IT / C::KG, STRIP = 32 * C::OUT_LD * 4, FIT = C::CODES / STRIP;
  static_assert(FIT * C::NS >= 8, "the output strips fit the stage buffers");
  uint8_t* const own = (wave / FIT == 0 ? q0 : (wave / FIT == 1 ? q1 : (wave / FIT == 2 ? q2 : q3))) + wave % FIT * STRIP;
  float* const strip = reinterpret_cast<float*>(own);
  Fp8GemmParams to = p;
  if constexpr (SPLIT) {
    to.C = p.part + (int64_t)blockIdx.y * p.M * p.N;
    to.ldc = p.N;
    to.relu = 0;
    to.mask = nullptr;
  }
#pragma unroll
  for (int i = 0; i < STRIPS; ++i) {
    const int64_t row0 = m0 + wm * C::WM + (kg * STRIPS + i) * 32, col0 = n0 + wn * C::WN;
    const StripMask<T, C::WN> mask(to, row0, col0);
#pragma unroll
    for (int j = 0; j < C::JT; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        strip[(8 * (r >> 2) + 4 * half + (r & 3)) * C::OUT_LD + j * 32 + lrow] = acc[i][j][r];
    __builtin_amdgcn_wave_barrier();
    store_strip<T, C::WN, C::OUT_LD, NT>(to, strip, mask, row0, col0);
    __builtin_amdgcn_wave_barrier();
  }
}

// The parts of a split product added in order, with the product's epilogue.
template <class T>
__global__ __launch_bounds__(256) void fp8_split_sum_kernel(Fp8GemmParams p, int splits) {
  const int64_t quads = (p.N + 3) / 4, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
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

// ---------------------------------------------------------------------------
// Few rows of A (serving: single tokens): the weights stream from memory to
// registers once, 16 outputs a block, its waves take every eighth block of K
// and add up in LDS.  A from raw rows (X is quantized here, in registers: every
// block of threads needs all of it, but it is small) or from codes.
// Lane l holds row l % 16, codes 32 (l / 16) .. + 31 of a block, eight of them a
// v_mfma_f32_16x16x32_bf16.  Latency bounds it: one bfloat16 row through 4096 x
// 1024 weights (4.2 MB) takes 4.0 us.
// ---------------------------------------------------------------------------
constexpr int ROW_WAVES = 8;

template <class X>
__device__ __forceinline__ v8i row_block(const X* x, int64_t left, int& byte) {
  Quad<X> v[8];
  uint32_t key = 0u;
  typename Quad<X>::ColTop unused{};
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i].load(x + 4 * i, left - 4 * i);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    typename Quad<X>::RowTop r;
    v[i].top(r, unused);
    const uint32_t k = Quad<X>::row_key(r);
    key = key > k ? key : k;
  }
  auto s = __builtin_amdgcn_permlane16_swap(key, key, false, false);
  key = s[0] > s[1] ? s[0] : s[1];
  s = __builtin_amdgcn_permlane32_swap(key, key, false, false);
  key = Quad<X>::bf_keys(s[0] > s[1] ? s[0] : s[1]) & 0xffffu;
  const uint32_t e = scale_bytes(key) & 0xffffu;
  byte = (int)(key >= NAN_KEY ? 255u : e);
  v8i q;
#pragma unroll
  for (int i = 0; i < 8; ++i) q[i] = key >= NAN_KEY ? 0x7f7f7f7f : (int)v[i].row_codes(scale_up(e));
  return q;
}
__device__ __forceinline__ v8i code_block(const uint8_t* q) {
  const v4i a = *reinterpret_cast<const v4i*>(q), b = *reinterpret_cast<const v4i*>(q + 16);
  return v8i{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
}

// X: the raw rows' type, or void: codes.  MT: 16 MT >= M.
template <class T, class X, int MT>
__global__ __launch_bounds__(64 * ROW_WAVES) void fp8_rows_kernel(Fp8GemmParams p, const void* x, int64_t ldx) {
  __shared__ float sum[ROW_WAVES][MT][256];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, g = lane >> 4;
  const int64_t n0 = block_id() * 16;
  if (n0 >= p.N) return;
  const int64_t n = n0 + r < p.N ? n0 + r : p.N - 1;
  const int64_t pitch = fp8_pitch(p.K);
  const int nk = (int)fp8_blocks(p.K);
  const uint8_t* const w = p.B + n * pitch + 32 * g;
  v4f acc[MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) acc[m] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
  // the weights two turns ahead
  v8i b0{}, b1{};
  int s0 = 127, s1 = 127;
  auto weights = [&](int k, v8i& b, int& sb) __attribute__((always_inline)) {
    if (k >= nk) return;
    b = code_block(w + (int64_t)k * FP8_BLOCK);
    sb = p.eB[((int64_t)(k >> 2) * p.N + n) * 4 + (k & 3)];
  };
  weights(wave, b0, s0);
  weights(wave + ROW_WAVES, b1, s1);
  for (int k = wave; k < nk; k += ROW_WAVES) {
    const v8i b = b0;
    const int sb = s0;
    b0 = b1;
    s0 = s1;
    weights(k + 2 * ROW_WAVES, b1, s1);
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      const int64_t row = 16 * m + r;
      v8i a{0, 0, 0, 0, 0, 0, 0, 0};
      int sa = 127;
      if constexpr (std::is_void<X>::value) {
        if (row < p.M) {
          a = code_block(p.A + row * pitch + (int64_t)k * FP8_BLOCK + 32 * g);
          sa = p.eA[((int64_t)(k >> 2) * p.M + row) * 4 + (k & 3)];
        }
      } else {
        const int64_t at = (int64_t)k * FP8_BLOCK + 32 * g;
        a = row_block(static_cast<const X*>(x) + (row < p.M ? row : 0) * ldx + at, row < p.M ? p.K - at : 0, sa);
      }
      const float fa = scale_of(sa), fb = scale_of(sb);
#pragma unroll
      for (int q = 0; q < 4; ++q)
        acc[m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen(b[2 * q], b[2 * q + 1], fb),
                                                         widen(a[2 * q], a[2 * q + 1], fa), acc[m], 0, 0, 0);
    }
  }
  // lane: output columns n0 + 4 g .., row r
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int i = 0; i < 4; ++i) sum[wave][m][r * 16 + 4 * g + i] = acc[m][i];
  __syncthreads();
  for (int i = threadIdx.x; i < MT * 256; i += 64 * ROW_WAVES) {
    const int64_t row = i >> 4, col = n0 + (i & 15);
    if (row >= p.M || col >= p.N) continue;
    float o = 0.0f;
#pragma unroll
    for (int v = 0; v < ROW_WAVES; ++v) o += sum[v][i >> 8][i & 255];
    if (p.relu) o = o < 0.0f ? 0.0f : o;
    if (p.mask) o = (float)static_cast<const T*>(p.mask)[row * p.ldmask + col] > 0.0f ? o : 0.0f;
    static_cast<T*>(p.C)[row * p.ldc + col] = (T)o;
  }
}

// ---------------------------------------------------------------------------
// launches
// ---------------------------------------------------------------------------
using MidTile = PipeTile<256, 128, 64, 64, 1, 3>;
using SmallTile = PipeTile<128, 128, 64, 64, 2, 4>;
// For 16-bit outputs: sums in the order of the larger tiles, so that a row of an
// activation has the same bits whichever tile the number of rows leads to.
// Halves of K / one order, us: 2048 x 4096 x 1024 24.2 / 24.1, 300 x 1024 x 512
// 9.0 / 8.7, 1024 x 1024 x 4096 21.0 / 21.0, 4096 x 1024 x 8192 67 / 72.
using SmallTile16 = PipeTile<128, 128, 64, 32, 1, 4>;

static int64_t tiles_of(int64_t M, int64_t N, int64_t bm, int64_t bn) {
  return ((M + bm - 1) / bm) * ((N + bn - 1) / bn);
}

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
struct Plan {
  enum Tile { SMALL, MID, LARGE } tile;
  int splits, chunk;  // parts along K, stages of each
};
static Plan plan_of(int64_t M, int64_t N, int64_t K) {
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
    if (s > 1) t += 4.0 + (double)(M * N) * 8.0 * s / 4.0e6;  // written and read at about 4 TB/s
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
static bool several_tiles(const Plan& plan, int64_t M, int64_t N, bool masked, bool lines) {
  return plan.tile == Plan::LARGE && lines && !masked && tiles_of(M, N, LargeTile::BM, LargeTile::BN) > 256 &&
         N % LargeTile::BN == 0 && plan.chunk % 2 == 0 && plan.chunk >= 4;
}

fqt_fp8_form fp8_gemm_form(int64_t M, int64_t N, int64_t K, bool masked, bool lines) {
  if (M <= ROWS_MAX) return FQT_FP8_ROWS;
  const Plan plan = plan_of(M, N, K);
  switch (plan.tile) {
    case Plan::SMALL: return plan.splits > 1 ? FQT_FP8_PARTS : FQT_FP8_SMALL;
    case Plan::MID: return FQT_FP8_MIDDLE;
    case Plan::LARGE: break;
  }
  return several_tiles(plan, M, N, masked, lines) ? FQT_FP8_SEVERAL : FQT_FP8_LARGE;
}

int64_t fp8_gemm_partials(int64_t M, int64_t N, int64_t K) {
  if (M <= ROWS_MAX) return 0;
  const int64_t s = plan_of(M, N, K).splits;
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
    const Plan plan = plan_of(p.M, p.N, p.K);
    auto tiles = [&](auto c) {
      using C = decltype(c);
      return tiles_of(p.M, p.N, C::BM, C::BN);
    };
    const int64_t blocks = plan.tile == Plan::LARGE ? tiles(LargeTile{}) : plan.tile == Plan::MID ? tiles(MidTile{}) : tiles(SmallTile{});
    if (blocks > 0x7FFFFF) return hipErrorInvalidValue;  // 2^32 threads, 2^37 outputs
    int64_t grid = blocks;
    auto go = [&](auto kernel, auto... more) {
      hipLaunchKernelGGL(kernel, dim3((unsigned)grid, (unsigned)plan.splits), dim3(512), 0, s, p, more...);
      return hipGetLastError();
    };
    if (plan.tile == Plan::LARGE) {
      if (several_tiles(plan, p.M, p.N, p.mask != nullptr, nt)) {
        grid = 256;  // one block a unit
        return go(fp8_gemm_large_kernel<T, true, true>);
      }
      return nt ? go(fp8_gemm_large_kernel<T, true, false>) : go(fp8_gemm_large_kernel<T, false, false>);
    }
    if (plan.tile == Plan::MID)
      return nt ? go(fp8_gemm_pipe_kernel<T, MidTile, false, true>, plan.chunk)
                : go(fp8_gemm_pipe_kernel<T, MidTile, false, false>, plan.chunk);
    using Small = std::conditional_t<sizeof(T) == 2, SmallTile16, SmallTile>;
    if (plan.splits == 1)
      return nt ? go(fp8_gemm_pipe_kernel<T, Small, false, true>, plan.chunk)
                : go(fp8_gemm_pipe_kernel<T, Small, false, false>, plan.chunk);
    const hipError_t err = go(fp8_gemm_pipe_kernel<float, SmallTile, true, false>, plan.chunk);
    if (err != hipSuccess) return err;
    const int64_t quads = p.M * ((p.N + 3) / 4);
    hipLaunchKernelGGL((fp8_split_sum_kernel<T>), dim3((unsigned)((quads + 255) / 256)), dim3(256), 0, s, p, plan.splits);
    return hipGetLastError();
  });
}

}  // namespace fqt
