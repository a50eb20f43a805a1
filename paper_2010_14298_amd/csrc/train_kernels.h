// Internal interface and device helpers of the floating-point operators
// around the layers (norm.hip, fp8_quant.hip, fp8_gemm.hip, clip.hip), whose
// entry points are in api_train.hip.  Not part of the public ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "../../include/fqt.h"

namespace fqt {

// ---------------------------------------------------------------------------
// element types: float, __bf16, _Float16; arithmetic is always float32 or more
// ---------------------------------------------------------------------------
// V consecutive elements at any element-aligned address.  The address mode
// of this target takes unaligned wide accesses, so a row of odd pitch still
// moves by 16-byte instructions.
template <class T, int V>
struct Packed {
  typedef T type __attribute__((ext_vector_type(V), aligned(sizeof(T))));
};

template <class T, int V>
__device__ __forceinline__ void load_vec(const T* p, float (&f)[V]) {
  const typename Packed<T, V>::type v = *reinterpret_cast<const typename Packed<T, V>::type*>(p);
#pragma unroll
  for (int i = 0; i < V; ++i) f[i] = (float)v[i];
}
template <class T, int V>
__device__ __forceinline__ void store_vec(T* p, const float (&f)[V]) {
  typename Packed<T, V>::type v;
#pragma unroll
  for (int i = 0; i < V; ++i) v[i] = (T)f[i];
  *reinterpret_cast<typename Packed<T, V>::type*>(p) = v;
}
// The first n of V elements (n may be <= 0 or >= V); the others read as zero.
template <class T, int V>
__device__ __forceinline__ void load_part(const T* p, int64_t n, float (&f)[V]) {
  if (n >= V) {
    load_vec<T, V>(p, f);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) f[i] = i < n ? (float)p[i] : 0.0f;
  }
}
template <class T, int V>
__device__ __forceinline__ void store_part(T* p, int64_t n, const float (&f)[V]) {
  if (n >= V) {
    store_vec<T, V>(p, f);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (i < n) p[i] = (T)f[i];
  }
}

// Calls f with a value of the element type that `type` names.
template <class F>
inline hipError_t with_type(fqt_dtype type, F f) {
  switch (type) {
    case FQT_F32: return f(float{});
    case FQT_BF16: return f(__bf16{});
    case FQT_F16: return f(_Float16{});
  }
  return hipErrorInvalidValue;
}
inline bool valid_type(fqt_dtype t) { return t == FQT_F32 || t == FQT_BF16 || t == FQT_F16; }

// ---------------------------------------------------------------------------
// one-dimensional launches of any length: a dimension of a grid holds fewer
// than 2^32 threads (more are cut off without an error), so long launches get a
// second one.  Blocks from `blocks` on find nothing to do.
// ---------------------------------------------------------------------------
inline dim3 grid_of(int64_t blocks, int threads) {
  const int64_t most = ((int64_t)1 << 31) / threads, y = (blocks + most - 1) / most;
  return dim3((unsigned)(y > 1 ? most : blocks), (unsigned)y);
}
__device__ __forceinline__ int64_t block_id() { return (int64_t)blockIdx.y * gridDim.x + blockIdx.x; }

// ---------------------------------------------------------------------------
// reductions over a wave: every lane gets the result, in a fixed order.
// Rotations inside rows of 16 lanes, then row and half-wave swaps.
// ---------------------------------------------------------------------------
template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, CTRL, 0xf, 0xf, true);
}
constexpr int DPP_ROR = 0x120;  // + n: rotate right by n inside 16 lanes

template <class Op>
__device__ __forceinline__ uint32_t row16_reduce(uint32_t v, Op op) {
  v = op(v, dpp<DPP_ROR + 8>(v));
  v = op(v, dpp<DPP_ROR + 4>(v));
  v = op(v, dpp<DPP_ROR + 2>(v));
  return op(v, dpp<DPP_ROR + 1>(v));
}
template <class Op>
__device__ __forceinline__ uint32_t half_reduce(uint32_t v, Op op) {  // over 32 lanes
  v = row16_reduce(v, op);
  const auto s = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  return op(s[0], s[1]);
}
template <class Op>
__device__ __forceinline__ uint32_t wave_reduce(uint32_t v, Op op) {
  v = half_reduce(v, op);
  const auto s = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return op(s[0], s[1]);
}
struct AddF {
  __device__ __forceinline__ uint32_t operator()(uint32_t a, uint32_t b) const {
    return __float_as_uint(__uint_as_float(a) + __uint_as_float(b));
  }
};
__device__ __forceinline__ float wave_sum(float v) { return __uint_as_float(wave_reduce(__float_as_uint(v), AddF{})); }

// ---------------------------------------------------------------------------
// layer norm
// ---------------------------------------------------------------------------
struct NormParams {
  const void* x;
  int64_t ldx;
  int64_t rows, cols;
  const float* gamma;  // may be null (ones)
  const float* beta;   // may be null (zeros)
  float eps;
  void* y;             // forward: output; backward: grad_X
  int64_t ldy;
  float* mean;         // forward: may be null
  float* rstd;
  // backward
  const void* g;
  int64_t ldg;
  float* grad_gamma;   // both null: not formed
  float* grad_beta;
  float* part;         // [blocks][2][cols]
  // checkpoint of xh (null: none): written by the forward, read by the backward
  // in place of x and mean
  uint8_t* q8;
  uint8_t* e8;
};
hipError_t launch_norm_forward(fqt_dtype type, const NormParams& p, hipStream_t s);
int64_t norm_backward_partials(int64_t rows, int64_t cols);  // floats
hipError_t launch_norm_backward(fqt_dtype type, const NormParams& p, hipStream_t s);

// ---------------------------------------------------------------------------
// 8-bit floating point operands: codes [rows, pitch], pitch = whole blocks of
// 128, and one power-of-two scale byte for each row and block (fqt.h)
// ---------------------------------------------------------------------------
constexpr int FP8_BLOCK = 128;
__host__ __device__ inline int64_t fp8_blocks(int64_t K) { return (K + FP8_BLOCK - 1) / FP8_BLOCK; }
__host__ __device__ inline int64_t fp8_pitch(int64_t K) { return fp8_blocks(K) * FP8_BLOCK; }
__host__ __device__ inline int64_t fp8_exp_bytes(int64_t rows, int64_t K) { return (fp8_blocks(K) + 3) / 4 * 4 * rows; }

// Checkpoints: codes [rows, pitch], pitch = whole blocks of 32, and one scale
// byte for each block, [rows, pitch / 32].
constexpr int KEPT_BLOCK = 32;
__host__ __device__ inline int64_t kept_blocks(int64_t cols) { return (cols + KEPT_BLOCK - 1) / KEPT_BLOCK; }
__host__ __device__ inline int64_t kept_pitch(int64_t cols) { return kept_blocks(cols) * KEPT_BLOCK; }
struct Kept {
  uint8_t* q;  // null: none
  uint8_t* e;
};

struct Fp8QuantParams {
  const void* x;
  int64_t rows, cols, ldx;
  int tile;        // one scale for 128 x 128
  int stochastic;
  uint64_t seed;
  uint8_t* q_row;  // operand of x (null: not wanted)
  uint8_t* e_row;
  uint8_t* q_col;  // operand of x^T (null: not wanted)
  uint8_t* e_col;
};
hipError_t launch_fp8_quantize(fqt_dtype type, const Fp8QuantParams& p, hipStream_t s);

// Codes that lie column by column (element (r, k) at k rows + r) into rows; src
// null: nothing to do.
struct Fp8Turn {
  const uint8_t* src;
  int64_t rows, K;
  uint8_t* dst;
};
hipError_t launch_fp8_turn(const Fp8Turn& t, hipStream_t s);
// The quantizer (or nothing, if neither operand is wanted) and two of those, in
// one launch where both of the quantizer's operands are wanted.
hipError_t launch_fp8_quantize_turn(fqt_dtype type, const Fp8QuantParams& p, const Fp8Turn& a, const Fp8Turn& b,
                                    hipStream_t s);

struct Fp8GemmParams {
  static constexpr bool GATED = false, KEEP = false;  // gated; checkpoints too
  const uint8_t* A;   // [M, pitch(K)]
  const uint8_t* eA;
  const uint8_t* B;   // [N, pitch(K)]
  const uint8_t* eB;
  int64_t M, N, K;
  void* C;
  int64_t ldc;
  int relu;
  const void* mask;   // same type as C, or null: C = 0 where mask <= 0
  int64_t ldmask;
  float* part;        // split-K partial sums [splits][M][N]
};
// Raw rows X [M, K] of C's type against B (A is not read), if fp8_rows_raw(M).
bool fp8_rows_raw(int64_t M);
hipError_t launch_fp8_rows(fqt_dtype type, const Fp8GemmParams& p, const void* x, int64_t ldx, hipStream_t s);
int64_t fp8_gemm_partials(int64_t M, int64_t N, int64_t K);  // floats
// Which tile, and for small tiles into how many parts along K a product is split.
struct Fp8Plan {
  enum Tile { SMALL, MID, LARGE } tile;
  int splits, chunk;  // parts along K, stages of each
};
// pass: us of a launch that adds the parts.
Fp8Plan fp8_plan(int64_t M, int64_t N, int64_t K, double pass = 4.0);
// us of a product by itself, as fp8_plan estimates it.
double fp8_plan_time(int64_t M, int64_t N, const Fp8Plan& plan, double pass = 4.0);
hipError_t launch_fp8_parts(const Fp8GemmParams& p, const Fp8Plan& plan, hipStream_t s);  // to p.part
fqt_fp8_form fp8_gemm_form(int64_t M, int64_t N, int64_t K, bool masked, bool lines);
hipError_t launch_fp8_gemm(fqt_dtype type, const Fp8GemmParams& p, hipStream_t s);
// Two products that do not depend on each other, a with float32 outputs; whether
// their parts run at once (and need room of their own).  any_order: b's sums need
// not have the order that b has by itself.
bool fp8_two_at_once(int64_t Ma, int64_t Na, int64_t Ka, int64_t Mb, int64_t Nb, int64_t Kb);
hipError_t launch_fp8_two(fqt_dtype type, const Fp8GemmParams& a, const Fp8GemmParams& b, bool any_order, hipStream_t s);

// ---------------------------------------------------------------------------
// gated layer
// ---------------------------------------------------------------------------
// A product whose outputs are H [M, hidden]: B is [W_gate; W_up] (N = 2 hidden
// rows), C is H.  Checkpoints may be null.
struct GatedGemmParams : Fp8GemmParams {
  static constexpr bool GATED = true;
  int64_t hidden;
  fqt_act act;
  Kept gate, up;
};
// Whether a call that keeps nothing reads X [M, K] as it is (p.A is not read).
bool gated_rows_raw(int64_t M, int64_t hidden, int64_t K);
int64_t gated_partials(int64_t M, int64_t hidden, int64_t K);  // floats
hipError_t launch_gated_gemm(fqt_dtype type, const GatedGemmParams& p, const void* x, int64_t ldx, hipStream_t s);

// The quantizer of D = [G gate | G up] [rows, cols = 2 hidden], q.x and q.ldx those
// of G, with kept operands to lay out, as above.
struct GatedQuantParams {
  Fp8QuantParams q;
  int64_t hidden;
  const uint8_t *q_gate, *e_gate, *q_up, *e_up;
};
hipError_t launch_gated_quantize(fqt_dtype type, const GatedQuantParams& p, const Fp8Turn& a, const Fp8Turn& b,
                                 hipStream_t s);

// ---------------------------------------------------------------------------
// gradient norm and clipping
// ---------------------------------------------------------------------------
// Tensors of one launch: their table travels in the kernel's arguments (4 KB),
// so nothing is copied to the device beforehand.
constexpr int CLIP_TENSORS = 168;
constexpr int CLIP_PARTS = 1024;        // partial sums of one launch
constexpr int64_t CLIP_BYTES = 16384;   // a chunk: one block's turn
struct ClipTable {
  const void* g[CLIP_TENSORS];  // none of them empty
  void* out[CLIP_TENSORS];
  uint32_t first[CLIP_TENSORS + 1];  // first chunk of each tensor
  uint16_t tail[CLIP_TENSORS];       // bytes of its last chunk
  uint8_t type[CLIP_TENSORS];
  int count;
};
static_assert(sizeof(ClipTable) <= 4000, "kernel arguments");
hipError_t launch_clip_norm(const ClipTable& t, double* part, hipStream_t s);
hipError_t launch_clip_scale(const ClipTable& t, const double* part, int64_t parts, double max_norm, float* norm,
                             hipStream_t s);

}  // namespace fqt
