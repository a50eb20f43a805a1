// C ABI of the floating-point operators around the layers (include/fqt.h):
// argument checks, workspace carving and launch sequences.
#include <math.h>
#include <stdint.h>

#include "../../include/fqt.h"
#include "train_kernels.h"

namespace fqt {
namespace {

struct Carver {
  char* base;
  size_t off = 0;
  explicit Carver(void* b) : base(static_cast<char*>(b)) {}
  template <class T>
  T* take(int64_t count) {
    off = (off + 255) & ~(size_t)255;
    T* p = base ? reinterpret_cast<T*>(base + off) : nullptr;
    off += (size_t)count * sizeof(T);
    return p;
  }
};

constexpr int64_t MAX_SIDE = (int64_t)1 << 31;   // rows or columns of a matrix
bool side(int64_t n) { return n >= 1 && n < MAX_SIDE; }
// the products address a tile of 256 rows of codes with 31-bit offsets
constexpr int64_t MAX_CONTRACTION = (int64_t)1 << 23;
size_t type_bytes(fqt_dtype t) { return t == FQT_F32 ? 4 : 2; }
bool aligned(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }
// an input matrix: element-aligned; its rows may overlap (ld 0: one row for all)
bool input(const void* p, fqt_dtype t, int64_t ld) {
  return p && aligned(p, type_bytes(t)) && ld >= 0 && ld < ((int64_t)1 << 40);
}
// an output matrix: its rows are at least cols apart
bool output(const void* p, fqt_dtype t, int64_t cols, int64_t ld) { return input(p, t, ld) && ld >= cols; }
bool operand(const fqt_fp8* a) {
  return a && a->q && a->exp && aligned(a->q, 16) && aligned(a->exp, 4) && (a->k_major == 0 || a->k_major == 1);
}
// one that a call writes: row by row only
bool written(const fqt_fp8* a) { return operand(a) && a->k_major == 0; }

#define FQT_TRY(expr)                              \
  do {                                             \
    const hipError_t e_ = (expr);                  \
    if (e_ != hipSuccess) return FQT_EDEVICE;      \
  } while (0)

struct Fp8Buffers {
  uint8_t *q, *e;
};
Fp8Buffers take_operand(Carver& c, int64_t rows, int64_t K) {
  Fp8Buffers b;
  b.q = c.take<uint8_t>(rows * fp8_pitch(K));
  b.e = c.take<uint8_t>(fp8_exp_bytes(rows, K));
  return b;
}

// An operand's codes row by row: its own, or laid out in `room` by `turn`.
const uint8_t* rows_of(const fqt_fp8* a, int64_t rows, int64_t K, uint8_t* room, Fp8Turn* turn) {
  if (!a->k_major) return a->q;
  *turn = Fp8Turn{a->q, rows, K, room};
  return room;
}

struct GemmWs {
  uint8_t *a, *b;  // room for operands that come column by column
  float* part;
};
GemmWs carve_gemm(Carver& c, int64_t M, int64_t N, int64_t K) {
  GemmWs w;
  w.a = c.take<uint8_t>(M * fp8_pitch(K));
  w.b = c.take<uint8_t>(N * fp8_pitch(K));
  w.part = c.take<float>(fp8_gemm_partials(M, N, K));
  return w;
}
struct ForwardWs {
  Fp8Buffers x;
  uint8_t* w;
  float* part;
};
ForwardWs carve_forward(Carver& c, int64_t N, int64_t d_in, int64_t d_out) {
  ForwardWs w;
  w.w = c.take<uint8_t>(d_out * fp8_pitch(d_in));
  w.x = take_operand(c, N, d_in);
  w.part = c.take<float>(fp8_gemm_partials(N, d_out, d_in));
  return w;
}
struct BackwardWs {
  Fp8Buffers g, gt;
  uint8_t *x, *w;
  float* part;
};
// The two products run one behind the other and share their partial sums.
BackwardWs carve_backward(Carver& c, int64_t N, int64_t d_in, int64_t d_out) {
  BackwardWs w;
  w.g = take_operand(c, N, d_out);
  w.gt = take_operand(c, d_out, N);
  w.x = c.take<uint8_t>(d_in * fp8_pitch(N));
  w.w = c.take<uint8_t>(d_in * fp8_pitch(d_out));
  const int64_t a = fp8_gemm_partials(N, d_in, d_out), b = fp8_gemm_partials(d_out, d_in, N);
  w.part = c.take<float>(a > b ? a : b);
  return w;
}

}  // namespace
}  // namespace fqt

using namespace fqt;

extern "C" {

// ---------------------------------------------------------------------------
// layer norm
// ---------------------------------------------------------------------------
fqt_status fqt_layernorm_forward(const void* X, fqt_dtype type, int64_t rows, int64_t cols, int64_t ldx,
                                 const float* gamma, const float* beta, float eps, void* Y, int64_t ldy, float* mean,
                                 float* rstd, fqt_stream_t s) {
  if (!valid_type(type) || !side(rows) || !side(cols) || !(eps >= 0.0f) || !isfinite(eps)) return FQT_EINVAL;
  if (!input(X, type, ldx) || !output(Y, type, cols, ldy)) return FQT_EINVAL;
  if (!aligned(gamma, 4) || !aligned(beta, 4) || !aligned(mean, 4) || !aligned(rstd, 4)) return FQT_EINVAL;
  NormParams p{};
  p.x = X;
  p.ldx = ldx;
  p.rows = rows;
  p.cols = cols;
  p.gamma = gamma;
  p.beta = beta;
  p.eps = eps;
  p.y = Y;
  p.ldy = ldy;
  p.mean = mean;
  p.rstd = rstd;
  FQT_TRY(launch_norm_forward(type, p, s));
  return FQT_OK;
}

size_t fqt_layernorm_backward_workspace(int64_t rows, int64_t cols) {
  if (!side(rows) || !side(cols)) return 0;
  return (size_t)norm_backward_partials(rows, cols) * sizeof(float);
}

fqt_status fqt_layernorm_backward(const void* G, int64_t ldg, const void* X, int64_t ldx, fqt_dtype type, int64_t rows,
                                  int64_t cols, const float* mean, const float* rstd, const float* gamma, void* grad_X,
                                  int64_t ldgx, float* grad_gamma, float* grad_beta, void* ws, size_t ws_bytes,
                                  fqt_stream_t s) {
  if (!valid_type(type) || !side(rows) || !side(cols) || !mean || !rstd) return FQT_EINVAL;
  if (!input(G, type, ldg) || !input(X, type, ldx) || !output(grad_X, type, cols, ldgx))
    return FQT_EINVAL;
  if (!aligned(gamma, 4) || !aligned(mean, 4) || !aligned(rstd, 4) || !aligned(grad_gamma, 4) ||
      !aligned(grad_beta, 4))
    return FQT_EINVAL;
  if (grad_gamma || grad_beta) {
    if (!ws || !aligned(ws, 16) || ws_bytes < fqt_layernorm_backward_workspace(rows, cols)) return FQT_EWORKSPACE;
  }
  NormParams p{};
  p.g = G;
  p.ldg = ldg;
  p.x = X;
  p.ldx = ldx;
  p.rows = rows;
  p.cols = cols;
  p.mean = const_cast<float*>(mean);
  p.rstd = const_cast<float*>(rstd);
  p.gamma = gamma;
  p.y = grad_X;
  p.ldy = ldgx;
  p.grad_gamma = grad_gamma;
  p.grad_beta = grad_beta;
  p.part = static_cast<float*>(ws);
  FQT_TRY(launch_norm_backward(type, p, s));
  return FQT_OK;
}

// ---------------------------------------------------------------------------
// 8-bit floating point layers
// ---------------------------------------------------------------------------
size_t fqt_fp8_pitch(int64_t K) { return side(K) ? (size_t)fp8_pitch(K) : 0; }
size_t fqt_fp8_exp_bytes(int64_t rows, int64_t K) { return side(rows) && side(K) ? (size_t)fp8_exp_bytes(rows, K) : 0; }

fqt_status fqt_fp8_quantize(const void* x, fqt_dtype type, int64_t rows, int64_t cols, int64_t ldx, int tile,
                            int stochastic, uint64_t seed, const fqt_fp8* by_row, const fqt_fp8* by_col,
                            fqt_stream_t s) {
  if (!valid_type(type) || !side(rows) || !side(cols) || !input(x, type, ldx)) return FQT_EINVAL;
  if ((tile != 0 && tile != 1) || (stochastic != 0 && stochastic != 1) || (!by_row && !by_col)) return FQT_EINVAL;
  if ((by_row && !written(by_row)) || (by_col && !written(by_col))) return FQT_EINVAL;
  Fp8QuantParams p{};
  p.x = x;
  p.rows = rows;
  p.cols = cols;
  p.ldx = ldx;
  p.tile = tile;
  p.stochastic = stochastic;
  p.seed = seed;
  if (by_row) {
    p.q_row = by_row->q;
    p.e_row = by_row->exp;
  }
  if (by_col) {
    p.q_col = by_col->q;
    p.e_col = by_col->exp;
  }
  FQT_TRY(launch_fp8_quantize(type, p, s));
  return FQT_OK;
}

size_t fqt_fp8_gemm_workspace(int64_t M, int64_t N, int64_t K) {
  if (!side(M) || !side(N) || !side(K)) return 0;
  Carver c(nullptr);
  carve_gemm(c, M, N, K);
  return c.off;
}

fqt_status fqt_fp8_gemm(const fqt_fp8* A, const fqt_fp8* B, int64_t M, int64_t N, int64_t K, fqt_dtype type, int relu,
                        const void* mask, int64_t ldmask, void* C, int64_t ldc, void* ws, size_t ws_bytes,
                        fqt_stream_t s) {
  if (!valid_type(type) || !side(M) || !side(N) || !side(K) || !operand(A) || !operand(B)) return FQT_EINVAL;
  if (!output(C, type, N, ldc) || (mask && !input(mask, type, ldmask)) || (relu != 0 && relu != 1))
    return FQT_EINVAL;
  if (K > MAX_CONTRACTION) return FQT_EUNSUPPORTED;
  if (!ws || !aligned(ws, 16) || ws_bytes < fqt_fp8_gemm_workspace(M, N, K)) return FQT_EWORKSPACE;
  Carver c(ws);
  const GemmWs w = carve_gemm(c, M, N, K);
  Fp8GemmParams p{};
  Fp8Turn a{}, b{};
  p.A = rows_of(A, M, K, w.a, &a);
  p.eA = A->exp;
  p.B = rows_of(B, N, K, w.b, &b);
  p.eB = B->exp;
  FQT_TRY(launch_fp8_turn(a, s));
  FQT_TRY(launch_fp8_turn(b, s));
  p.M = M;
  p.N = N;
  p.K = K;
  p.C = C;
  p.ldc = ldc;
  p.relu = relu;
  p.mask = mask;
  p.ldmask = ldmask;
  p.part = w.part;
  FQT_TRY(launch_fp8_gemm(type, p, s));
  return FQT_OK;
}

int32_t fqt_fp8_gemm_form(int64_t M, int64_t N, int64_t K, int masked, int lines) {
  if (!side(M) || !side(N) || !side(K) || K > MAX_CONTRACTION) return -1;
  return fp8_gemm_form(M, N, K, masked != 0, lines != 0);
}

size_t fqt_fp8_linear_forward_workspace(int64_t N, int64_t d_in, int64_t d_out) {
  if (!side(N) || !side(d_in) || !side(d_out)) return 0;
  Carver c(nullptr);
  carve_forward(c, N, d_in, d_out);
  return c.off;
}

fqt_status fqt_fp8_linear_forward(const void* X, fqt_dtype type, int64_t N, int64_t d_in, int64_t ldx,
                                  const fqt_fp8* W8, int64_t d_out, int relu, void* Y, int64_t ldy,
                                  const fqt_fp8* X8t, void* ws, size_t ws_bytes, fqt_stream_t s) {
  if (!valid_type(type) || !side(N) || !side(d_in) || !side(d_out) || !operand(W8)) return FQT_EINVAL;
  if (!input(X, type, ldx) || !output(Y, type, d_out, ldy) || (relu != 0 && relu != 1)) return FQT_EINVAL;
  if (X8t && !written(X8t)) return FQT_EINVAL;
  if (d_in > MAX_CONTRACTION) return FQT_EUNSUPPORTED;
  if (!ws || !aligned(ws, 16) || ws_bytes < fqt_fp8_linear_forward_workspace(N, d_in, d_out)) return FQT_EWORKSPACE;
  Carver c(ws);
  const ForwardWs w = carve_forward(c, N, d_in, d_out);
  // few rows are quantized by the product itself
  const bool raw = fp8_rows_raw(N);
  Fp8QuantParams q{};
  q.x = X;
  q.rows = N;
  q.cols = d_in;
  q.ldx = ldx;
  if (!raw) {
    q.q_row = w.x.q;
    q.e_row = w.x.e;
  }
  if (X8t) {
    q.q_col = X8t->q;
    q.e_col = X8t->exp;
  }
  Fp8GemmParams p{};
  Fp8Turn turn{};
  p.A = w.x.q;
  p.eA = w.x.e;
  p.B = rows_of(W8, d_out, d_in, w.w, &turn);
  p.eB = W8->exp;
  FQT_TRY(launch_fp8_quantize_turn(type, q, turn, Fp8Turn{}, s));
  p.M = N;
  p.N = d_out;
  p.K = d_in;
  p.C = Y;
  p.ldc = ldy;
  p.relu = relu;
  p.part = w.part;
  if (raw)
    FQT_TRY(launch_fp8_rows(type, p, X, ldx, s));
  else
    FQT_TRY(launch_fp8_gemm(type, p, s));
  return FQT_OK;
}

size_t fqt_fp8_linear_backward_workspace(int64_t N, int64_t d_in, int64_t d_out) {
  if (!side(N) || !side(d_in) || !side(d_out)) return 0;
  Carver c(nullptr);
  carve_backward(c, N, d_in, d_out);
  return c.off;
}

fqt_status fqt_fp8_linear_backward(const void* G, fqt_dtype type, int64_t N, int64_t d_out, int64_t ldg,
                                   const fqt_fp8* X8t, const fqt_fp8* W8t, int64_t d_in, int stochastic, uint64_t seed,
                                   const void* relu_input, int64_t ldr, float* grad_W, void* grad_X, int64_t ldgx,
                                   void* ws, size_t ws_bytes, fqt_stream_t s) {
  if (!valid_type(type) || !side(N) || !side(d_in) || !side(d_out) || !input(G, type, ldg)) return FQT_EINVAL;
  if ((!grad_W && !grad_X) || (stochastic != 0 && stochastic != 1)) return FQT_EINVAL;
  if (grad_W && (!operand(X8t) || !aligned(grad_W, 4))) return FQT_EINVAL;
  if (grad_X && (!operand(W8t) || !output(grad_X, type, d_in, ldgx))) return FQT_EINVAL;
  if (relu_input && !input(relu_input, type, ldr)) return FQT_EINVAL;
  if ((grad_W && N > MAX_CONTRACTION) || (grad_X && d_out > MAX_CONTRACTION)) return FQT_EUNSUPPORTED;
  if (!ws || !aligned(ws, 16) || ws_bytes < fqt_fp8_linear_backward_workspace(N, d_in, d_out)) return FQT_EWORKSPACE;
  Carver c(ws);
  const BackwardWs w = carve_backward(c, N, d_in, d_out);
  Fp8QuantParams q{};
  q.x = G;
  q.rows = N;
  q.cols = d_out;
  q.ldx = ldg;
  q.stochastic = stochastic;
  q.seed = seed;
  if (grad_X) {
    q.q_row = w.g.q;
    q.e_row = w.g.e;
  }
  if (grad_W) {
    q.q_col = w.gt.q;
    q.e_col = w.gt.e;
  }
  Fp8Turn turn_x{}, turn_w{};
  const uint8_t* const x8 = grad_W ? rows_of(X8t, d_in, N, w.x, &turn_x) : nullptr;
  const uint8_t* const w8 = grad_X ? rows_of(W8t, d_in, d_out, w.w, &turn_w) : nullptr;
  FQT_TRY(launch_fp8_quantize_turn(type, q, turn_x, turn_w, s));
  Fp8GemmParams p{};
  p.part = w.part;
  p.N = d_in;
  if (grad_W) {
    p.A = w.gt.q;
    p.eA = w.gt.e;
    p.B = x8;
    p.eB = X8t->exp;
    p.M = d_out;
    p.K = N;
    p.C = grad_W;
    p.ldc = d_in;
    FQT_TRY(launch_fp8_gemm(FQT_F32, p, s));
  }
  if (grad_X) {
    p.A = w.g.q;
    p.eA = w.g.e;
    p.B = w8;
    p.eB = W8t->exp;
    p.M = N;
    p.K = d_out;
    p.C = grad_X;
    p.ldc = ldgx;
    p.mask = relu_input;
    p.ldmask = ldr;
    FQT_TRY(launch_fp8_gemm(type, p, s));
  }
  return FQT_OK;
}

// ---------------------------------------------------------------------------
// gradient norm and clipping
// ---------------------------------------------------------------------------
size_t fqt_grad_norm_clip_workspace(int64_t count) {
  if (count < 1 || count > MAX_SIDE) return 0;
  return (size_t)((count + CLIP_TENSORS - 1) / CLIP_TENSORS) * CLIP_PARTS * sizeof(double);
}

fqt_status fqt_grad_norm_clip(const void* const* grads, void* const* outs, const int64_t* sizes, const int32_t* types,
                              int64_t count, double max_norm, float* norm, void* ws, size_t ws_bytes, fqt_stream_t s) {
  if (!grads || !sizes || !types || count < 1 || count > MAX_SIDE) return FQT_EINVAL;
  if (!(max_norm > 0.0) || !aligned(norm, 4)) return FQT_EINVAL;
  for (int64_t i = 0; i < count; ++i) {
    const fqt_dtype t = (fqt_dtype)types[i];
    if (!valid_type(t) || sizes[i] < 0 || sizes[i] > ((int64_t)1 << 40)) return FQT_EINVAL;
    if (sizes[i] == 0) continue;
    if (!grads[i] || !aligned(grads[i], type_bytes(t))) return FQT_EINVAL;
    if (outs && (!outs[i] || !aligned(outs[i], type_bytes(t)))) return FQT_EINVAL;
  }
  if (!ws || !aligned(ws, 16) || ws_bytes < fqt_grad_norm_clip_workspace(count)) return FQT_EWORKSPACE;
  double* part = static_cast<double*>(ws);
  // tables of up to CLIP_TENSORS tensors that are not empty; next: where the following one begins
  auto table = [&](int64_t& next, ClipTable& t) {
    t.count = 0;
    uint64_t chunks = 0;
    for (; next < count && t.count < CLIP_TENSORS; ++next) {
      if (sizes[next] == 0) continue;
      const int k = t.count++;
      const uint64_t bytes = (uint64_t)sizes[next] * type_bytes((fqt_dtype)types[next]);
      const uint64_t n = (bytes + CLIP_BYTES - 1) / CLIP_BYTES;
      t.g[k] = grads[next];
      t.out[k] = outs ? outs[next] : const_cast<void*>(grads[next]);
      t.type[k] = (uint8_t)types[next];
      t.tail[k] = (uint16_t)(bytes - (n - 1) * CLIP_BYTES);
      t.first[k] = (uint32_t)chunks;
      chunks += n;
      if (chunks > 0x7FFFFFFFu) return false;
    }
    t.first[t.count] = (uint32_t)chunks;
    return true;
  };
  ClipTable t;
  int64_t launches = 0, next = 0;
  while (next < count || launches == 0) {
    if (!table(next, t)) return FQT_EUNSUPPORTED;
    ++launches;
  }
  next = 0;
  for (int64_t l = 0; l < launches; ++l) {
    table(next, t);
    FQT_TRY(launch_clip_norm(t, part + l * CLIP_PARTS, s));
  }
  next = launches == 1 ? count : 0;  // one table serves both
  for (int64_t l = 0; l < launches; ++l) {
    if (launches > 1) table(next, t);
    FQT_TRY(launch_clip_scale(t, part, launches * CLIP_PARTS, max_norm, l == 0 ? norm : nullptr, s));
  }
  return FQT_OK;
}

}  // extern "C"
