// Layer norm over the last axis, forward and backward.
//
//   mean = 1/D sum x,  var = 1/D sum (x - mean)^2,  r = 1 / sqrt(var + eps)
//   xh = (x - mean) r,  y = xh gamma + beta
//   c = g gamma,  gx = r (c - mean(c) - xh mean(c xh))
//   ggamma = sum over rows of g xh,  gbeta = sum over rows of g
//
// A team of threads (a wave, or a block) holds its whole row in registers:
// one read of each input, one write of each output.  Statistics, sums and
// parameter gradients are float32; the outputs are rounded once.
//
// Forward, 8192 x 4096 float32 (268 MB): 51 us, 5.3 TB/s, a large copy's rate;
// memory bounds it.  Backward, 8192 x 1024 bfloat16 (50 MB): 15.4 us, 3.3 TB/s,
// and 3.8 us for the partial sums; two rows a wave, whose waves wait three
// quarters of the time for their loads.  float32 (101 MB): 24.0 us, 4.2 TB/s, waits
// half of the time.  One row of 4096 bfloat16 forward: 3.0 us, a launch and a chain
// of latencies.
//
// With a checkpoint of xh in 8 bits, E + 127 and codes of each block of 32 along a
// row: the forward finds the blocks' scales across neighbouring lanes of the team,
// the backward reads one byte an element in place of x.  8192 x 1024 bfloat16 (42 MB)
// forward 11.4 us, 3.7 TB/s; backward 12.6 us, 3.3 TB/s, and 3.8 us for the partial
// sums.  8192 x 4096 float32 backward (303 MB): 58 us, 5.2
// TB/s, a large copy's rate.
#include "fp8_codes.h"

namespace fqt {

// Elements of a row that each thread of a team of TPR threads holds: NV
// vectors of VEC, vector v at column (v TPR + t) VEC.
template <int TPR_, int VEC_, int NV_, int THREADS_ = TPR_ < 256 ? 256 : TPR_>
struct Team {
  static constexpr int TPR = TPR_, VEC = VEC_, NV = NV_, THREADS = THREADS_;
  static constexpr int PER_BLOCK = THREADS / TPR;  // rows at a time
  static constexpr int WAVES = TPR / 64;
  static constexpr int64_t COLS = (int64_t)TPR * VEC * NV;
};

// Sums of N values over the team, in every thread.  sh: the team's [WAVES][N];
// teams of several waves meet at block barriers, which every team of the block
// has to reach.
template <class C, int N>
__device__ __forceinline__ void team_sum(float (&v)[N], float (*sh)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = wave_sum(v[i]);
  if constexpr (C::WAVES > 1) {
    const int wave = threadIdx.x % C::TPR >> 6;
    __syncthreads();  // the last sums have been read
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int i = 0; i < N; ++i) sh[wave][i] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      v[i] = 0.0f;
#pragma unroll
      for (int w = 0; w < C::WAVES; ++w) v[i] += sh[w][i];
    }
  }
}

// ---------------------------------------------------------------------------
// Checkpoints of xh: V neighbouring elements a thread, so that the threads of a
// block of 32 are neighbours in a wave (and all of them, or none, come here).
// ---------------------------------------------------------------------------
template <int V>
struct CodesOf {
  typedef uint8_t type __attribute__((ext_vector_type(V), aligned(V)));
};
// The thread's codes of v at column col of a row; values past the row are 0.
template <int V>
__device__ __forceinline__ void keep_codes(uint8_t* q, uint8_t* e, int64_t cols, int64_t col, const float (&v)[V]) {
  static_assert(V == 2 || V == 4 || V == 8, "16, 8 or 4 threads a block");
  uint32_t key = 0u;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const uint32_t m = __float_as_uint(v[i]) & 0x7fffffffu;
    key = key > m ? key : m;
  }
  auto larger = [](uint32_t a, uint32_t b) { return a > b ? a : b; };
  key = larger(key, dpp<0xB1>(key));                         // lanes 1, 0, 3, 2 of four
  key = larger(key, dpp<0x4E>(key));                         // lanes 2, 3, 0, 1
  if constexpr (V <= 4) key = larger(key, dpp<0x141>(key));  // eight lanes reversed
  if constexpr (V == 2) key = larger(key, dpp<0x140>(key));  // sixteen lanes reversed
  key = Quad<float>::key(key);
  if (col >= kept_pitch(cols)) return;
  const uint32_t byte = scale_bytes(key) & 0xffffu;
  const float scale = scale_up(byte);
  typename CodesOf<V>::type w;
#pragma unroll
  for (int i = 0; i < V; i += 2) {
    const s16x2 c = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(s16x2{0, 0}, v[i], v[i + 1], scale, false);
    const uint32_t both = key >= NAN_KEY ? 0x7f7fu : as<uint32_t>(c);
    w[i] = (uint8_t)both;
    w[i + 1] = (uint8_t)(both >> 8);
  }
  *reinterpret_cast<typename CodesOf<V>::type*>(q + col) = w;
  if (col % KEPT_BLOCK == 0) e[col / KEPT_BLOCK] = stored_byte(key, byte);
}
// What the checkpoint has there: 0 past the row.
template <int V>
__device__ __forceinline__ void kept_values(const uint8_t* q, const uint8_t* e, int64_t n, int64_t col, float (&v)[V]) {
  if (n <= 0) {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = 0.0f;
    return;
  }
  const auto w = *reinterpret_cast<const typename CodesOf<V>::type*>(q + col);
  const float scale = scale_up(e[col / KEPT_BLOCK]);
#pragma unroll
  for (int i = 0; i < V; i += 2) {
    const auto f = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[i] | (uint32_t)w[i + 1] << 8, scale, false);
    v[i] = i < n ? f[0] : 0.0f;
    v[i + 1] = i + 1 < n ? f[1] : 0.0f;
  }
}

template <class T, class C>
__global__ __launch_bounds__(C::THREADS) void norm_forward_kernel(NormParams p) {
  __shared__ float sh[C::WAVES][1];
  const int t = threadIdx.x % C::TPR;
  const int64_t row = block_id() * C::PER_BLOCK + threadIdx.x / C::TPR;
  if (row >= p.rows) return;  // whole waves and no barrier below, or whole blocks
  const T* x = static_cast<const T*>(p.x) + row * p.ldx;
  float v[C::NV][C::VEC];
  float s[1] = {0.0f};
#pragma unroll
  for (int k = 0; k < C::NV; ++k) {
    const int64_t col = (int64_t)(k * C::TPR + t) * C::VEC;
    load_part<T, C::VEC>(x + col, p.cols - col, v[k]);
  }
#pragma unroll
  for (int k = 0; k < C::NV; ++k)
#pragma unroll
    for (int i = 0; i < C::VEC; ++i) s[0] += v[k][i];
  team_sum<C, 1>(s, sh);
  const float inv = 1.0f / (float)p.cols;
  const float mean = s[0] * inv;
  s[0] = 0.0f;
#pragma unroll
  for (int k = 0; k < C::NV; ++k) {
    const int64_t col = (int64_t)(k * C::TPR + t) * C::VEC;
#pragma unroll
    for (int i = 0; i < C::VEC; ++i) {
      const float d = col + i < p.cols ? v[k][i] - mean : 0.0f;
      s[0] = fmaf(d, d, s[0]);
    }
  }
  team_sum<C, 1>(s, sh);
  const float rstd = 1.0f / sqrtf(fmaf(s[0], inv, p.eps));
  if (t == 0) {
    if (p.mean) p.mean[row] = mean;
    if (p.rstd) p.rstd[row] = rstd;
  }
  T* y = static_cast<T*>(p.y) + row * p.ldy;
#pragma unroll
  for (int k = 0; k < C::NV; ++k) {
    const int64_t col = (int64_t)(k * C::TPR + t) * C::VEC;
    float ga[C::VEC], be[C::VEC], o[C::VEC];
#pragma unroll
    for (int i = 0; i < C::VEC; ++i) {
      ga[i] = 1.0f;
      be[i] = 0.0f;
    }
    if (p.gamma) load_part<float, C::VEC>(p.gamma + col, p.cols - col, ga);
    if (p.beta) load_part<float, C::VEC>(p.beta + col, p.cols - col, be);
#pragma unroll
    for (int i = 0; i < C::VEC; ++i) o[i] = fmaf((v[k][i] - mean) * rstd, ga[i], be[i]);
    store_part<T, C::VEC>(y + col, p.cols - col, o);
  }
}

// A vector of V elements of a row, as it lies in memory.  No branch around a load
// (it would wait for the others): vectors that are not whole are read from the
// row's end, and moved down by `value`.  SHORT: the row may be shorter than one.
template <class T, int V, bool SHORT>
struct RowVec {
  static constexpr int W = V * (int)sizeof(T) / 4;
  uint32_t w[W];
  __device__ __forceinline__ void load(const T* row, int col, int cols) {
    typedef uint32_t words __attribute__((ext_vector_type(W), aligned(sizeof(T))));
    const int last = cols - V, from = col < last ? col : last;
    words x;
    if (SHORT && last < 0) {  // all in the first vector
      T e[V];
#pragma unroll
      for (int i = 0; i < V; ++i) e[i] = row[i < cols ? i : cols - 1];
      __builtin_memcpy(&x, e, sizeof(x));
    } else {
      x = *reinterpret_cast<const words*>(row + from);
    }
#pragma unroll
    for (int i = 0; i < W; ++i) w[i] = x[i];
  }
  // left: the row's columns from the vector's first on; 0 past the row.
  __device__ __forceinline__ void value(int left, int cols, float (&v)[V]) const {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] = __uint_as_float(left > 0 ? w[i] : 0u);
    } else {
      typedef T pair __attribute__((ext_vector_type(2)));
#pragma unroll
      for (int i = 0; i < V; i += 2) {
        const pair two = as<pair>(left > 0 ? w[i / 2] : 0u);
        v[i] = (float)two[0];
        v[i + 1] = (float)two[1];
      }
    }
    if (cols % V != 0 && left < V) {
      const int past = SHORT && cols < V ? 0 : V - left;
#pragma unroll
      for (int d = V / 2; d > 0; d /= 2) {  // down by past, bit by bit
        const bool move = past > 0 && (past & d);
#pragma unroll
        for (int i = 0; i + d < V; ++i) {
          const float up = v[i + d], here = v[i];
          v[i] = move ? up : here;  // (of v[...] themselves it would choose the address)
        }
      }
#pragma unroll
      for (int i = 1; i < V; ++i) v[i] = i < left ? v[i] : 0.0f;
    }
  }
};

// With the checkpoint of xh.  All loads are under way before the first sum: 8192 x
// 1024 bfloat16 11.4 us, 12.5 with gamma and beta loaded when they are needed and
// branches at the row's end (float32 13.4, 15.2); 70 registers, seven waves a SIMD
// (held to 64 the loads wait for spilled registers: 15.4).
template <class T, class C>
__global__ __launch_bounds__(C::THREADS) void norm_forward8_kernel(NormParams p) {
  __shared__ float sh[C::WAVES][1];
  constexpr int V = C::VEC, NV = C::NV;
  constexpr bool SHORT = C::COLS <= 64 * 4;
  const int t = threadIdx.x % C::TPR, cols = (int)p.cols;
  const int64_t row = block_id() * C::PER_BLOCK + threadIdx.x / C::TPR;
  if (row >= p.rows) return;  // whole waves and no barrier below, or whole blocks
  RowVec<T, V, SHORT> x[NV];
  RowVec<float, V, SHORT> ga[NV], be[NV];
#pragma unroll
  for (int k = 0; k < NV; ++k) x[k].load(static_cast<const T*>(p.x) + row * p.ldx, (k * C::TPR + t) * V, cols);
  if (p.gamma) {
#pragma unroll
    for (int k = 0; k < NV; ++k) ga[k].load(p.gamma, (k * C::TPR + t) * V, cols);
  }
  if (p.beta) {
#pragma unroll
    for (int k = 0; k < NV; ++k) be[k].load(p.beta, (k * C::TPR + t) * V, cols);
  }
  float v[NV][V];
  float s[1] = {0.0f};
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    x[k].value(cols - (k * C::TPR + t) * V, cols, v[k]);
#pragma unroll
    for (int i = 0; i < V; ++i) s[0] += v[k][i];
  }
  team_sum<C, 1>(s, sh);
  const float inv = 1.0f / (float)p.cols;
  const float mean = s[0] * inv;
  s[0] = 0.0f;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int col = (k * C::TPR + t) * V;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float d = col + i < cols ? v[k][i] - mean : 0.0f;
      s[0] = fmaf(d, d, s[0]);
    }
  }
  team_sum<C, 1>(s, sh);
  const float rstd = 1.0f / sqrtf(fmaf(s[0], inv, p.eps));
  if (t == 0) p.rstd[row] = rstd;
  T* const y = static_cast<T*>(p.y) + row * p.ldy;
  const int64_t pitch = kept_pitch(p.cols);
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int col = (k * C::TPR + t) * V;
    float a[V], b[V], o[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      a[i] = 1.0f;
      b[i] = 0.0f;
    }
    if (p.gamma) ga[k].value(cols - col, cols, a);
    if (p.beta) be[k].value(cols - col, cols, b);
#pragma unroll
    for (int i = 0; i < V; ++i) v[k][i] = col + i < cols ? (v[k][i] - mean) * rstd : 0.0f;
    keep_codes<V>(p.q8 + row * pitch, p.e8 + row * (pitch / KEPT_BLOCK), p.cols, col, v[k]);
#pragma unroll
    for (int i = 0; i < V; ++i) o[i] = fmaf(v[k][i], a[i], b[i]);
    store_part<T, V>(y + col, cols - col, o);
  }
}

// Rows longer than a team's registers: the row is read three times (sum,
// squares, output), the later ones from the caches.
template <class T, class C, bool KEEP>
__global__ __launch_bounds__(C::THREADS) void norm_forward_long_kernel(NormParams p) {
  __shared__ float sh[C::WAVES][1];
  const int64_t row = block_id();
  if (row >= p.rows) return;
  const T* x = static_cast<const T*>(p.x) + row * p.ldx;
  const int64_t step = (int64_t)C::TPR * C::VEC, first = (int64_t)threadIdx.x * C::VEC;
  float v[C::VEC];
  float s[1] = {0.0f};
  for (int64_t col = first; col < p.cols; col += step) {
    load_part<T, C::VEC>(x + col, p.cols - col, v);
#pragma unroll
    for (int i = 0; i < C::VEC; ++i) s[0] += v[i];
  }
  team_sum<C, 1>(s, sh);
  const float inv = 1.0f / (float)p.cols;
  const float mean = s[0] * inv;
  s[0] = 0.0f;
  for (int64_t col = first; col < p.cols; col += step) {
    load_part<T, C::VEC>(x + col, p.cols - col, v);
#pragma unroll
    for (int i = 0; i < C::VEC; ++i) {
      const float d = col + i < p.cols ? v[i] - mean : 0.0f;
      s[0] = fmaf(d, d, s[0]);
    }
  }
  team_sum<C, 1>(s, sh);
  const float rstd = 1.0f / sqrtf(fmaf(s[0], inv, p.eps));
  if (threadIdx.x == 0) {
    if (p.mean) p.mean[row] = mean;
    if (p.rstd) p.rstd[row] = rstd;
  }
  T* y = static_cast<T*>(p.y) + row * p.ldy;
  const int64_t pitch = kept_pitch(p.cols);
  for (int64_t col = first; col < (KEEP ? pitch : p.cols); col += step) {  // KEEP: whole blocks stay together
    load_part<T, C::VEC>(x + col, p.cols - col, v);
#pragma unroll
    for (int i = 0; i < C::VEC; ++i) v[i] = col + i < p.cols ? (v[i] - mean) * rstd : 0.0f;
    if constexpr (KEEP)
      keep_codes<C::VEC>(p.q8 + row * pitch, p.e8 + row * (pitch / KEPT_BLOCK), p.cols, col, v);
#pragma unroll
    for (int i = 0; i < C::VEC; ++i)
      if (col + i < p.cols) v[i] = fmaf(v[i], p.gamma ? p.gamma[col + i] : 1.0f, p.beta ? p.beta[col + i] : 0.0f);
    store_part<T, C::VEC>(y + col, p.cols - col, v);
  }
}

// Backward from the checkpoint.  The codes and G wait in registers as they were
// loaded, a row ahead of the arithmetic, and codes are decoded twice: for the sums
// and for the output.  Rows of one vector at least.
template <class T, class C>
struct KeptRow {
  static constexpr int V = C::VEC, QW = (V + 3) / 4;  // words of a vector's codes
  RowVec<T, V, false> g[C::NV];
  uint32_t q[C::NV][QW], e[C::NV];
  float rstd;
  __device__ __forceinline__ void load(const NormParams& p, int64_t row, int t) {
    const int64_t pitch = kept_pitch(p.cols);
    const T* const gr = static_cast<const T*>(p.g) + row * p.ldg;
    const uint8_t* const qr = p.q8 + row * pitch;
    const uint8_t* const er = p.e8 + row * (pitch / KEPT_BLOCK);
    const int cols = (int)p.cols, width = (int)pitch;
#pragma unroll
    for (int k = 0; k < C::NV; ++k) {
      const int col = (k * C::TPR + t) * V, at = col < width ? col : 0;
      if constexpr (V == 2) {
        q[k][0] = *reinterpret_cast<const uint16_t*>(qr + at);
      } else {
#pragma unroll
        for (int i = 0; i < QW; ++i) q[k][i] = *reinterpret_cast<const uint32_t*>(qr + at + 4 * i);
      }
      e[k] = er[at / KEPT_BLOCK];
      g[k].load(gr, col, cols);
    }
    rstd = p.rstd[row];
  }
  __device__ __forceinline__ void xhat(int k, float (&v)[V]) const {
    const float scale = scale_up(e[k]);
#pragma unroll
    for (int i = 0; i < V; i += 2) {
      const auto f = (i & 2) ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(q[k][i / 4], scale, true)
                             : __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(q[k][i / 4], scale, false);
      v[i] = f[0];
      v[i + 1] = f[1];
    }
  }
};

// The rows of a team: grad_X, and the sums sg and sb from 0.
template <class T, class C>
__device__ __forceinline__ void kept_rows(const NormParams& p, float (&sh)[C::PER_BLOCK][C::WAVES][2],
                                          float (&sg)[C::NV][C::VEC], float (&sb)[C::NV][C::VEC]) {
  // a team is whole waves: its row's addresses stay scalar
  const int t = threadIdx.x % C::TPR, team = __builtin_amdgcn_readfirstlane(threadIdx.x / C::TPR), cols = (int)p.cols;
  const float inv = 1.0f / (float)p.cols;
  // every team of the block makes the same number of turns; a team without a row
  // works on the last one and stores and adds nothing
  const int64_t step = (int64_t)gridDim.x * C::PER_BLOCK;
  int64_t row = (int64_t)blockIdx.x * C::PER_BLOCK + team;
  constexpr bool AHEAD = C::TPR < 1024;
  KeptRow<T, C> next;
  if constexpr (AHEAD) next.load(p, row < p.rows ? row : p.rows - 1, t);
  RowVec<float, C::VEC, false> gamma[C::NV];
  if (p.gamma) {
#pragma unroll
    for (int k = 0; k < C::NV; ++k) gamma[k].load(p.gamma, (k * C::TPR + t) * C::VEC, cols);
  }
  float ga[C::NV][C::VEC];
#pragma unroll
  for (int k = 0; k < C::NV; ++k) {
#pragma unroll
    for (int i = 0; i < C::VEC; ++i) ga[k][i] = 1.0f;
    if (p.gamma) gamma[k].value(cols - (k * C::TPR + t) * C::VEC, cols, ga[k]);
  }
  for (int64_t base = (int64_t)blockIdx.x * C::PER_BLOCK; base < p.rows; base += step, row += step) {
    if constexpr (!AHEAD) next.load(p, row < p.rows ? row : p.rows - 1, t);
    const KeptRow<T, C> r = next;
    if (AHEAD && base + step < p.rows) next.load(p, row + step < p.rows ? row + step : p.rows - 1, t);
    float s[2] = {0.0f, 0.0f};
    float gv[C::NV][C::VEC];
    if (row < p.rows) {
      // What a code past the row may stand for (NaN, if its block's scale is) meets
      // a zero of G in columns that are not stored, and in the sums of a row that
      // is NaN as well.
#pragma unroll
      for (int k = 0; k < C::NV; ++k) {
        float xh[C::VEC];
        r.xhat(k, xh);
        r.g[k].value(cols - (k * C::TPR + t) * C::VEC, cols, gv[k]);
#pragma unroll
        for (int i = 0; i < C::VEC; ++i) {
          sg[k][i] = fmaf(gv[k][i], xh[i], sg[k][i]);
          sb[k][i] += gv[k][i];
          gv[k][i] *= ga[k][i];
          s[0] += gv[k][i];
          s[1] = fmaf(gv[k][i], xh[i], s[1]);
        }
      }
    }
    team_sum<C, 2>(s, sh[team]);
    const float a = s[0] * inv, b = s[1] * inv;
    T* y = static_cast<T*>(p.y) + row * p.ldy;
#pragma unroll
    for (int k = 0; k < C::NV; ++k) {
      const int64_t col = (int64_t)(k * C::TPR + t) * C::VEC;
      float xh[C::VEC], o[C::VEC];
      r.xhat(k, xh);
#pragma unroll
      for (int i = 0; i < C::VEC; ++i) o[i] = r.rstd * ((gv[k][i] - a) - xh[i] * b);
      store_part<T, C::VEC>(y + col, row < p.rows ? cols - col : 0, o);
    }
  }
}

// Backward: one block of 1024 threads a unit, so that there are few partial
// sums (8192 x 1024 bfloat16: 1024 blocks of four teams leave 8 MB of them, 21.1
// us in all instead of 17.8; float32 29.5, 27.3).  Each team takes every (teams)-th row and keeps its columns'
// sums of g xh and g in registers; at the end the block's teams meet in LDS
// pairwise and one writes the block's partial row (an only block writes the
// parameter gradients themselves).  KEPT: from the checkpoint.
template <class T, class C, bool KEPT>
__global__ __launch_bounds__(C::THREADS) void norm_backward_kernel(NormParams p) {
  __shared__ float sh[C::PER_BLOCK][C::WAVES][2];
  __shared__ __attribute__((aligned(16))) float col_sum[C::PER_BLOCK > 1 ? C::PER_BLOCK / 2 : 1][2][C::PER_BLOCK > 1 ? C::COLS : 4];
  const int t = threadIdx.x % C::TPR, team = threadIdx.x / C::TPR;
  const float inv = 1.0f / (float)p.cols;
  float sg[C::NV][C::VEC], sb[C::NV][C::VEC];
#pragma unroll
  for (int k = 0; k < C::NV; ++k)
#pragma unroll
    for (int i = 0; i < C::VEC; ++i) sg[k][i] = sb[k][i] = 0.0f;
  // 16 elements of each of a row's 1024 threads do not fit the registers with what kept_rows
  // holds besides: 2048 x 16000 bfloat16 90 us, row by row 57 (float32 123, 86).  Of 512
  // threads (16-bit types, 4097 - 8192 columns) six registers are spilled, and the row ahead
  // gains all the same, the call in a graph with / row by row: 8192 x 8192 bfloat16 76 / 105, 2048 x 8192 26 / 28,
  // 8192 x 4104 float16 57 / 73; 300 x 6144, blocks of a row or two, 13.9 / 13.7
  constexpr bool AHEAD = KEPT && (C::TPR < 1024 || C::NV * C::VEC <= 8);
  if constexpr (AHEAD) kept_rows<T, C>(p, sh, sg, sb);
  // every team of the block makes the same number of turns (the barriers
  // inside team_sum meet); a team without a row reads and writes nothing
  for (int64_t base = (int64_t)blockIdx.x * C::PER_BLOCK; !AHEAD && base < p.rows; base += (int64_t)gridDim.x * C::PER_BLOCK) {
    const bool any = base + team < p.rows;
    const int64_t row = any ? base + team : 0;
    const int cols = any ? (int)p.cols : 0;
    const T* x = static_cast<const T*>(p.x) + row * p.ldx;
    const T* g = static_cast<const T*>(p.g) + row * p.ldg;
    float xh[C::NV][C::VEC], gv[C::NV][C::VEC];
#pragma unroll
    for (int k = 0; k < C::NV; ++k) {
      const int col = (k * C::TPR + t) * C::VEC;
      if constexpr (KEPT)
        kept_values<C::VEC>(p.q8 + row * kept_pitch(p.cols), p.e8 + row * kept_blocks(p.cols), cols - col, col, xh[k]);
      else
        load_part<T, C::VEC>(x + col, cols - col, xh[k]);
      load_part<T, C::VEC>(g + col, cols - col, gv[k]);
    }
    const float mean = KEPT ? 0.0f : p.mean[row], rstd = p.rstd[row];
    float s[2] = {0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < C::NV; ++k) {
      const int col = (k * C::TPR + t) * C::VEC;
      float ga[C::VEC];
#pragma unroll
      for (int i = 0; i < C::VEC; ++i) ga[i] = 1.0f;
      // read again for every row: from the nearest cache, and the registers
      // hold more waves instead
      if (p.gamma) load_part<float, C::VEC>(p.gamma + col, (int)p.cols - col, ga);
#pragma unroll
      for (int i = 0; i < C::VEC; ++i) {
        // no column (or no row): xh is 0 like g, since (0 - mean) rstd may be infinite
        if constexpr (!KEPT) xh[k][i] = col + i < cols ? (xh[k][i] - mean) * rstd : 0.0f;
        sg[k][i] = fmaf(gv[k][i], xh[k][i], sg[k][i]);
        sb[k][i] += gv[k][i];
        gv[k][i] *= ga[i];
        s[0] += gv[k][i];
        s[1] = fmaf(gv[k][i], xh[k][i], s[1]);
      }
    }
    team_sum<C, 2>(s, sh[team]);
    const float a = s[0] * inv, b = s[1] * inv;
    T* y = static_cast<T*>(p.y) + row * p.ldy;
#pragma unroll
    for (int k = 0; k < C::NV; ++k) {
      const int64_t col = (int64_t)(k * C::TPR + t) * C::VEC;
      float o[C::VEC];
#pragma unroll
      for (int i = 0; i < C::VEC; ++i) o[i] = rstd * ((gv[k][i] - a) - xh[k][i] * b);
      store_part<T, C::VEC>(y + col, cols - col, o);
    }
  }
  if (!p.grad_gamma && !p.grad_beta) return;
#pragma unroll
  for (int w = C::PER_BLOCK / 2; w > 0; w /= 2) {  // teams w .. 2 w - 1 hand over to 0 .. w - 1
    if (team >= w && team < 2 * w) {
#pragma unroll
      for (int k = 0; k < C::NV; ++k) {
        const int col = (k * C::TPR + t) * C::VEC;
        store_vec<float, C::VEC>(&col_sum[team - w][0][col], sg[k]);
        store_vec<float, C::VEC>(&col_sum[team - w][1][col], sb[k]);
      }
    }
    __syncthreads();
    if (team < w) {
#pragma unroll
      for (int k = 0; k < C::NV; ++k) {
        const int col = (k * C::TPR + t) * C::VEC;
        float a[C::VEC], b[C::VEC];
        load_vec<float, C::VEC>(&col_sum[team][0][col], a);
        load_vec<float, C::VEC>(&col_sum[team][1][col], b);
#pragma unroll
        for (int i = 0; i < C::VEC; ++i) {
          sg[k][i] += a[i];
          sb[k][i] += b[i];
        }
      }
    }
    __syncthreads();
  }
  if (team != 0) return;
  float* part = p.part + (int64_t)blockIdx.x * 2 * p.cols;
  float* const to_gamma = gridDim.x == 1 ? p.grad_gamma : part;
  float* const to_beta = gridDim.x == 1 ? p.grad_beta : part + p.cols;
#pragma unroll
  for (int k = 0; k < C::NV; ++k) {
    const int64_t col = (int64_t)(k * C::TPR + t) * C::VEC;
    if (to_gamma) store_part<float, C::VEC>(to_gamma + col, p.cols - col, sg[k]);
    if (to_beta) store_part<float, C::VEC>(to_beta + col, p.cols - col, sb[k]);
  }
}

// Rows longer than a team's registers: inputs read twice, no parameter sums.
template <class T, class C, bool KEPT>
__global__ __launch_bounds__(C::THREADS) void norm_backward_long_kernel(NormParams p) {
  __shared__ float sh[C::WAVES][2];
  const int64_t row = block_id();
  if (row >= p.rows) return;
  const T* x = static_cast<const T*>(p.x) + row * p.ldx;
  const T* g = static_cast<const T*>(p.g) + row * p.ldg;
  T* y = static_cast<T*>(p.y) + row * p.ldy;
  const float mean = KEPT ? 0.0f : p.mean[row], rstd = p.rstd[row], inv = 1.0f / (float)p.cols;
  const uint8_t* const q8 = p.q8 + row * kept_pitch(p.cols);
  const uint8_t* const e8 = p.e8 + row * kept_blocks(p.cols);
  auto load_xh = [&](int64_t col, float (&v)[C::VEC]) __attribute__((always_inline)) {
    if constexpr (KEPT) {
      kept_values<C::VEC>(q8, e8, p.cols - col, col, v);
    } else {
      load_part<T, C::VEC>(x + col, p.cols - col, v);
#pragma unroll
      for (int i = 0; i < C::VEC; ++i) v[i] = col + i < p.cols ? (v[i] - mean) * rstd : 0.0f;  // (0 - mean) rstd may be infinite
    }
  };
  const int64_t step = (int64_t)C::TPR * C::VEC, first = (int64_t)threadIdx.x * C::VEC;
  float xv[C::VEC], gv[C::VEC];
  float s[2] = {0.0f, 0.0f};
  for (int64_t col = first; col < p.cols; col += step) {
    load_xh(col, xv);
    load_part<T, C::VEC>(g + col, p.cols - col, gv);
#pragma unroll
    for (int i = 0; i < C::VEC; ++i) {
      const float c = gv[i] * (p.gamma && col + i < p.cols ? p.gamma[col + i] : 1.0f);
      s[0] += c;
      s[1] = fmaf(c, xv[i], s[1]);
    }
  }
  team_sum<C, 2>(s, sh);
  const float a = s[0] * inv, b = s[1] * inv;
  for (int64_t col = first; col < p.cols; col += step) {
    load_xh(col, xv);
    load_part<T, C::VEC>(g + col, p.cols - col, gv);
#pragma unroll
    for (int i = 0; i < C::VEC; ++i) {
      const float c = gv[i] * (p.gamma && col + i < p.cols ? p.gamma[col + i] : 1.0f);
      gv[i] = rstd * ((c - a) - xv[i] * b);
    }
    store_part<T, C::VEC>(y + col, p.cols - col, gv);
  }
}

// The parameter sums of long rows: a block takes 256 columns of a run of rows.
constexpr int LONG_RUNS = 64;
template <class T, bool KEPT>
__global__ __launch_bounds__(256) void norm_columns_kernel(NormParams p) {
  const int64_t col = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (col >= p.cols) return;
  float sg = 0.0f, sb = 0.0f;
  for (int64_t row = blockIdx.y; row < p.rows; row += gridDim.y) {
    const float g = (float)static_cast<const T*>(p.g)[row * p.ldg + col];
    float xh;
    if constexpr (KEPT) {
      const int64_t pitch = kept_pitch(p.cols);
      xh = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(p.q8[row * pitch + col], scale_up(p.e8[(row * pitch + col) / KEPT_BLOCK]), false)[0];
    } else {
      xh = ((float)static_cast<const T*>(p.x)[row * p.ldx + col] - p.mean[row]) * p.rstd[row];
    }
    sg = fmaf(g, xh, sg);
    sb += g;
  }
  p.part[(int64_t)blockIdx.y * 2 * p.cols + col] = sg;
  p.part[((int64_t)blockIdx.y * 2 + 1) * p.cols + col] = sb;
}

// The partial rows added up: 64 columns a block, one wave a run of partials,
// the waves' sums in order.
constexpr int REDUCE_WAVES = 16;
__global__ __launch_bounds__(64 * REDUCE_WAVES) void norm_reduce_kernel(const float* part, int64_t parts, int64_t cols,
                                                                         float* grad_gamma, float* grad_beta) {
  __shared__ float sh[REDUCE_WAVES][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t col = block_id() * 64 + lane;  // of 2 * cols: gamma's, then beta's
  float s = 0.0f;
  if (col < 2 * cols) {
#pragma unroll 4
    for (int64_t i = wave; i < parts; i += REDUCE_WAVES) s += part[i * 2 * cols + col];
  }
  sh[wave][lane] = s;
  __syncthreads();
  if (wave == 0 && col < 2 * cols) {
    for (int w = 1; w < REDUCE_WAVES; ++w) s += sh[w][lane];
    if (col < cols) {
      if (grad_gamma) grad_gamma[col] = s;
    } else if (grad_beta) {
      grad_beta[col - cols] = s;
    }
  }
}

// ---------------------------------------------------------------------------
// launches
// ---------------------------------------------------------------------------
// Teams by row length; 16 elements a thread.  A wave up to 1024 columns needs no
// barrier (8192 x 1024: bfloat16 9.6 us, with four waves a row 13.1; float32
// 13.0, 15.9; backward 17.8, 22.1 and 27.3, 29.5); at 2048 columns 32 elements
// a thread gain nothing (15.5 us with four waves, 16.1 with one; float32 27.6,
// 29.9; backward 30.7, 30.5 and 44.5, 44.2).  A call of one row of 1024 is the other
// way round, 2.9 us against 2.6 and 6.2 against 4.1 in the backward, whose block
// adds up idle teams too.
template <class T, class F>
static hipError_t with_team(int64_t cols, F f) {
  constexpr int V = 16 / (int)sizeof(T);  // elements of 16 bytes
  constexpr int H = V / 2;
  if (cols <= 64 * 4) return f(Team<64, H, 4 / H>{});
  if (cols <= 64 * 8) return f(Team<64, V, 8 / V>{});
  if (cols <= 64 * 16) return f(Team<64, V, 16 / V>{});
  if (cols <= 256 * 8) return f(Team<256, V, 8 / V>{});
  if (cols <= 256 * 16) return f(Team<256, V, 16 / V>{});
  if (cols <= 512 * 16) return f(Team<512, V, 16 / V>{});
  return f(Team<1024, V, 16 / V>{});
}
constexpr int64_t TEAM_COLS = 1024 * 16;

template <class T, bool KEEP>
static hipError_t norm_forward(const NormParams& p, hipStream_t s) {
  return with_team<T>(p.cols, [&](auto c) {
    using C = decltype(c);
    const int64_t blocks = (p.rows + C::PER_BLOCK - 1) / C::PER_BLOCK;
    const dim3 grid = grid_of(blocks, C::THREADS);
    auto kernel = [] {
      if constexpr (KEEP)
        return norm_forward8_kernel<T, C>;
      else
        return norm_forward_kernel<T, C>;
    }();
    if (p.cols <= TEAM_COLS)
      hipLaunchKernelGGL(kernel, grid, dim3(C::THREADS), 0, s, p);
    else if constexpr (C::TPR == 1024)
      hipLaunchKernelGGL((norm_forward_long_kernel<T, C, KEEP>), grid, dim3(C::THREADS), 0, s, p);
    return hipGetLastError();
  });
}
hipError_t launch_norm_forward(fqt_dtype type, const NormParams& p, hipStream_t s) {
  return with_type(type, [&](auto e) {
    using T = decltype(e);
    return p.q8 ? norm_forward<T, true>(p, s) : norm_forward<T, false>(p, s);
  });
}

// Backward: blocks of 1024 threads.
template <class T, class F>
static hipError_t with_block(int64_t cols, F f) {
  constexpr int V = 16 / (int)sizeof(T);
  constexpr int H = V / 2;
  if (cols <= 64 * 4) return f(Team<64, H, 4 / H, 1024>{});
  if (cols <= 64 * 8) return f(Team<64, V, 8 / V, 1024>{});
  if (cols <= 64 * 16) return f(Team<64, V, 16 / V, 1024>{});
  if (cols <= 256 * 8) return f(Team<256, V, 8 / V, 1024>{});
  if (cols <= 256 * 16) return f(Team<256, V, 16 / V, 1024>{});
  if (cols <= 512 * 16) return f(Team<512, V, 16 / V, 1024>{});
  return f(Team<1024, V, 16 / V>{});
}
constexpr int64_t BACKWARD_BLOCKS = 256;
static int64_t backward_blocks(int64_t rows, int64_t cols) {
  if (cols > TEAM_COLS) return rows < LONG_RUNS ? rows : LONG_RUNS;
  const int64_t per = cols <= 64 * 16 ? 16 : cols <= 256 * 16 ? 4 : cols <= 512 * 16 ? 2 : 1;
  const int64_t blocks = (rows + per - 1) / per;
  return blocks < BACKWARD_BLOCKS ? blocks : BACKWARD_BLOCKS;
}
int64_t norm_backward_partials(int64_t rows, int64_t cols) { return backward_blocks(rows, cols) * 2 * cols; }

// From a checkpoint: 8 float32 elements a thread, so that the next row's fit the
// registers (8192 x 4096, 302 MB, with 16 of them and no row ahead 80 us, so 58).
// The workspace is the plain form's, and so are the blocks: smaller teams make more
// turns (2048 x 1024: two, on 128 units).
template <class T, class F>
static hipError_t with_kept_block(int64_t cols, F f) {
  if constexpr (sizeof(T) == 4) {
    if (cols <= 64 * 4) return f(Team<64, 2, 2, 1024>{});
    if (cols <= 64 * 8) return f(Team<64, 4, 2, 1024>{});
    if (cols <= 128 * 8) return f(Team<128, 4, 2, 1024>{});
    if (cols <= 256 * 8) return f(Team<256, 4, 2, 1024>{});
    if (cols <= 512 * 8) return f(Team<512, 4, 2, 1024>{});
    if (cols <= 1024 * 8) return f(Team<1024, 4, 2>{});
    return f(Team<1024, 4, 4>{});
  } else {
    return with_block<T>(cols, f);
  }
}
static bool in_team(const NormParams& p) { return p.cols <= TEAM_COLS && !(p.q8 && p.cols < 8); }
template <class T, bool KEPT>
static hipError_t norm_backward_long(const NormParams& p, bool sums, int64_t blocks, hipStream_t s) {
  using C = Team<1024, 16 / (int)sizeof(T), (int)sizeof(T)>;
  hipLaunchKernelGGL((norm_backward_long_kernel<T, C, KEPT>), grid_of(p.rows, C::THREADS), dim3(C::THREADS), 0, s, p);
  if (sums)
    hipLaunchKernelGGL((norm_columns_kernel<T, KEPT>), dim3((unsigned)((p.cols + 255) / 256), (unsigned)blocks), dim3(256),
                       0, s, p);
  return hipGetLastError();
}
template <class T>
static hipError_t norm_backward(const NormParams& p, bool sums, int64_t blocks, hipStream_t s) {
  if (!in_team(p)) return p.q8 ? norm_backward_long<T, true>(p, sums, blocks, s) : norm_backward_long<T, false>(p, sums, blocks, s);
  const dim3 grid((unsigned)blocks);
  if (p.q8)
    return with_kept_block<T>(p.cols, [&](auto c) {
      using C = decltype(c);
      hipLaunchKernelGGL((norm_backward_kernel<T, C, true>), grid, dim3(C::THREADS), 0, s, p);
      return hipGetLastError();
    });
  return with_block<T>(p.cols, [&](auto c) {
    using C = decltype(c);
    hipLaunchKernelGGL((norm_backward_kernel<T, C, false>), grid, dim3(C::THREADS), 0, s, p);
    return hipGetLastError();
  });
}
hipError_t launch_norm_backward(fqt_dtype type, const NormParams& p, hipStream_t s) {
  const bool sums = p.grad_gamma || p.grad_beta;
  const int64_t blocks = backward_blocks(p.rows, p.cols);
  const hipError_t e = with_type(type, [&](auto el) {
    using T = decltype(el);
    return norm_backward<T>(p, sums, blocks, s);
  });
  if (e != hipSuccess || !sums || (blocks == 1 && in_team(p))) return e;
  hipLaunchKernelGGL(norm_reduce_kernel, grid_of((2 * p.cols + 63) / 64, 64 * REDUCE_WAVES), dim3(64 * REDUCE_WAVES),
                     0, s, p.part, blocks, p.cols, p.grad_gamma, p.grad_beta);
  return hipGetLastError();
}

}  // namespace fqt
