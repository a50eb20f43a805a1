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
#include "train_kernels.h"

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

// Rows longer than a team's registers: the row is read three times (sum,
// squares, output), the later ones from the caches.
template <class T, class C>
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
  for (int64_t col = first; col < p.cols; col += step) {
    load_part<T, C::VEC>(x + col, p.cols - col, v);
#pragma unroll
    for (int i = 0; i < C::VEC; ++i)
      if (col + i < p.cols)
        v[i] = fmaf((v[i] - mean) * rstd, p.gamma ? p.gamma[col + i] : 1.0f, p.beta ? p.beta[col + i] : 0.0f);
    store_part<T, C::VEC>(y + col, p.cols - col, v);
  }
}

// Backward: one block of 1024 threads a unit, so that there are few partial
// sums (8192 x 1024 bfloat16: 1024 blocks of four teams leave 8 MB of them, 21.1
// us in all instead of 17.8; float32 29.5, 27.3).  Each team takes every (teams)-th row and keeps its columns'
// sums of g xh and g in registers; at the end the block's teams meet in LDS
// pairwise and one writes the block's partial row (an only block writes the
// parameter gradients themselves).
template <class T, class C>
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
  // every team of the block makes the same number of turns (the barriers
  // inside team_sum meet); a team without a row reads and writes nothing
  for (int64_t base = (int64_t)blockIdx.x * C::PER_BLOCK; base < p.rows; base += (int64_t)gridDim.x * C::PER_BLOCK) {
    const bool any = base + team < p.rows;
    const int64_t row = any ? base + team : 0;
    const int cols = any ? (int)p.cols : 0;
    const T* x = static_cast<const T*>(p.x) + row * p.ldx;
    const T* g = static_cast<const T*>(p.g) + row * p.ldg;
    float xh[C::NV][C::VEC], gv[C::NV][C::VEC];
#pragma unroll
    for (int k = 0; k < C::NV; ++k) {
      const int col = (k * C::TPR + t) * C::VEC;
      load_part<T, C::VEC>(x + col, cols - col, xh[k]);
      load_part<T, C::VEC>(g + col, cols - col, gv[k]);
    }
    const float mean = p.mean[row], rstd = p.rstd[row];
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
        xh[k][i] = col + i < cols ? (xh[k][i] - mean) * rstd : 0.0f;
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
template <class T, class C>
__global__ __launch_bounds__(C::THREADS) void norm_backward_long_kernel(NormParams p) {
  __shared__ float sh[C::WAVES][2];
  const int64_t row = block_id();
  if (row >= p.rows) return;
  const T* x = static_cast<const T*>(p.x) + row * p.ldx;
  const T* g = static_cast<const T*>(p.g) + row * p.ldg;
  T* y = static_cast<T*>(p.y) + row * p.ldy;
  const float mean = p.mean[row], rstd = p.rstd[row], inv = 1.0f / (float)p.cols;
  const int64_t step = (int64_t)C::TPR * C::VEC, first = (int64_t)threadIdx.x * C::VEC;
  float xv[C::VEC], gv[C::VEC];
  float s[2] = {0.0f, 0.0f};
  for (int64_t col = first; col < p.cols; col += step) {
    load_part<T, C::VEC>(x + col, p.cols - col, xv);
    load_part<T, C::VEC>(g + col, p.cols - col, gv);
#pragma unroll
    for (int i = 0; i < C::VEC; ++i) {
      const bool in = col + i < p.cols;
      const float c = gv[i] * (p.gamma && in ? p.gamma[col + i] : 1.0f);
      s[0] += c;
      s[1] = fmaf(c, in ? (xv[i] - mean) * rstd : 0.0f, s[1]);  // (0 - mean) rstd may be infinite
    }
  }
  team_sum<C, 2>(s, sh);
  const float a = s[0] * inv, b = s[1] * inv;
  for (int64_t col = first; col < p.cols; col += step) {
    load_part<T, C::VEC>(x + col, p.cols - col, xv);
    load_part<T, C::VEC>(g + col, p.cols - col, gv);
#pragma unroll
    for (int i = 0; i < C::VEC; ++i) {
      const float c = gv[i] * (p.gamma && col + i < p.cols ? p.gamma[col + i] : 1.0f);
      gv[i] = rstd * ((c - a) - (xv[i] - mean) * rstd * b);
    }
    store_part<T, C::VEC>(y + col, p.cols - col, gv);
  }
}

// The parameter sums of long rows: a block takes 256 columns of a run of rows.
constexpr int LONG_RUNS = 64;
template <class T>
__global__ __launch_bounds__(256) void norm_columns_kernel(NormParams p) {
  const int64_t col = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (col >= p.cols) return;
  float sg = 0.0f, sb = 0.0f;
  for (int64_t row = blockIdx.y; row < p.rows; row += gridDim.y) {
    const float g = (float)static_cast<const T*>(p.g)[row * p.ldg + col];
    const float x = (float)static_cast<const T*>(p.x)[row * p.ldx + col];
    sg = fmaf(g, (x - p.mean[row]) * p.rstd[row], sg);
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

hipError_t launch_norm_forward(fqt_dtype type, const NormParams& p, hipStream_t s) {
  return with_type(type, [&](auto e) {
    using T = decltype(e);
    return with_team<T>(p.cols, [&](auto c) {
      using C = decltype(c);
      const int64_t blocks = (p.rows + C::PER_BLOCK - 1) / C::PER_BLOCK;
      const dim3 grid = grid_of(blocks, C::THREADS);
      if (p.cols <= TEAM_COLS)
        hipLaunchKernelGGL((norm_forward_kernel<T, C>), grid, dim3(C::THREADS), 0, s, p);
      else if constexpr (C::TPR == 1024)
        hipLaunchKernelGGL((norm_forward_long_kernel<T, C>), grid, dim3(C::THREADS), 0, s, p);
      return hipGetLastError();
    });
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

hipError_t launch_norm_backward(fqt_dtype type, const NormParams& p, hipStream_t s) {
  const bool sums = p.grad_gamma || p.grad_beta;
  const int64_t blocks = backward_blocks(p.rows, p.cols);
  const hipError_t e = with_type(type, [&](auto el) {
    using T = decltype(el);
    return with_block<T>(p.cols, [&](auto c) {
      using C = decltype(c);
      if (p.cols <= TEAM_COLS) {
        hipLaunchKernelGGL((norm_backward_kernel<T, C>), dim3((unsigned)blocks), dim3(C::THREADS), 0, s, p);
      } else if constexpr (C::TPR == 1024) {
        hipLaunchKernelGGL((norm_backward_long_kernel<T, C>), grid_of(p.rows, C::THREADS), dim3(C::THREADS), 0, s, p);
        if (sums)
          hipLaunchKernelGGL((norm_columns_kernel<T>), dim3((unsigned)((p.cols + 255) / 256), (unsigned)blocks),
                             dim3(256), 0, s, p);
      }
      return hipGetLastError();
    });
  });
  if (e != hipSuccess || !sums || (blocks == 1 && p.cols <= TEAM_COLS)) return e;
  hipLaunchKernelGGL(norm_reduce_kernel, grid_of((2 * p.cols + 63) / 64, 64 * REDUCE_WAVES), dim3(64 * REDUCE_WAVES),
                     0, s, p.part, blocks, p.cols, p.grad_gamma, p.grad_beta);
  return hipGetLastError();
}

}  // namespace fqt
