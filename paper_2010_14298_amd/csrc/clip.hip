// Global gradient norm over many tensors, and clipping:
//   n = sqrt(sum over tensors and elements of g^2)
//   out = g * (max_norm / n) where n > max_norm and n is finite, else g
//
// Squares and sums are float64 (a float32 squared is exact there and cannot
// overflow), in an order that the sizes alone decide.  Two launches for up
// to CLIP_TENSORS tensors: partial sums, then every block of the scaling
// launch adds the partials up for itself and scales its chunks.
#include "train_kernels.h"

namespace fqt {

constexpr int CLIP_THREADS = 256;
constexpr int64_t CLIP_CHUNK = 16384;  // elements of one block's turn
int64_t clip_chunks(int64_t n) { return (n + CLIP_CHUNK - 1) / CLIP_CHUNK; }

__device__ __forceinline__ double block_sum(double v, double* sh) {
#pragma unroll
  for (int m = 32; m; m >>= 1) v += __shfl_xor(v, m);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
  __syncthreads();
  v = 0.0;
  for (int w = 0; w < CLIP_THREADS / 64; ++w) v += sh[w];
  return v;
}

// The tensor that holds a chunk: the last one whose first chunk is not past it.
__device__ __forceinline__ int tensor_of(const ClipTable& t, uint32_t chunk) {
  int lo = 0, hi = t.count;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (t.first[mid] <= chunk)
      lo = mid;
    else
      hi = mid;
  }
  return lo;
}

template <class T>
__device__ __forceinline__ double chunk_squares(const T* g, int64_t n) {
  constexpr int V = 16 / (int)sizeof(T);
  double s = 0.0;
  for (int64_t i = (int64_t)threadIdx.x * V; i < n; i += CLIP_THREADS * V) {
    float v[V];
    load_part<T, V>(g + i, n - i, v);
#pragma unroll
    for (int j = 0; j < V; ++j) s = fma((double)v[j], (double)v[j], s);
  }
  return s;
}

template <class T>
__device__ __forceinline__ void chunk_scale(const T* g, T* out, int64_t n, float c) {
  constexpr int V = 16 / (int)sizeof(T);
  for (int64_t i = (int64_t)threadIdx.x * V; i < n; i += CLIP_THREADS * V) {
    float v[V];
    load_part<T, V>(g + i, n - i, v);
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] *= c;
    store_part<T, V>(out + i, n - i, v);
  }
}

__global__ __launch_bounds__(CLIP_THREADS) void clip_norm_kernel(ClipTable t, double* part) {
  __shared__ double sh[CLIP_THREADS / 64];
  double s = 0.0;
  for (uint32_t c = blockIdx.x; c < t.first[t.count]; c += gridDim.x) {
    const int k = tensor_of(t, c);
    const int64_t at = (int64_t)(c - t.first[k]) * CLIP_CHUNK;
    const int64_t n = t.n[k] - at < CLIP_CHUNK ? t.n[k] - at : CLIP_CHUNK;
    if (t.type[k] == FQT_F32)
      s += chunk_squares(static_cast<const float*>(t.g[k]) + at, n);
    else if (t.type[k] == FQT_BF16)
      s += chunk_squares(static_cast<const __bf16*>(t.g[k]) + at, n);
    else
      s += chunk_squares(static_cast<const _Float16*>(t.g[k]) + at, n);
  }
  s = block_sum(s, sh);
  if (threadIdx.x == 0) part[blockIdx.x] = s;
}

__global__ __launch_bounds__(CLIP_THREADS) void clip_scale_kernel(ClipTable t, const double* part, int64_t parts,
                                                                   double max_norm, float* norm) {
  __shared__ double sh[CLIP_THREADS / 64];
  double s = 0.0;
  for (int64_t i = threadIdx.x; i < parts; i += CLIP_THREADS) s += part[i];
  const double n = sqrt(block_sum(s, sh));
  if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)n;
  // a norm that is not finite scales nothing: the caller sees it and drops the step
  const bool clip = n > max_norm && n < __builtin_huge_val();
  const float scale = clip ? (float)(max_norm / n) : 1.0f;
  for (uint32_t c = blockIdx.x; c < t.first[t.count]; c += gridDim.x) {
    const int k = tensor_of(t, c);
    if (!clip && t.out[k] == t.g[k]) continue;
    const int64_t at = (int64_t)(c - t.first[k]) * CLIP_CHUNK;
    const int64_t len = t.n[k] - at < CLIP_CHUNK ? t.n[k] - at : CLIP_CHUNK;
    if (t.type[k] == FQT_F32)
      chunk_scale(static_cast<const float*>(t.g[k]) + at, static_cast<float*>(t.out[k]) + at, len, scale);
    else if (t.type[k] == FQT_BF16)
      chunk_scale(static_cast<const __bf16*>(t.g[k]) + at, static_cast<__bf16*>(t.out[k]) + at, len, scale);
    else
      chunk_scale(static_cast<const _Float16*>(t.g[k]) + at, static_cast<_Float16*>(t.out[k]) + at, len, scale);
  }
}

hipError_t launch_clip_norm(const ClipTable& t, double* part, hipStream_t s) {
  hipLaunchKernelGGL(clip_norm_kernel, dim3(CLIP_PARTS), dim3(CLIP_THREADS), 0, s, t, part);
  return hipGetLastError();
}
hipError_t launch_clip_scale(const ClipTable& t, const double* part, int64_t parts, double max_norm, float* norm,
                             hipStream_t s) {
  const uint32_t chunks = t.first[t.count];
  const unsigned blocks = chunks < 2048 ? (chunks ? chunks : 1) : 2048;
  hipLaunchKernelGGL(clip_scale_kernel, dim3(blocks), dim3(CLIP_THREADS), 0, s, t, part, parts, max_norm, norm);
  return hipGetLastError();
}

}  // namespace fqt
