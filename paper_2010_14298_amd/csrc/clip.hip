// Global gradient norm over many tensors, and clipping:
//   n = sqrt(sum over tensors and elements of g^2)
//   out = g * (max_norm / n) where n > max_norm and n, as it is returned (float32), is finite, else g
//
// Squares and sums are float64 (a float32 squared is exact there and cannot
// overflow), in an order that the sizes alone decide.  Two launches for up
// to CLIP_TENSORS tensors: partial sums, then every block of the scaling
// launch adds the partials up for itself and scales its chunks.  A chunk is
// four 16-byte loads a thread; turns this small spread tensors of any size
// evenly over the blocks.
//
// Memory bounds it: 25.2 M float32 gradients take 25.5 us for the norm (101 MB,
// 4.0 TB/s) and 34.3 us for the scaling (201 MB, 5.9 TB/s: part of the second
// read comes from the last cache).  161 bfloat16 tensors, 51 MB: 13.4 + 19.7 us.
#include "train_kernels.h"

namespace fqt {

constexpr int CLIP_THREADS = 256;
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

// A thread's part of a chunk, as it lies in memory; zeros past the tensor.
struct Raw {
  typedef uint32_t u32x4u __attribute__((ext_vector_type(4), aligned(2)));
  static constexpr int N = (int)CLIP_BYTES / (16 * CLIP_THREADS);
  u32x4u v[N];
  __device__ __forceinline__ void load(const char* p, int bytes) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int at = 16 * (i * CLIP_THREADS + (int)threadIdx.x);
      if (at + 16 <= bytes) {
        v[i] = *reinterpret_cast<const u32x4u*>(p + at);
      } else {
        v[i] = u32x4u{0u, 0u, 0u, 0u};
#pragma unroll
        for (int h = 0; h < 8; ++h)  // elements have two or four bytes
          if (at + 2 * h < bytes)
            v[i][h / 2] |= (uint32_t)*reinterpret_cast<const uint16_t*>(p + at + 2 * h) << (16 * (h & 1));
      }
    }
  }
  __device__ __forceinline__ void store(char* p, int bytes) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int at = 16 * (i * CLIP_THREADS + (int)threadIdx.x);
      if (at + 16 <= bytes) {
        *reinterpret_cast<u32x4u*>(p + at) = v[i];
      } else {
#pragma unroll
        for (int h = 0; h < 8; ++h)
          if (at + 2 * h < bytes) *reinterpret_cast<uint16_t*>(p + at + 2 * h) = (uint16_t)(v[i][h / 2] >> (16 * (h & 1)));
      }
    }
  }
  template <class T>
  __device__ __forceinline__ double squares(double s) const {
    constexpr int V = 16 / (int)sizeof(T);
    typedef T vec __attribute__((ext_vector_type(V)));
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const vec x = __builtin_bit_cast(vec, v[i]);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const double d = (double)(float)x[j];
        s = fma(d, d, s);
      }
    }
    return s;
  }
  template <class T>
  __device__ __forceinline__ void scale(float f) {
    constexpr int V = 16 / (int)sizeof(T);
    typedef T vec __attribute__((ext_vector_type(V)));
#pragma unroll
    for (int i = 0; i < N; ++i) {
      vec x = __builtin_bit_cast(vec, v[i]);
#pragma unroll
      for (int j = 0; j < V; ++j) x[j] = (T)((float)x[j] * f);
      v[i] = __builtin_bit_cast(u32x4u, x);
    }
  }
};

// The table in LDS, in one round of loads.
__device__ __forceinline__ void table_to_lds(ClipTable& t) {
  static_assert(sizeof(ClipTable) % 4 == 0, "whole words");
  const __attribute__((address_space(4))) uint32_t* args =
      (const __attribute__((address_space(4))) uint32_t*)__builtin_amdgcn_kernarg_segment_ptr();  // the first argument
  uint32_t* to = reinterpret_cast<uint32_t*>(&t);
#pragma unroll
  for (int i = 0; i < (int)(sizeof(ClipTable) / 4 + CLIP_THREADS - 1) / CLIP_THREADS; ++i) {
    const int w = i * CLIP_THREADS + (int)threadIdx.x;
    if (w < (int)sizeof(ClipTable) / 4) to[w] = args[w];
  }
  __syncthreads();
}

// Where a chunk lies.
struct Place {
  const char* g;
  char* out;
  int bytes;
  int type;
};
// Its tensor: as many first chunks as are not past it, counted over the lanes
// (one after the other costs an LDS latency each, 161 tensors 7 us).
__device__ __forceinline__ Place place_of(const ClipTable& t, uint32_t chunk) {
  const int lane = threadIdx.x & 63;
  int k = -1;
  for (int i = 0; i < t.count; i += 64)
    k += __popcll(__builtin_amdgcn_ballot_w64(i + lane < t.count && t.first[i + lane] <= chunk));
  k = __builtin_amdgcn_readfirstlane(k);
  const int64_t at = (int64_t)(chunk - t.first[k]) * CLIP_BYTES;
  return Place{static_cast<const char*>(t.g[k]) + at, static_cast<char*>(t.out[k]) + at,
               chunk + 1 == t.first[k + 1] ? (int)t.tail[k] : (int)CLIP_BYTES, t.type[k]};
}

// A chunk scaled by a factor that float32 would round to fewer bits, or to 0.
template <class T>
__device__ __forceinline__ void scale_exactly(const Place& at, double f) {
#pragma unroll 1
  for (int i = threadIdx.x; i < at.bytes / (int)sizeof(T); i += CLIP_THREADS)
    reinterpret_cast<T*>(at.out)[i] = (T)(float)((double)(float)reinterpret_cast<const T*>(at.g)[i] * f);
}

__global__ __launch_bounds__(CLIP_THREADS) void clip_norm_kernel(ClipTable, double* part) {
  __shared__ double sh[CLIP_THREADS / 64];
  __shared__ ClipTable t;
  table_to_lds(t);
  const uint32_t chunks = t.first[t.count];
  double s = 0.0;
  int type = 0;
  Raw now, next;  // the next turn's loads are on their way while this one's are worked on
  auto fetch = [&](uint32_t c) __attribute__((always_inline)) {
    if (c >= chunks) return;
    const Place at = place_of(t, c);
    type = at.type;
    next.load(at.g, at.bytes);
  };
  fetch(blockIdx.x);
  for (uint32_t c = blockIdx.x; c < chunks; c += gridDim.x) {
    now = next;
    const int what = type;
    fetch(c + gridDim.x);
    if (what == FQT_F32)
      s = now.squares<float>(s);
    else if (what == FQT_BF16)
      s = now.squares<__bf16>(s);
    else
      s = now.squares<_Float16>(s);
  }
  s = block_sum(s, sh);
  if (threadIdx.x == 0) part[blockIdx.x] = s;
}

// From the last chunk to the first: what the norm read last is still in the
// caches.  Six waves a SIMD: left to itself the compiler takes 84 registers, five
// waves (25.2 M float32, both launches, 61.3 us against 60.2).
__global__ __launch_bounds__(CLIP_THREADS, 6) void clip_scale_kernel(ClipTable, const double* part, int64_t parts,
                                                                   double max_norm, float* norm) {
  __shared__ double sh[CLIP_THREADS / 64];
  __shared__ ClipTable t;
  table_to_lds(t);
  double s = 0.0;
  for (int64_t i = threadIdx.x; i < parts; i += CLIP_THREADS) s += part[i];
  const double n = sqrt(block_sum(s, sh));
  const float seen = (float)n;
  if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = seen;
  // a norm that is not finite for the caller, who sees it in float32, scales
  // nothing: the step can be dropped
  const bool clip = n > max_norm && seen < __builtin_huge_valf();
  const double exact = clip ? max_norm / n : 1.0;
  const float scale = (float)exact;
  const uint32_t chunks = t.first[t.count];
  if (exact < 0x1p-126) {
    for (uint32_t c = blockIdx.x; c < chunks; c += gridDim.x) {
      const Place at = place_of(t, c);
      if (at.type == FQT_F32)
        scale_exactly<float>(at, exact);
      else if (at.type == FQT_BF16)
        scale_exactly<__bf16>(at, exact);
      else
        scale_exactly<_Float16>(at, exact);
    }
    return;
  }
  for (uint32_t i = blockIdx.x; i < chunks; i += gridDim.x) {
    const uint32_t c = chunks - 1 - i;
    const Place at = place_of(t, c);
    if (!clip && at.out == at.g) continue;
    Raw v;
    v.load(at.g, at.bytes);
    if (at.type == FQT_F32)
      v.scale<float>(scale);
    else if (at.type == FQT_BF16)
      v.scale<__bf16>(scale);
    else
      v.scale<_Float16>(scale);
    v.store(at.out, at.bytes);
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
