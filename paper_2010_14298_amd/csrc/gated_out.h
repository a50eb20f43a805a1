// What the gated layer's products do with their sums: H and, for the backward,
// the checkpoints of its two derivatives, from accumulators to memory.
#pragma once

#include "fp8_codes.h"
#include "gated_act.h"

namespace fqt {

typedef float v16f __attribute__((ext_vector_type(16)));

// The larger magnitude, NaN if either is.
__device__ __forceinline__ float top_of(float a, float b) {
  return __builtin_elementwise_maximum(__builtin_fabsf(a), __builtin_fabsf(b));
}

// A lane's 16 of a token's 32 hidden units, register r at 8 (r / 4) + 4 half + r % 4
// (half: lane / 32; the lane 32 further holds the others).  Sixteen bytes a
// lane and store: words of two lanes are exchanged so that each has neighbours.
__device__ __forceinline__ void swap_halves(uint32_t& a, uint32_t& b) {
  const auto s = __builtin_amdgcn_permlane32_swap(a, b, false, false);
  a = s[0];  // lower lanes: their a; upper lanes: the lower ones' b
  b = s[1];  // lower lanes: the upper ones' a; upper lanes: their b
}

// The checkpoint's codes and scale byte of a token's block.
__device__ __forceinline__ void keep_block(const Kept& k, const float (&v)[16], int64_t row, int64_t pitch, int64_t col0,
                                           bool store) {
  float top = top_of(v[0], v[1]);
#pragma unroll
  for (int r = 2; r < 16; ++r) top = top_of(top, v[r]);
  const uint32_t bits = __float_as_uint(top);
  const auto s = __builtin_amdgcn_permlane32_swap(bits, bits, false, false);
  const uint32_t key = Quad<float>::key(s[0] > s[1] ? s[0] : s[1]);  // bits sort like magnitudes, NaN above all
  const uint32_t byte = scale_bytes(key) & 0xffffu;
  const float scale = scale_up(byte);
  uint32_t w[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const Quad<float> x{{v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]}};
    w[q] = key >= NAN_KEY ? 0x7f7f7f7fu : x.row_codes(scale);
  }
  swap_halves(w[0], w[2]);
  swap_halves(w[1], w[3]);
  const int half = (threadIdx.x >> 5) & 1;
  const int64_t at = row * pitch + col0;
  if (!store) return;
  *reinterpret_cast<uint4*>(k.q + at + 16 * half) = make_uint4(w[0], w[2], w[1], w[3]);
  // both lanes of a token store the same byte
  k.e[at / KEPT_BLOCK] = stored_byte(key, byte);
}

// Tokens row0 .. row0 + 32 STRIPS - 1 (the lane's at lane % 32), hidden units
// col0 .. col0 + 31; T: the type of H.
template <class T, int STRIPS, class P>
__device__ __forceinline__ void gated_store(const P& p, const v16f (&acc)[STRIPS][2], int64_t row0, int64_t rows,
                                            int64_t col0, T) {
  if (col0 >= p.hidden) return;
  const int lane = threadIdx.x & 63, half = lane >> 5;
  const bool whole = col0 + 32 <= p.hidden;
  const int64_t pitch = kept_pitch(p.hidden);
  with_act(p.act, [&](auto act) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < STRIPS; ++i) {
      const int64_t row = row0 + i * 32 + (lane & 31);
      const bool store = row < rows;
      float h[16], dg[16], du[16];
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float b = acc[i][1][r];
        float slope;
        activate<decltype(act)::value>(acc[i][0][r], du[r], slope);
        h[r] = du[r] * b;
        dg[r] = slope * b;
        if (!whole && col0 + 8 * (r >> 2) + 4 * half + (r & 3) >= p.hidden) dg[r] = du[r] = 0.0f;
      }
      T* const to = static_cast<T*>(p.C) + row * p.ldc + col0;
      if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const float o[4] = {h[4 * q], h[4 * q + 1], h[4 * q + 2], h[4 * q + 3]};
          const int c = 8 * q + 4 * half;
          if (whole && store)
            store_vec<T, 4>(to + c, o);
          else if (store)
            store_part<T, 4>(to + c, p.hidden - col0 - c, o);
        }
      } else {
        typedef T pair __attribute__((ext_vector_type(2)));
        uint32_t w[8];
#pragma unroll
        for (int r = 0; r < 16; r += 2) w[r / 2] = as<uint32_t>(pair{(T)h[r], (T)h[r + 1]});
#pragma unroll
        for (int q = 0; q < 4; q += 2) {
          swap_halves(w[2 * q], w[2 * q + 2]);
          swap_halves(w[2 * q + 1], w[2 * q + 3]);
          typedef uint32_t quad __attribute__((ext_vector_type(4)));
          const auto o = as<typename Packed<T, 8>::type>(quad{w[2 * q], w[2 * q + 1], w[2 * q + 2], w[2 * q + 3]});
          const int c = 8 * q + 8 * half;
          if (whole && store) {
            *reinterpret_cast<typename Packed<T, 8>::type*>(to + c) = o;
          } else if (store) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
              if (col0 + c + j < p.hidden) to[c + j] = o[j];
          }
        }
      }
      if constexpr (P::KEEP) {
        if (p.gate.q) keep_block(p.gate, dg, row, pitch, col0, store);
        if (p.up.q) keep_block(p.up, du, row, pitch, col0, store);
      }
    }
  });
}

}  // namespace fqt
