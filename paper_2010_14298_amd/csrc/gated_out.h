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

// The checkpoint's codes of a token's block, 16 bytes of it in each of its two
// lanes (at 16 half), and its scale byte.
__device__ __forceinline__ uint4 block_codes(const float (&v)[16], uint8_t& stored) {
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
  stored = stored_byte(key, byte);
  return make_uint4(w[0], w[2], w[1], w[3]);
}
__device__ __forceinline__ void keep_block(const Kept& k, const float (&v)[16], int64_t row, int64_t pitch, int64_t col0,
                                           bool store) {
  uint8_t byte;
  const uint4 w = block_codes(v, byte);
  const int64_t at = row * pitch + col0;
  if (!store) return;
  *reinterpret_cast<uint4*>(k.q + at + 16 * ((threadIdx.x >> 5) & 1)) = w;
  k.e[at / KEPT_BLOCK] = byte;  // both lanes of a token store the same
}

// 32 hidden units of 16-bit H as 16 bytes a lane: words 2 q .. 2 q + 3 at column
// 8 q + 8 half, for q = 0 and 2.
template <class T>
__device__ __forceinline__ void row_words(const float (&h)[16], uint32_t (&w)[8]) {
  typedef T pair __attribute__((ext_vector_type(2)));
#pragma unroll
  for (int r = 0; r < 16; r += 2) w[r / 2] = as<uint32_t>(pair{(T)h[r], (T)h[r + 1]});
#pragma unroll
  for (int q = 0; q < 4; q += 2) {
    swap_halves(w[2 * q], w[2 * q + 2]);
    swap_halves(w[2 * q + 1], w[2 * q + 3]);
  }
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
        uint32_t w[8];
        row_words<T>(h, w);
#pragma unroll
        for (int q = 0; q < 4; q += 2) {
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

// A whole block of 128 tokens (WM of each of four waves, which hold 32 hidden units
// each) by way of LDS, 64 tokens at a time, so that the stores are whole lines:
// in lds_h 64 rows of 256 bytes of H (16-bit types), in lds_q 64 rows of 128
// bytes of each checkpoint.  16-byte chunks lie at their index XOR the row, so that
// neither side meets in a bank.  8192, 1024 -> 4096 bfloat16 with checkpoints 147 us,
// 151 with the waves' own 32 bytes of a line each.  The codes, which the backward
// reads, go past the caches: with the pass that reads H next 226 us, 229.  (H past
// them too: 232.)
template <class T, class P, class Meet>
__device__ __forceinline__ void gated_store_block(const P& p, const v16f (&acc)[4][2], int64_t row0, int64_t n0, int wn,
                                                  uint8_t* lds_h, uint8_t* lds_q, Meet meet) {
  const int lane = threadIdx.x & 63, half = lane >> 5, token = lane & 31;
  const int64_t pitch = kept_pitch(p.hidden);
  with_act(p.act, [&](auto act) __attribute__((always_inline)) {
#pragma unroll
    for (int round = 0; round < 2; ++round) {
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const int i = 2 * round + s, r0 = 32 * s + token;
        float h[16], dg[16], du[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float b = acc[i][1][r];
          float slope;
          activate<decltype(act)::value>(acc[i][0][r], du[r], slope);
          h[r] = du[r] * b;
          dg[r] = slope * b;
        }
        const int64_t row = row0 + 32 * i + token;
        if constexpr (sizeof(T) == 4) {
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const float o[4] = {h[4 * q], h[4 * q + 1], h[4 * q + 2], h[4 * q + 3]};
            store_vec<T, 4>(static_cast<T*>(p.C) + row * p.ldc + n0 + 32 * wn + 8 * q + 4 * half, o);
          }
        } else {
          uint32_t w[8];
          row_words<T>(h, w);
#pragma unroll
          for (int q = 0; q < 4; q += 2)
            *reinterpret_cast<uint4*>(lds_h + r0 * 256 + 16 * ((4 * wn + q + half) ^ (r0 & 15))) =
                make_uint4(w[2 * q], w[2 * q + 1], w[2 * q + 2], w[2 * q + 3]);
        }
        if constexpr (P::KEEP) {
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            uint8_t byte;
            *reinterpret_cast<uint4*>(lds_q + k * 8192 + r0 * 128 + 16 * ((2 * wn + half) ^ (r0 & 7))) =
                block_codes(k ? du : dg, byte);
            const Kept& to = k ? p.up : p.gate;
            if (to.q && half == 0) to.e[(row * pitch + n0) / KEPT_BLOCK + wn] = byte;
          }
        }
      }
      meet();
      const int64_t first = row0 + 64 * round;
      if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int r = 16 * wn + 4 * k + (lane >> 4), c = lane & 15;
          const auto v = *reinterpret_cast<const typename Packed<T, 8>::type*>(lds_h + r * 256 + 16 * (c ^ (r & 15)));
          *reinterpret_cast<typename Packed<T, 8>::type*>(static_cast<T*>(p.C) + (first + r) * p.ldc + n0 + 8 * c) = v;
        }
      }
      if constexpr (P::KEEP) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const Kept& to = k ? p.up : p.gate;
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const int r = 16 * wn + 8 * j + (lane >> 3), c = lane & 7;
            const uint4 v = *reinterpret_cast<const uint4*>(lds_q + k * 8192 + r * 128 + 16 * (c ^ (r & 7)));
            typedef uint32_t quad __attribute__((ext_vector_type(4)));
            quad* const at = reinterpret_cast<quad*>(to.q + (first + r) * pitch + n0 + 16 * c);
            if (to.q) __builtin_nontemporal_store(quad{v.x, v.y, v.z, v.w}, at);
          }
        }
      }
      if (round == 0) meet();
    }
  });
}

}  // namespace fqt
