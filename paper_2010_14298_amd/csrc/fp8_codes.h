// Block scales and nearest codes of the 8-bit floating point format, four
// elements at a time (fp8_quant.hip, fp8_gemm.hip).
#pragma once

#include "train_kernels.h"

namespace fqt {

typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
typedef short s16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

template <class To, class From>
__device__ __forceinline__ To as(From v) {
  return __builtin_bit_cast(To, v);
}
__device__ __forceinline__ uint32_t pk_max(uint32_t a, uint32_t b) {
  return as<uint32_t>(__builtin_elementwise_max(as<u16x2>(a), as<u16x2>(b)));
}
struct PkMax {
  __device__ __forceinline__ uint32_t operator()(uint32_t a, uint32_t b) const { return pk_max(a, b); }
};

// Four neighbouring elements as they were loaded, their magnitudes as 16-bit
// keys (two to a word) that sort like the magnitudes, NaN above infinity
// above the rest, and their codes.  A key decides the block's scale, so a
// float32 magnitude may be rounded up to 16 bits (sign, exponent, 7 bits): the
// bound 1.75 2^p is a key itself.
template <class T>
struct Quad;

template <>
struct Quad<float> {
  float v[4];
  __device__ __forceinline__ void load(const float* p, int64_t n) { load_part<float, 4>(p, n, v); }
  static __device__ __forceinline__ uint32_t key(uint32_t m) {
    const uint32_t up = (m + 0xffffu) >> 16;
    return m >= 0x7f800000u ? m >> 16 : (up < 0x7f7fu ? up : 0x7f7fu);
  }
  // running maxima: the row's in one value, the columns' in four
  typedef uint32_t RowTop;
  struct ColTop {
    uint32_t m[4];
  };
  __device__ __forceinline__ void top(RowTop& r, ColTop& c) const {
    r = 0u;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t m = __float_as_uint(v[j]) & 0x7fffffffu;
      r = r > m ? r : m;
      c.m[j] = c.m[j] > m ? c.m[j] : m;
    }
  }
  static __device__ __forceinline__ uint32_t row_key(RowTop r) { return key(r); }
  static __device__ __forceinline__ void col_keys(const ColTop& c, uint32_t (&w)[2]) {
    w[0] = key(c.m[0]) | key(c.m[1]) << 16;
    w[1] = key(c.m[2]) | key(c.m[3]) << 16;
  }
  static __device__ __forceinline__ uint32_t bf_keys(uint32_t w) { return w; }
  __device__ __forceinline__ float at(int j) const { return v[j]; }
  // the elements' sign bits, a byte each
  __device__ __forceinline__ uint32_t signs() const {
    const uint32_t a = __builtin_amdgcn_perm(__float_as_uint(v[1]), __float_as_uint(v[0]), 0x0c0c0703u);
    const uint32_t b = __builtin_amdgcn_perm(__float_as_uint(v[3]), __float_as_uint(v[2]), 0x07030c0cu);
    return (a | b) & 0x80808080u;
  }
  // nearest codes of this row's quad, and of column j over four rows
  __device__ __forceinline__ uint32_t row_codes(float scale) const {
    s16x2 w = {0, 0};
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, v[0], v[1], scale, false);
    return as<uint32_t>(__builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, v[2], v[3], scale, true));
  }
  static __device__ __forceinline__ uint32_t col_codes(const Quad* q, int j, float scale) {
    s16x2 w = {0, 0};
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, q[0].v[j], q[1].v[j], scale, false);
    return as<uint32_t>(__builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, q[2].v[j], q[3].v[j], scale, true));
  }
};

// 16-bit types: two elements a word throughout.
template <class T>
struct Quad16 {
  uint32_t w[2];
  __device__ __forceinline__ void load(const T* p, int64_t n) {
    if (n >= 4) {
      const auto v = *reinterpret_cast<const typename Packed<uint16_t, 4>::type*>(p);
      w[0] = v[0] | (uint32_t)v[1] << 16;
      w[1] = v[2] | (uint32_t)v[3] << 16;
    } else {
      const uint16_t* h = reinterpret_cast<const uint16_t*>(p);
      w[0] = (n > 0 ? h[0] : 0u) | (n > 1 ? (uint32_t)h[1] << 16 : 0u);
      w[1] = n > 2 ? h[2] : 0u;
    }
  }
  typedef uint32_t RowTop;
  struct ColTop {
    uint32_t m[2];
  };
  __device__ __forceinline__ void top(RowTop& r, ColTop& c) const {
    const uint32_t a = w[0] & 0x7fff7fffu, b = w[1] & 0x7fff7fffu;
    c.m[0] = pk_max(c.m[0], a);
    c.m[1] = pk_max(c.m[1], b);
    r = pk_max(a, b);
  }
  static __device__ __forceinline__ uint32_t row_key(RowTop r) { return r >> 16 > (r & 0xffffu) ? r >> 16 : r & 0xffffu; }
  static __device__ __forceinline__ void col_keys(const ColTop& c, uint32_t (&k)[2]) {
    k[0] = c.m[0];
    k[1] = c.m[1];
  }
  __device__ __forceinline__ uint32_t signs() const { return __builtin_amdgcn_perm(w[1], w[0], 0x07050301u) & 0x80808080u; }
  // the words of rows a and b: element j of each
  static __device__ __forceinline__ uint32_t pair(uint32_t a, uint32_t b, int j) {
    return __builtin_amdgcn_perm(b, a, (j & 1) ? 0x07060302u : 0x05040100u);
  }
};

template <>
struct Quad<__bf16> : Quad16<__bf16> {
  static __device__ __forceinline__ uint32_t bf_keys(uint32_t k) { return k; }
  __device__ __forceinline__ float at(int j) const {
    return __uint_as_float((j & 1) ? w[j >> 1] & 0xffff0000u : w[j >> 1] << 16);
  }
  __device__ __forceinline__ uint32_t row_codes(float scale) const {
    s16x2 o = {0, 0};
    o = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(o, as<bf16x2>(w[0]), scale, false);
    return as<uint32_t>(__builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(o, as<bf16x2>(w[1]), scale, true));
  }
  static __device__ __forceinline__ uint32_t col_codes(const Quad* q, int j, float scale) {
    s16x2 o = {0, 0};
    o = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(o, as<bf16x2>(pair(q[0].w[j >> 1], q[1].w[j >> 1], j)), scale, false);
    return as<uint32_t>(
        __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(o, as<bf16x2>(pair(q[2].w[j >> 1], q[3].w[j >> 1], j)), scale, true));
  }
};

template <>
struct Quad<_Float16> : Quad16<_Float16> {
  // a float16 magnitude as the upper half of a float32, rounded up like Quad<float>'s
  static __device__ __forceinline__ uint32_t bf_keys(uint32_t k) {
    const f16x2 v = as<f16x2>(k);
    return Quad<float>::key(__float_as_uint((float)v[0])) | Quad<float>::key(__float_as_uint((float)v[1])) << 16;
  }
  __device__ __forceinline__ float at(int j) const { return (float)as<f16x2>(w[j >> 1])[j & 1]; }
  __device__ __forceinline__ uint32_t row_codes(float scale) const {
    s16x2 o = {0, 0};
    o = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(o, as<f16x2>(w[0]), scale, false);
    return as<uint32_t>(__builtin_amdgcn_cvt_scalef32_pk_fp8_f16(o, as<f16x2>(w[1]), scale, true));
  }
  static __device__ __forceinline__ uint32_t col_codes(const Quad* q, int j, float scale) {
    s16x2 o = {0, 0};
    o = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(o, as<f16x2>(pair(q[0].w[j >> 1], q[1].w[j >> 1], j)), scale, false);
    return as<uint32_t>(
        __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(o, as<f16x2>(pair(q[2].w[j >> 1], q[3].w[j >> 1], j)), scale, true));
  }
};

// E + 127 of a block whose largest magnitude has the given key (0: 0, a block
// of zeros; 247 where it should be NaN's 255), two at a time: the exponent,
// one more above 1.75 2^p, less the format's 8, and not below 0.
__device__ __forceinline__ uint32_t scale_bytes(uint32_t keys) {
  const u16x2 e = (as<u16x2>(keys) + (unsigned short)0x1f) >> (unsigned short)7;
  return as<uint32_t>(__builtin_elementwise_sub_sat(e, u16x2{8, 8}));
}
constexpr uint32_t NAN_KEY = 0x7f80u;  // keys from here on: infinity, NaN
__device__ __forceinline__ uint8_t stored_byte(uint32_t key, uint32_t byte) {
  return (uint8_t)(key == 0u ? 127u : (key >= NAN_KEY ? 255u : byte));
}
// 2^E, and its inverse.  (Byte 0 is the subnormal 2^-127.)
__device__ __forceinline__ float scale_up(uint32_t byte) { return __uint_as_float(byte ? byte << 23 : 0x400000u); }
__device__ __forceinline__ float scale_down(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }

}  // namespace fqt
