// Block quantizer to 8-bit floating point (4 exponent bits, 3 mantissa bits,
// largest value 448): codes with one power-of-two scale for each block of
// 128 along the contraction, as the matrix cores' scaled instruction reads
// them.
//
//   E = the least integer >= -127 with max|block| <= 448 2^E (0: empty block)
//   y = x 2^-E (exact),  code = the format's value nearest to y, ties to even,
//   or stochastic: with t = |y| / step, step the format's spacing at y, round
//   t up iff u < frac(t) 2^24, u the low 24 bits of the element's random word
//
// A block that holds a NaN or an infinity gets the scale byte 255 and NaN
// codes, so that the products that read it are NaN.
//
// One launch forms both operands of a matrix (x for one product, x^T for the
// other) from one read: a block of threads holds a 128 x 128 tile in
// registers, its row and column maxima give all the tile's scales.
#include "fqt_device.h"
#include "train_kernels.h"

namespace fqt {

constexpr int TILE = FP8_BLOCK;
constexpr int QT = 256;           // threads of a tile: 32 column quads x 8 row groups
constexpr int GROUP = TILE / (QT / 32);  // rows of one thread: 16

// E + 127 from the bits of the largest magnitude; 255 for NaN / Inf.
__device__ __forceinline__ uint32_t scale_byte(uint32_t top) {
  if (top == 0u) return 127u;
  if (top >= 0x7f800000u) return 255u;
  const int b = (int)(top >> 23) - 8 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0);
  return b < 0 ? 0u : (uint32_t)b;
}
// 2^-E.  (E + 127 = 255: the codes are replaced afterwards.)
__device__ __forceinline__ float scale_down(uint32_t byte) {
  return __uint_as_float((byte == 255u ? 127u : 254u - byte) << 23);
}

// Two nearest-even codes into the low or high half of w.
template <bool HI>
__device__ __forceinline__ uint32_t cvt2(float a, float b, uint32_t w) {
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(a, b, (int)w, HI);
}

// Stochastic code of y, |y| <= 448.  In units of the step 2^(max(E8, -6) - 3)
// times 2^-24, t 2^24 is an integer for |y| >= 2^-6 (24-bit significands
// with 20 bits below the step) and is rounded up to one below; adding
// 2^24 - 1 - u carries into bit 24 exactly when u < frac(t) 2^24.
__device__ __forceinline__ uint32_t stochastic_code(float y, uint32_t word) {
  const uint32_t bits = __float_as_uint(y), mag = bits & 0x7fffffffu;
  const bool small = mag < 0x3c800000u;  // 2^-6
  const uint32_t tn = ((mag & 0x7fffffu) | 0x800000u) << 4;
  const uint32_t ts = (uint32_t)ceilf(__uint_as_float(mag) * 8589934592.0f);  // 2^9 2^24
  const uint32_t r = ((small ? ts : tn) + (~word & 0xffffffu)) >> 24;
  const uint32_t base = small ? 0u : ((mag >> 23) - 121u) << 3;
  return base + r + ((bits >> 24) & 0x80u);
}

template <class T, bool ROW, bool COL, bool SQUARE, bool SR>
__global__ __launch_bounds__(QT) void fp8_tile_kernel(Fp8QuantParams p) {
  __shared__ uint32_t col_top[QT / 32][TILE];
  __shared__ __attribute__((aligned(16))) uint8_t turned[COL ? TILE * TILE : 16];
  const int tid = threadIdx.x, quad = tid & 31, grp = tid >> 5;
  const int64_t row_blocks = fp8_blocks(p.rows);
  const int64_t rb = (int64_t)blockIdx.x % row_blocks, cb = (int64_t)blockIdx.x / row_blocks;
  const int64_t r0 = rb * TILE, c0 = cb * TILE;
  const int64_t row = r0 + grp * GROUP, col = c0 + 4 * quad;
  const T* x = static_cast<const T*>(p.x) + row * p.ldx + col;
  float v[GROUP][4];
#pragma unroll
  for (int i = 0; i < GROUP; ++i) load_part<T, 4>(x + i * p.ldx, row + i < p.rows ? p.cols - col : 0, v[i]);

  // maxima of magnitudes, as integers (NaN above infinity above the rest)
  uint32_t rt[GROUP], ct[4] = {0u, 0u, 0u, 0u};
#pragma unroll
  for (int i = 0; i < GROUP; ++i) {
    rt[i] = 0u;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t m = __float_as_uint(v[i][j]) & 0x7fffffffu;
      if (ROW && !SQUARE) rt[i] = rt[i] > m ? rt[i] : m;
      ct[j] = ct[j] > m ? ct[j] : m;
    }
  }
  if constexpr (COL || SQUARE) {
#pragma unroll
    for (int j = 0; j < 4; ++j) col_top[grp][4 * quad + j] = ct[j];
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 4; ++j) {
#pragma unroll
      for (int k = 0; k < QT / 32; ++k) {
        const uint32_t m = col_top[k][4 * quad + j];
        ct[j] = ct[j] > m ? ct[j] : m;
      }
    }
  }
  uint32_t rbyte[GROUP], cbyte[4];
  if constexpr (SQUARE) {
    uint32_t m = ct[0] > ct[1] ? ct[0] : ct[1];
    const uint32_t n = ct[2] > ct[3] ? ct[2] : ct[3];
    const uint32_t b = scale_byte(half_reduce(m > n ? m : n, MaxU{}));
#pragma unroll
    for (int i = 0; i < GROUP; ++i) rbyte[i] = b;
#pragma unroll
    for (int j = 0; j < 4; ++j) cbyte[j] = b;
  } else {
#pragma unroll
    for (int i = 0; i < GROUP; ++i) rbyte[i] = ROW ? scale_byte(half_reduce(rt[i], MaxU{})) : 127u;
#pragma unroll
    for (int j = 0; j < 4; ++j) cbyte[j] = scale_byte(ct[j]);
  }

  if constexpr (ROW) {
    const int64_t pitch = fp8_pitch(p.cols), kb = fp8_blocks(p.cols);
#pragma unroll
    for (int i = 0; i < GROUP; ++i) {
      const float s = scale_down(rbyte[i]);
      uint32_t w = 0u;
      if constexpr (SR) {
        const uint64_t e = (uint64_t)(row + i) * (uint64_t)p.cols + (uint64_t)col;
        u32x4 u = philox_of_block(e >> 2, p.seed, 1u);
        const int o = (int)(e & 3);
        if (o != 0) {  // the quad spans two random blocks
          const u32x4 n = philox_of_block((e >> 2) + 1, p.seed, 1u);
          u = o == 1 ? u32x4{u.y, u.z, u.w, n.x} : (o == 2 ? u32x4{u.z, u.w, n.x, n.y} : u32x4{u.w, n.x, n.y, n.z});
        }
        w = stochastic_code(v[i][0] * s, u.x) | stochastic_code(v[i][1] * s, u.y) << 8 |
            stochastic_code(v[i][2] * s, u.z) << 16 | stochastic_code(v[i][3] * s, u.w) << 24;
      } else {
        w = cvt2<true>(v[i][2] * s, v[i][3] * s, cvt2<false>(v[i][0] * s, v[i][1] * s, 0u));
      }
      if (rbyte[i] == 255u) w = 0x7f7f7f7fu;
      if (row + i < p.rows) {
        *reinterpret_cast<uint32_t*>(p.q_row + (row + i) * pitch + col) = w;
        if (quad == 0) {
          uint8_t* e = p.e_row + ((cb >> 2) * p.rows + row + i) * 4;
          e[cb & 3] = (uint8_t)rbyte[i];
          if (cb == kb - 1)  // the blocks that fill up the last four
            for (int64_t b = (cb & 3) + 1; b < 4; ++b) e[b] = 127;
        }
      }
    }
  }
  if constexpr (COL) {
    const int64_t pitch = fp8_pitch(p.rows), kb = row_blocks;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float s = scale_down(cbyte[j]);
      uint32_t w[GROUP / 4];
#pragma unroll
      for (int i = 0; i < GROUP / 4; ++i) {
        if constexpr (SR) {
          w[i] = 0u;
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const uint64_t e = (uint64_t)(row + 4 * i + k) * (uint64_t)p.cols + (uint64_t)(col + j);
            const u32x4 u = philox_of_block(e >> 2, p.seed, 0u);
            const int o = (int)(e & 3);
            const uint32_t word = o == 0 ? u.x : (o == 1 ? u.y : (o == 2 ? u.z : u.w));
            w[i] |= stochastic_code(v[4 * i + k][j] * s, word) << (8 * k);
          }
        } else {
          w[i] = cvt2<true>(v[4 * i + 2][j] * s, v[4 * i + 3][j] * s,
                            cvt2<false>(v[4 * i][j] * s, v[4 * i + 1][j] * s, 0u));
        }
        if (cbyte[j] == 255u) w[i] = 0x7f7f7f7fu;
      }
      // column 4 quad + j, rows 16 grp ..: chunk index swizzled by the quad so
      // that eight lanes' 16-byte words fall on distinct banks
      *reinterpret_cast<uint4*>(turned + (4 * quad + j) * TILE + 16 * (grp ^ (quad & 7))) =
          make_uint4(w[0], w[1], w[2], w[3]);
    }
    if (grp == 0) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (col + j < p.cols) {
          uint8_t* e = p.e_col + ((rb >> 2) * p.cols + col + j) * 4;
          e[rb & 3] = (uint8_t)cbyte[j];
          if (rb == kb - 1)
            for (int64_t b = (rb & 3) + 1; b < 4; ++b) e[b] = 127;
        }
    }
    __syncthreads();
    // eight lanes store one column's 128-byte block
#pragma unroll
    for (int k = 0; k < TILE * TILE / 16 / QT; ++k) {
      const int c = (tid >> 3) + k * (QT / 8), chunk = tid & 7;
      const uint4 w = *reinterpret_cast<const uint4*>(turned + c * TILE + 16 * (chunk ^ ((c >> 2) & 7)));
      if (c0 + c < p.cols) *reinterpret_cast<uint4*>(p.q_col + (c0 + c) * pitch + r0 + 16 * chunk) = w;
    }
  }
}

// Codes laid out column by column, [pitch][rows], into rows [rows][pitch]:
// 128 x 128 bytes a block, turned over in LDS.
__global__ __launch_bounds__(QT) void fp8_turn_kernel(const uint8_t* src, int64_t rows, int64_t pitch, uint8_t* dst) {
  __shared__ uint8_t sh[TILE][TILE + 4];
  const int64_t kblocks = pitch / TILE;
  const int64_t k0 = (int64_t)blockIdx.x % kblocks * TILE, r0 = (int64_t)blockIdx.x / kblocks * TILE;
  for (int i = threadIdx.x; i < TILE * TILE; i += QT) {
    const int k = i / TILE, r = i % TILE;
    if (r0 + r < rows) sh[r][k] = src[(k0 + k) * rows + r0 + r];
  }
  __syncthreads();
  for (int i = threadIdx.x; i < TILE * TILE / 4; i += QT) {
    const int r = i / (TILE / 4), k = 4 * (i % (TILE / 4));
    if (r0 + r < rows)
      *reinterpret_cast<uint32_t*>(dst + (r0 + r) * pitch + k0 + k) = *reinterpret_cast<const uint32_t*>(&sh[r][k]);
  }
}

hipError_t launch_fp8_turn(const uint8_t* src, int64_t rows, int64_t K, uint8_t* dst, hipStream_t s) {
  const int64_t blocks = fp8_blocks(rows) * fp8_blocks(K);
  if (blocks > 0x7FFFFFFF) return hipErrorInvalidValue;
  hipLaunchKernelGGL(fp8_turn_kernel, dim3((unsigned)blocks), dim3(QT), 0, s, src, rows, fp8_pitch(K), dst);
  return hipGetLastError();
}

hipError_t launch_fp8_quantize(fqt_dtype type, const Fp8QuantParams& p, hipStream_t s) {
  const int64_t blocks = fp8_blocks(p.rows) * fp8_blocks(p.cols);
  if (blocks > 0x7FFFFFFF) return hipErrorInvalidValue;
  return with_type(type, [&](auto e) {
    using T = decltype(e);
    const bool row = p.q_row, col = p.q_col;
    auto go = [&](auto kernel) {
      hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(QT), 0, s, p);
      return hipGetLastError();
    };
    auto pick = [&](auto square, auto sr) {
      constexpr bool Q = decltype(square)::value, S = decltype(sr)::value;
      if (row && col) return go(fp8_tile_kernel<T, true, true, Q, S>);
      return row ? go(fp8_tile_kernel<T, true, false, Q, S>) : go(fp8_tile_kernel<T, false, true, Q, S>);
    };
    using yes = std::true_type;
    using no = std::false_type;
    if (p.tile) return p.stochastic ? pick(yes{}, yes{}) : pick(yes{}, no{});
    return p.stochastic ? pick(no{}, yes{}) : pick(no{}, no{});
  });
}

}  // namespace fqt
