// Block quantizer to 8-bit floating point (4 exponent bits, 3 mantissa bits,
// largest value 448): codes with one power-of-two scale for each block of
// 128 along the contraction, as the products read them.
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
//
// To nearest, 8192 x 1024 bfloat16 to both operands (34 MB): 9.9 us, 3.4 TB/s.
// Two tiles a unit, each a chain of load, maxima and store; vector issue is 40 %
// busy.  Stochastic, 8192 x 4096 bfloat16 (134 MB): 44.5 us, 3.0 TB/s, vector issue
// 90 % busy: two random blocks for four elements are 28 wide multiplies.  Where
// many elements lie far below their block's largest (1 % of rows a thousand times
// the rest) 51 us against 46.5 in the same run.
#include "fp8_codes.h"
#include "fqt_device.h"

namespace fqt {

constexpr int TILE = FP8_BLOCK;
constexpr int QT = 256;                  // threads of a tile: 32 column quads x 8 row groups
constexpr int GROUP = TILE / (QT / 32);  // rows of one thread: 16

// Stochastic codes of four elements v 2^-E, |v 2^-E| <= 448, from the low 24
// bits u of a word each.  With m the bits of |v 2^-E|: from 2^-6 on, the part
// below the format's three mantissa bits is m's low 20 bits, so u < frac 2^24
// says that u >> 4 is below them: m + 2^20 - 1 - (u >> 4) has carried into the
// code, bits 20 and up, exactly then (less the exponents' difference of 120;
// an element that is zero stays below and saturates to code 0).  Below 2^-6
// the step is 2^-9: ceil(|v 2^-E| 2^9 2^24) plus the complement of u carries
// into bit 24.  sign: the elements' sign bits, a byte each.
__device__ __forceinline__ uint32_t quad_codes(const float (&v)[4], const float (&down)[4], const u32x4& u,
                                               uint32_t sign) {
  const uint32_t word[4] = {u.x, u.y, u.z, u.w};
  uint32_t m[4], c[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    m[j] = __float_as_uint(__builtin_fabsf(v[j]) * down[j]);
    const uint32_t f = word[j] >> 4 & 0xfffffu;
    c[j] = __builtin_elementwise_sub_sat(__builtin_elementwise_sub_sat(m[j], f), (120u << 23) - 0xfffffu);
  }
  // zeros are right as they are; anything else below 2^-6 is rare where a block's
  // elements are alike: one in thousands lies that far below the largest
  const uint32_t a = m[0] < m[1] ? m[0] : m[1], b = m[2] < m[3] ? m[2] : m[3];
  if (__builtin_amdgcn_ballot_w64((a < b ? a : b) < 0x3c800000u) != 0) {
    uint32_t least = ~0u;
#pragma unroll
    for (int j = 0; j < 4; ++j) least = least < m[j] - 1u ? least : m[j] - 1u;
    if (__builtin_amdgcn_ballot_w64(least < 0x3c7fffffu) != 0) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t t = (uint32_t)ceilf(__uint_as_float(m[j]) * 8589934592.0f) + (~word[j] & 0xffffffu);
        c[j] = m[j] < 0x3c800000u ? t >> 4 : c[j];
      }
    }
  }
  // bits 20 .. 26 of each, side by side
  const u16x2 lo = as<u16x2>(__builtin_amdgcn_perm(c[1], c[0], 0x07060302u)) >> (unsigned short)4;
  const u16x2 hi = as<u16x2>(__builtin_amdgcn_perm(c[3], c[2], 0x07060302u)) >> (unsigned short)4;
  uint32_t w = __builtin_amdgcn_perm(as<uint32_t>(hi), as<uint32_t>(lo), 0x06040200u) | sign;
  asm volatile("" : "+v"(w));  // packed here: the compiler would keep all rows' codes apart to the end
  return w;
}
// 4 x 4 bytes turned over: byte k of o[j] is byte j of r[k].
__device__ __forceinline__ void turn4(const uint32_t* r, uint32_t (&o)[4]) {
  const uint32_t lo0 = __builtin_amdgcn_perm(r[1], r[0], 0x05010400u), hi0 = __builtin_amdgcn_perm(r[1], r[0], 0x07030602u);
  const uint32_t lo1 = __builtin_amdgcn_perm(r[3], r[2], 0x05010400u), hi1 = __builtin_amdgcn_perm(r[3], r[2], 0x07030602u);
  o[0] = __builtin_amdgcn_perm(lo1, lo0, 0x05040100u);
  o[1] = __builtin_amdgcn_perm(lo1, lo0, 0x07060302u);
  o[2] = __builtin_amdgcn_perm(hi1, hi0, 0x05040100u);
  o[3] = __builtin_amdgcn_perm(hi1, hi0, 0x07060302u);
}
// The random words of elements e .. e + 3.
__device__ __forceinline__ u32x4 quad_words(uint64_t e, uint64_t seed, uint32_t stream, bool whole) {
  u32x4 u = philox_of_block(e >> 2, seed, stream);
  if (!whole) {  // rows of a length off four: the quad may span two random blocks
    const int o = (int)(e & 3);
    const u32x4 n = philox_of_block((e >> 2) + 1, seed, stream);
    if (o != 0)
      u = o == 1 ? u32x4{u.y, u.z, u.w, n.x} : (o == 2 ? u32x4{u.z, u.w, n.x, n.y} : u32x4{u.w, n.x, n.y, n.z});
  }
  return u;
}

// One tile of 128 x 128, by a block of threads; `turned`: LDS, 16 KB where COL.
template <class T, bool ROW, bool COL, bool SQUARE, bool SR>
__device__ __forceinline__ void quantize_tile(const Fp8QuantParams& p, uint32_t block, uint8_t* turned) {
  __shared__ uint32_t col_top[QT / 32][TILE / 2];
  __shared__ __attribute__((aligned(8))) uint16_t keys[2][TILE];  // of the rows, of the columns
  const int tid = threadIdx.x, quad = tid & 31, grp = tid >> 5;
  const uint32_t row_blocks = (uint32_t)fp8_blocks(p.rows);
  const uint32_t cb = block / row_blocks, rb = block - cb * row_blocks;
  const int64_t r0 = (int64_t)rb * TILE, c0 = (int64_t)cb * TILE;
  const int64_t row = r0 + grp * GROUP, col = c0 + 4 * quad;
  const T* x = static_cast<const T*>(p.x) + row * p.ldx + col;
  Quad<T> v[GROUP];
#pragma unroll
  for (int i = 0; i < GROUP; ++i) v[i].load(x + i * p.ldx, row + i < p.rows ? p.cols - col : 0);

  // keys of the rows (two to a word) and columns
  typename Quad<T>::ColTop ct{};
  uint32_t rk[GROUP / 2], ck[2];
#pragma unroll
  for (int i = 0; i < GROUP; i += 2) {
    typename Quad<T>::RowTop a, b;
    v[i].top(a, ct);
    v[i + 1].top(b, ct);
    if (ROW && !SQUARE) rk[i / 2] = Quad<T>::row_key(a) | Quad<T>::row_key(b) << 16;
  }
  Quad<T>::col_keys(ct, ck);
  if constexpr (COL || SQUARE) {
    *reinterpret_cast<uint2*>(&col_top[grp][2 * quad]) = make_uint2(ck[0], ck[1]);
    __syncthreads();
#pragma unroll
    for (int k = 0; k < QT / 32; ++k) {
      const uint2 m = *reinterpret_cast<const uint2*>(&col_top[k][2 * quad]);
      ck[0] = pk_max(ck[0], m.x);
      ck[1] = pk_max(ck[1], m.y);
    }
  }
  // the scale bytes of a line of blocks: one thread each, from the keys in LDS
  auto store_bytes = [&](uint8_t* exp, int64_t lines, int64_t line, uint32_t b, uint32_t blocks,
                         uint32_t k) __attribute__((always_inline)) {
    if (line >= lines) return;
    uint8_t* e = exp + ((int64_t)(b >> 2) * lines + line) * 4;
    e[b & 3] = stored_byte(k, scale_bytes(k) & 0xffffu);
    if (b == blocks - 1)  // the blocks that fill up the last four
      for (uint32_t i = (b & 3) + 1; i < 4; ++i) e[i] = 127;
  };
  if constexpr (SQUARE) {
    const uint32_t m = half_reduce(pk_max(ck[0], ck[1]), PkMax{});
    const uint32_t one = Quad<T>::bf_keys(pk_max(m, m >> 16 | m << 16));
    ck[0] = ck[1] = one;
#pragma unroll
    for (int i = 0; i < GROUP / 2; ++i) rk[i] = one;
  } else {
    if constexpr (ROW) {
#pragma unroll
      for (int i = 0; i < GROUP / 2; ++i) rk[i] = Quad<T>::bf_keys(half_reduce(rk[i], PkMax{}));
    }
    ck[0] = Quad<T>::bf_keys(ck[0]);
    ck[1] = Quad<T>::bf_keys(ck[1]);
  }
  if (ROW && quad == 0) {
#pragma unroll
    for (int i = 0; i < GROUP / 2; i += 2)
      *reinterpret_cast<uint2*>(&keys[0][grp * GROUP + 2 * i]) = make_uint2(rk[i], rk[i + 1]);
  }
  if (COL && grp == 0) *reinterpret_cast<uint2*>(&keys[1][4 * quad]) = make_uint2(ck[0], ck[1]);
  __syncthreads();
  if (ROW && tid < TILE) store_bytes(p.e_row, p.rows, r0 + tid, cb, (uint32_t)fp8_blocks(p.cols), keys[0][tid]);
  if (COL && tid >= QT - TILE)
    store_bytes(p.e_col, p.cols, c0 + tid - (QT - TILE), rb, row_blocks, keys[1][tid - (QT - TILE)]);
  const bool whole = (p.cols & 3) == 0;  // a quad's elements share one random block

  uint32_t key[4], byte[4], w[4][GROUP / 4];  // the columns'
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int sh = 16 * (j & 1);
    key[j] = ck[j / 2] >> sh & 0xffffu;
    byte[j] = scale_bytes(ck[j / 2]) >> sh & 0xffffu;
  }
  const int64_t row_pitch = fp8_pitch(p.cols);
  uint8_t* const q_row = p.q_row + row * row_pitch + col;
  auto store_row = [&](int i, uint32_t key, uint32_t codes) __attribute__((always_inline)) {
    if (row + i < p.rows) *reinterpret_cast<uint32_t*>(q_row + i * row_pitch) = key >= NAN_KEY ? 0x7f7f7f7fu : codes;
  };
  if constexpr (SR) {
    // both operands' codes of a row together: what their random words share is
    // not kept over all rows
#pragma unroll
    for (int i = 0; i < GROUP; i += 4) {
      uint32_t r[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float f[4] = {v[i + k].at(0), v[i + k].at(1), v[i + k].at(2), v[i + k].at(3)};
        const uint32_t sign = v[i + k].signs();
        const uint64_t e = (uint64_t)(row + i + k) * (uint64_t)p.cols + (uint64_t)col;
        if constexpr (ROW) {
          const int sh = 16 * (k & 1);
          const uint32_t rkey = rk[(i + k) / 2] >> sh & 0xffffu, rbyte = scale_bytes(rk[(i + k) / 2]) >> sh & 0xffffu;
          const float s = scale_down(rbyte);
          const float down[4] = {s, s, s, s};
          store_row(i + k, rkey, quad_codes(f, down, quad_words(e, p.seed, 1u, whole), sign));
        }
        if constexpr (COL) {
          const float down[4] = {scale_down(byte[0]), scale_down(byte[1]), scale_down(byte[2]), scale_down(byte[3])};
          r[k] = quad_codes(f, down, quad_words(e, p.seed, 0u, whole), sign);
        }
        __builtin_amdgcn_sched_barrier(0);  // one row at a time: fewer registers, more waves
      }
      if constexpr (COL) {
        uint32_t o[4];
        turn4(r, o);
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j][i / 4] = o[j];
      }
    }
  } else {
    if constexpr (ROW) {
#pragma unroll
      for (int i = 0; i < GROUP; ++i) {
        const int sh = 16 * (i & 1);
        const uint32_t rbyte = scale_bytes(rk[i / 2]) >> sh & 0xffffu;
        store_row(i, rk[i / 2] >> sh & 0xffffu, v[i].row_codes(scale_up(rbyte)));
      }
    }
    if constexpr (COL) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < GROUP; i += 4) w[j][i / 4] = Quad<T>::col_codes(v + i, j, scale_up(byte[j]));
    }
  }
  if constexpr (COL) {
    const int64_t pitch = fp8_pitch(p.rows);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (key[j] >= NAN_KEY) w[j][0] = w[j][1] = w[j][2] = w[j][3] = 0x7f7f7f7fu;
      // column 4 quad + j, rows 16 grp ..: chunk index swizzled by the quad so
      // that eight lanes' 16-byte words fall on distinct banks
      *reinterpret_cast<uint4*>(turned + (4 * quad + j) * TILE + 16 * (grp ^ (quad & 7))) =
          make_uint4(w[j][0], w[j][1], w[j][2], w[j][3]);
    }
    __syncthreads();
    // eight lanes store one column's 128-byte block
#pragma unroll
    for (int k = 0; k < TILE * TILE / 16 / QT; ++k) {
      const int c = (tid >> 3) + k * (QT / 8), chunk = tid & 7;
      const uint4 o = *reinterpret_cast<const uint4*>(turned + c * TILE + 16 * (chunk ^ ((c >> 2) & 7)));
      if (c0 + c < p.cols) *reinterpret_cast<uint4*>(p.q_col + (c0 + c) * pitch + r0 + 16 * chunk) = o;
    }
  }
}

// Codes laid out column by column, [pitch][rows], into rows [rows][pitch]:
// 128 x 128 bytes a block; a thread turns 4 x 4 bytes over in registers, LDS
// gathers rows of 128.
typedef uint32_t TurnLds[TILE][TILE / 4 + 1];
__device__ __forceinline__ void turn_tile(const uint8_t* src, int64_t rows, int64_t pitch, uint8_t* dst, uint32_t block,
                                          TurnLds& sh) {
  const uint32_t kblocks = (uint32_t)(pitch / TILE);
  const int64_t k0 = (int64_t)(block % kblocks) * TILE, r0 = (int64_t)(block / kblocks) * TILE;
  const int quad = threadIdx.x & 31, grp = threadIdx.x >> 5;
  const int64_t row = r0 + 4 * quad, left = rows - row;
  uint32_t in[GROUP];
#pragma unroll
  for (int i = 0; i < GROUP; ++i) {
    const uint8_t* p = src + (k0 + grp * GROUP + i) * rows + row;
    if (left >= 4) {
      __builtin_memcpy(&in[i], p, 4);
    } else {
      in[i] = (left > 0 ? p[0] : 0u) | (left > 1 ? (uint32_t)p[1] << 8 : 0u) | (left > 2 ? (uint32_t)p[2] << 16 : 0u);
    }
  }
#pragma unroll
  for (int i = 0; i < GROUP; i += 4) {
    uint32_t o[4];
    turn4(in + i, o);
#pragma unroll
    for (int j = 0; j < 4; ++j) sh[4 * quad + j][(grp * GROUP + i) / 4] = o[j];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < TILE * TILE / 16 / QT; ++i) {
    const int r = (threadIdx.x >> 3) + i * (QT / 8), c = 4 * (threadIdx.x & 7);
    if (r0 + r < rows)
      *reinterpret_cast<uint4*>(dst + (r0 + r) * pitch + k0 + 4 * c) =
          make_uint4(sh[r][c], sh[r][c + 1], sh[r][c + 2], sh[r][c + 3]);
  }
}

template <class T, bool ROW, bool COL, bool SQUARE, bool SR>
__global__ __launch_bounds__(QT) void fp8_tile_kernel(Fp8QuantParams p) {
  __shared__ __attribute__((aligned(16))) uint8_t turned[COL ? TILE * TILE : 16];
  const int64_t block = block_id();
  if (block >= fp8_blocks(p.rows) * fp8_blocks(p.cols)) return;
  quantize_tile<T, ROW, COL, SQUARE, SR>(p, (uint32_t)block, turned);
}
__global__ __launch_bounds__(QT) void fp8_turn_kernel(Fp8Turn t) {
  __shared__ TurnLds sh;
  turn_tile(t.src, t.rows, fp8_pitch(t.K), t.dst, blockIdx.x, sh);
}
// Both in one launch: of every `step` blocks the last lays codes out, until there
// are `turns` of them.  They wait for memory while the others compute: a
// backward of 8192, 1024 -> 4096 bfloat16 with both kept operands to lay out takes
// 170 us, in three launches 174.5; of 1000, 512 -> 512 31.6 us, 36.6.
template <class T, bool SR>
__global__ __launch_bounds__(QT) void fp8_tile_turn_kernel(Fp8QuantParams p, Fp8Turn a, Fp8Turn b, uint32_t turns_a,
                                                           uint32_t turns, uint32_t step) {
  __shared__ __attribute__((aligned(16))) uint8_t room[sizeof(TurnLds) > TILE * TILE ? sizeof(TurnLds) : TILE * TILE];
  const uint32_t before = blockIdx.x / step;  // of those that lay out, up to `turns`
  if (before >= turns || blockIdx.x - before * step != step - 1) {
    quantize_tile<T, true, true, false, SR>(p, blockIdx.x - (before < turns ? before : turns), room);
  } else {
    const bool first = before < turns_a;
    const Fp8Turn t = first ? a : b;
    turn_tile(t.src, t.rows, fp8_pitch(t.K), t.dst, first ? before : before - turns_a, *reinterpret_cast<TurnLds*>(room));
  }
}

constexpr int64_t MOST_BLOCKS = (((int64_t)1 << 32) - 1) / QT;  // of one dimension: operands of 2^38 bytes
static int64_t turn_blocks(const Fp8Turn& t) { return t.src ? fp8_blocks(t.rows) * fp8_blocks(t.K) : 0; }

hipError_t launch_fp8_turn(const Fp8Turn& t, hipStream_t s) {
  const int64_t blocks = turn_blocks(t);
  if (blocks == 0) return hipSuccess;
  if (blocks > MOST_BLOCKS) return hipErrorInvalidValue;
  hipLaunchKernelGGL(fp8_turn_kernel, dim3((unsigned)blocks), dim3(QT), 0, s, t);
  return hipGetLastError();
}

hipError_t launch_fp8_quantize_turn(fqt_dtype type, const Fp8QuantParams& p, const Fp8Turn& a, const Fp8Turn& b,
                                    hipStream_t s) {
  const int64_t na = turn_blocks(a), nb = turn_blocks(b), blocks = fp8_blocks(p.rows) * fp8_blocks(p.cols) + na + nb;
  if (na + nb > 0 && p.q_row && p.q_col && !p.tile && blocks <= MOST_BLOCKS) {
    return with_type(type, [&](auto e) {
      using T = decltype(e);
      auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(QT), 0, s, p, a, b, (uint32_t)na, (uint32_t)(na + nb),
                           (uint32_t)(blocks / (na + nb)));
        return hipGetLastError();
      };
      return p.stochastic ? go(fp8_tile_turn_kernel<T, true>) : go(fp8_tile_turn_kernel<T, false>);
    });
  }
  hipError_t e = launch_fp8_turn(a, s);
  if (e == hipSuccess) e = launch_fp8_turn(b, s);
  if (e == hipSuccess && (p.q_row || p.q_col)) e = launch_fp8_quantize(type, p, s);
  return e;
}

hipError_t launch_fp8_quantize(fqt_dtype type, const Fp8QuantParams& p, hipStream_t s) {
  const int64_t blocks = fp8_blocks(p.rows) * fp8_blocks(p.cols);
  if (blocks > 0x7FFFFFFF) return hipErrorInvalidValue;
  return with_type(type, [&](auto e) {
    using T = decltype(e);
    const bool row = p.q_row, col = p.q_col;
    auto go = [&](auto kernel) {
      hipLaunchKernelGGL(kernel, grid_of(blocks, QT), dim3(QT), 0, s, p);
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
