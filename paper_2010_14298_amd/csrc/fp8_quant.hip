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
constexpr int QT = 256;                                  // threads of a tile: 32 column quads x 8 row groups
constexpr int group_of(int threads) { return TILE / (threads / 32); }  // rows of one thread: 16
constexpr int GROUP = group_of(QT);

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

// One stochastic code of v 2^-E into byte BYTE of w, from the complement n of a
// half word u in the upper half of n.  The instruction adds n's upper 20 bits to
// the first 20 bits of what is cut off, below 2^-6 as above (checked against
// that rule on 4 M values of every size): up iff 2^4 u < floor(frac 2^20).
template <int BYTE>
__device__ __forceinline__ uint32_t half_code(uint32_t w, float v, uint32_t n, float scale) {
  return (uint32_t)__builtin_amdgcn_cvt_scalef32_sr_fp8_f32((int)w, v, (int)(n | 0xffffu), scale, BYTE);
}

__device__ __forceinline__ float larger(float a, float b) {
  return __builtin_elementwise_maximum(__builtin_fabsf(a), __builtin_fabsf(b));
}

// Where a tile's elements come from: quads of rows row .. row + GROUP - 1 at
// column col, and their random words.
template <class T>
struct MatrixSource {
  typedef T Elem;
  static constexpr int THREADS = QT;
  static constexpr bool HALVES = false;  // the operands' words are of streams 1 and 0, not halves of stream 2's
  static __device__ __forceinline__ void load(const Fp8QuantParams& p, int64_t row, int64_t col, Quad<T> (&v)[GROUP]) {
    const T* x = static_cast<const T*>(p.x) + row * p.ldx + col;
#pragma unroll
    for (int i = 0; i < GROUP; ++i) v[i].load(x + i * p.ldx, row + i < p.rows ? p.cols - col : 0);
  }
};

// One tile of 128 x 128, by a block of threads; `turned`: LDS, 16 KB where COL.
template <class Source, bool ROW, bool COL, bool SQUARE, bool SR, class From>
__device__ __forceinline__ void quantize_tile(const Fp8QuantParams& p, uint32_t block, uint8_t* turned, const From& from) {
  typedef typename Source::Elem T;
  constexpr int QT = Source::THREADS, GROUP = group_of(QT);
  __shared__ uint32_t col_top[QT / 32][TILE / 2];
  __shared__ __attribute__((aligned(8))) uint16_t keys[2][TILE];  // of the rows, of the columns
  const int tid = threadIdx.x, quad = tid & 31, grp = tid >> 5;
  const uint32_t row_blocks = (uint32_t)fp8_blocks(p.rows);
  const uint32_t cb = block / row_blocks, rb = block - cb * row_blocks;
  const int64_t r0 = (int64_t)rb * TILE, c0 = (int64_t)cb * TILE;
  const int64_t row = r0 + grp * GROUP, col = c0 + 4 * quad;
  Quad<T> v[GROUP];
  Source::load(from, row, col, v);

  // keys of the rows (two to a word) and columns
  typename Quad<T>::ColTop ct{};
  uint32_t rk[GROUP / 2], ck[2];
  if constexpr (Source::HALVES) {  // the larger magnitudes of float32, NaN above all, three at a time
    float top[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < GROUP; i += 2) {
      float r[2];
#pragma unroll
      for (int k = 0; k < 2; ++k)
        r[k] = larger(larger(v[i + k].v[0], v[i + k].v[1]), larger(v[i + k].v[2], v[i + k].v[3]));
#pragma unroll
      for (int j = 0; j < 4; ++j) top[j] = larger(larger(v[i].v[j], v[i + 1].v[j]), top[j]);
      if (ROW) rk[i / 2] = Quad<T>::row_key(__float_as_uint(r[0])) | Quad<T>::row_key(__float_as_uint(r[1])) << 16;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) ct.m[j] = __float_as_uint(top[j]);
  } else {
#pragma unroll
    for (int i = 0; i < GROUP; i += 2) {
      typename Quad<T>::RowTop a, b;
      v[i].top(a, ct);
      v[i + 1].top(b, ct);
      if (ROW && !SQUARE) rk[i / 2] = Quad<T>::row_key(a) | Quad<T>::row_key(b) << 16;
    }
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
  // rows 4 k .. of this group, column 4 quad + j: 16-byte chunks swizzled by the quad
  [[maybe_unused]] auto put = [&](int j, int k, uint32_t codes) __attribute__((always_inline)) {
    const int at = grp * GROUP + 4 * k;
    *reinterpret_cast<uint32_t*>(turned + (4 * quad + j) * TILE + 16 * ((at >> 4) ^ (quad & 7)) + (at & 15)) =
        key[j] >= NAN_KEY ? 0x7f7f7f7fu : codes;
  };
  if constexpr (SR && Source::HALVES) {
    const float up[4] = {scale_up(byte[0]), scale_up(byte[1]), scale_up(byte[2]), scale_up(byte[3])};
    // aligned: a quad's elements share one random block; all: no row is past the last
    auto codes = [&](auto aligned, auto all) __attribute__((always_inline)) {
      uint64_t e = (uint64_t)row * (uint64_t)p.cols + (uint64_t)col;
      uint8_t* to = q_row;
#pragma unroll
      for (int i = 0; i < GROUP; ++i) {
        const u32x4 u = quad_words(e, p.seed, 2u, aligned || whole);
        e += (uint64_t)p.cols;
        const uint32_t n[4] = {~u.x, ~u.y, ~u.z, ~u.w};
        if constexpr (ROW) {
          const int sh = 16 * (i & 1);
          const uint32_t key = rk[i / 2] >> sh & 0xffffu;
          const uint32_t exponent = (scale_bytes(rk[i / 2]) >> sh & 0xffffu) << 23;
          const float s = __uint_as_float(exponent > 0x400000u ? exponent : 0x400000u);  // scale_up
          uint32_t c = half_code<0>(0u, v[i].at(0), n[0], s);
          c = half_code<1>(c, v[i].at(1), n[1], s);
          c = half_code<2>(c, v[i].at(2), n[2], s);
          c = half_code<3>(c, v[i].at(3), n[3], s);
          if (all || row + i < p.rows) *reinterpret_cast<uint32_t*>(to) = key >= NAN_KEY ? 0x7f7f7f7fu : c;
          to += row_pitch;
        }
        if constexpr (COL) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            uint32_t& c = w[j][0];
            const uint32_t low = n[j] << 16;
            if ((i & 3) == 0) c = half_code<0>(0u, v[i].at(j), low, up[j]);
            if ((i & 3) == 1) c = half_code<1>(c, v[i].at(j), low, up[j]);
            if ((i & 3) == 2) c = half_code<2>(c, v[i].at(j), low, up[j]);
            if ((i & 3) == 3) c = half_code<3>(c, v[i].at(j), low, up[j]);
            asm volatile("" : "+v"(c));  // now: the compiler would keep the random words of all rows to the end
            if ((i & 3) == 3) put(j, i / 4, c);
          }
        }
        __builtin_amdgcn_sched_barrier(0);  // one row at a time: fewer registers, more waves
      }
    };
    if (whole && r0 + TILE <= p.rows)
      codes(std::true_type{}, std::true_type{});
    else
      codes(std::false_type{}, std::false_type{});
  } else if constexpr (SR) {
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
    if constexpr (GROUP < 16) {
      if constexpr (!SR) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int k = 0; k < GROUP / 4; ++k) put(j, k, w[j][k]);
      }
    } else if constexpr (!(SR && Source::HALVES)) {  // (there they lie in LDS already)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (key[j] >= NAN_KEY) w[j][0] = w[j][1] = w[j][2] = w[j][3] = 0x7f7f7f7fu;
        // column 4 quad + j, rows 16 grp ..: chunk index swizzled by the quad so
        // that eight lanes' 16-byte words fall on distinct banks
        *reinterpret_cast<uint4*>(turned + (4 * quad + j) * TILE + 16 * (grp ^ (quad & 7))) =
            make_uint4(w[j][0], w[j][1], w[j][2], w[j][3]);
      }
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
template <int QT>
__device__ __forceinline__ void turn_tile(const uint8_t* src, int64_t rows, int64_t pitch, uint8_t* dst, uint32_t block,
                                          TurnLds& sh) {
  const uint32_t kblocks = (uint32_t)(pitch / TILE);
  const int64_t k0 = (int64_t)(block % kblocks) * TILE, r0 = (int64_t)(block / kblocks) * TILE;
  const int quad = threadIdx.x & 31, grp = threadIdx.x >> 5;
  const int64_t row = r0 + 4 * quad, left = rows - row;
  constexpr int GROUP = group_of(QT);
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
  quantize_tile<MatrixSource<T>, ROW, COL, SQUARE, SR>(p, (uint32_t)block, turned, p);
}
__global__ __launch_bounds__(QT) void fp8_turn_kernel(Fp8Turn t) {
  __shared__ TurnLds sh;
  turn_tile<QT>(t.src, t.rows, fp8_pitch(t.K), t.dst, blockIdx.x, sh);
}
// Both in one launch: of every `step` blocks the last lays codes out, until there
// are `turns` of them.  They wait for memory while the others compute: a
// backward of 8192, 1024 -> 4096 bfloat16 with both kept operands to lay out takes
// 170 us, in three launches 174.5; of 1000, 512 -> 512 31.6 us, 36.6.
struct TurnPlan {
  Fp8Turn a, b;
  uint32_t turns_a, turns, step;
  // Lays this block's codes out, or names the tile that it quantizes.
  template <int THREADS>
  __device__ __forceinline__ bool turns_here(uint32_t& tile, uint8_t* room) const {
    const uint32_t before = blockIdx.x / step;  // of those that lay out, up to `turns`
    if (before >= turns || blockIdx.x - before * step != step - 1) {
      tile = blockIdx.x - (before < turns ? before : turns);
      return false;
    }
    const bool first = before < turns_a;
    const Fp8Turn t = first ? a : b;
    turn_tile<THREADS>(t.src, t.rows, fp8_pitch(t.K), t.dst, first ? before : before - turns_a, *reinterpret_cast<TurnLds*>(room));
    return true;
  }
};
template <class T, bool SR>
__global__ __launch_bounds__(QT) void fp8_tile_turn_kernel(Fp8QuantParams p, TurnPlan t) {
  __shared__ __attribute__((aligned(16))) uint8_t room[sizeof(TurnLds) > TILE * TILE ? sizeof(TurnLds) : TILE * TILE];
  uint32_t block;
  if (t.turns_here<QT>(block, room)) return;
  quantize_tile<MatrixSource<T>, true, true, false, SR>(p, block, room, p);
}

constexpr int64_t MOST_BLOCKS = (((int64_t)1 << 32) - 1) / QT;  // of one dimension: operands of 2^38 bytes
static int64_t turn_blocks(const Fp8Turn& t) { return t.src ? fp8_blocks(t.rows) * fp8_blocks(t.K) : 0; }
// For a launch of `blocks`, tiles and those that lay out (some).
static TurnPlan turn_plan(const Fp8Turn& a, const Fp8Turn& b, int64_t blocks) {
  const int64_t na = turn_blocks(a), n = na + turn_blocks(b);
  return TurnPlan{a, b, (uint32_t)na, (uint32_t)n, (uint32_t)(blocks / n)};
}

hipError_t launch_fp8_turn(const Fp8Turn& t, hipStream_t s) {
  const int64_t blocks = turn_blocks(t);
  if (blocks == 0) return hipSuccess;
  if (blocks > MOST_BLOCKS) return hipErrorInvalidValue;
  hipLaunchKernelGGL(fp8_turn_kernel, dim3((unsigned)blocks), dim3(QT), 0, s, t);
  return hipGetLastError();
}

hipError_t launch_fp8_quantize_turn(fqt_dtype type, const Fp8QuantParams& p, const Fp8Turn& a, const Fp8Turn& b,
                                    hipStream_t s) {
  const int64_t tiles = fp8_blocks(p.rows) * fp8_blocks(p.cols), blocks = tiles + turn_blocks(a) + turn_blocks(b);
  if (blocks > tiles && p.q_row && p.q_col && !p.tile && blocks <= MOST_BLOCKS) {
    return with_type(type, [&](auto e) {
      using T = decltype(e);
      auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(QT), 0, s, p, turn_plan(a, b, blocks));
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

// ---------------------------------------------------------------------------
// The gradients of a gated layer's two pre-activations, D = [G d_gate | G d_up]
// [rows, 2 hidden], formed in float32 as they are quantized: G and the
// checkpoints are read, both operands written, nothing in between.  A tile is
// one of D, whose columns hidden .. 2 hidden - 1 read G once more.
//
// One random word an element serves both operands, half each: random numbers were
// the bound, and 16 bits are as many as 16-bit G times a code leaves to round (the
// layer's own quantizer takes two words of 24 bits, which float32 would need).
// 8192 x 8192 bfloat16 (268 MB with the second read of G, 24 MB of weights and X to
// lay out): 79 us, 3.7 TB/s; vector issue 68 % busy, waits 23 % of the time.
// ---------------------------------------------------------------------------
template <class G, int THREADS_>
struct GatedSource {
  typedef float Elem;
  static constexpr int THREADS = THREADS_, GROUP = group_of(THREADS);
  static constexpr bool HALVES = true;
  const G* g;
  const uint8_t *q, *e, *q_up, *e_up;  // of the half that col lies in; of the second
  const G* g0;                         // column 0 of g's rows
  int64_t ldx, pitch, rows;
  int at, left, col, hidden;           // column within the half, columns of it from there on; column of D
  __device__ __forceinline__ GatedSource(const GatedQuantParams& p, int64_t row, int64_t c)
      : ldx(p.q.ldx), pitch(kept_pitch(p.hidden)), rows(p.q.rows - row), col((int)c), hidden((int)p.hidden) {
    const bool up = c >= hidden;
    at = col - (up ? hidden : 0);
    left = hidden - at;
    g0 = static_cast<const G*>(p.q.x) + row * ldx;
    g = g0 + at;
    q_up = p.q_up + row * pitch;
    e_up = p.e_up + row * (pitch / KEPT_BLOCK);
    q = up ? q_up : p.q_gate + row * pitch;
    e = up ? e_up : p.e_gate + row * (pitch / KEPT_BLOCK);
  }
  static __device__ __forceinline__ void decode(uint32_t codes, float scale, float (&d)[4]) {
    const auto lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(codes, scale, false);
    const auto hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(codes, scale, true);
    d[0] = lo[0];
    d[1] = lo[1];
    d[2] = hi[0];
    d[3] = hi[1];
  }
  static __device__ __forceinline__ void load(const GatedQuantParams& p, int64_t row, int64_t col, Quad<float> (&v)[GROUP]) {
    GatedSource(p, row, col).load(v);
  }
  // A wave's rows (two groups) of a tile inside one half: all loads are under
  // way before the first product.
  __device__ __forceinline__ void load(Quad<float> (&v)[GROUP]) const {
    const int c0 = col / TILE * TILE;  // the tile's first column
    const bool inside = c0 >= hidden ? c0 + TILE <= 2 * hidden : c0 + TILE <= hidden;
    if (__builtin_amdgcn_readfirstlane(inside && rows >= 2 * GROUP)) {
      if ((hidden & 3) == 0)
        load_all<true>(v);
      else
        load_all<false>(v);
      return;
    }
#pragma unroll
    for (int i = 0; i < GROUP; ++i) load_one(i, v[i]);
  }
  // ONE: the four columns of a quad lie in one block, at a word.
  template <bool ONE>
  __device__ __forceinline__ void load_all(Quad<float> (&v)[GROUP]) const {
    typedef uint32_t word __attribute__((aligned(1)));
    typename Packed<G, 4>::type gv[GROUP];
    uint32_t codes[GROUP];
    uint8_t byte[GROUP], byte2[GROUP];
    const G* gi = g;
    const uint8_t *qi = q + at, *ei = e + at / KEPT_BLOCK;
    const int next = (at + 3) / KEPT_BLOCK - at / KEPT_BLOCK;
#pragma unroll
    for (int i = 0; i < GROUP; ++i) {
      gv[i] = *reinterpret_cast<const typename Packed<G, 4>::type*>(gi);
      codes[i] = *reinterpret_cast<const word*>(qi);
      byte[i] = *ei;
      if (!ONE) byte2[i] = ei[next];
      gi += ldx;
      qi += pitch;
      ei += pitch / KEPT_BLOCK;
    }
#pragma unroll
    for (int i = 0; i < GROUP; ++i) {
      float d[4];
      decode(codes[i], scale_up(byte[i]), d);
      if (!ONE) {
        float d2[4];
        decode(codes[i], scale_up(byte2[i]), d2);
#pragma unroll
        for (int j = 0; j < 4; ++j) d[j] = (at + j) / KEPT_BLOCK == at / KEPT_BLOCK ? d[j] : d2[j];
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) v[i].v[j] = (float)gv[i][j] * d[j];
    }
  }
  __device__ __forceinline__ void load_one(int i, Quad<float>& v) const {
#pragma unroll
    for (int j = 0; j < 4; ++j) v.v[j] = 0.0f;
    if (i >= rows || left <= 0) return;
    const uint8_t* const qi = q + i * pitch;
    const uint8_t* const ei = e + i * (pitch / KEPT_BLOCK);
    float gv[4], d[4];
    if ((hidden & 3) == 0) {  // four columns of one half and one block
      load_vec<G, 4>(g + i * ldx, gv);
      uint32_t codes;
      __builtin_memcpy(&codes, qi + at, 4);
      decode(codes, scale_up(ei[at / KEPT_BLOCK]), d);
    } else if (left >= 4) {  // four of one half, but perhaps of two blocks
      load_vec<G, 4>(g + i * ldx, gv);
      uint32_t codes;
      __builtin_memcpy(&codes, qi + at, 4);
      decode(codes, 1.0f, d);
      const float s0 = scale_up(ei[at / KEPT_BLOCK]), s1 = scale_up(ei[(at + 3) / KEPT_BLOCK]);
#pragma unroll
      for (int j = 0; j < 4; ++j) d[j] *= (at + j) / KEPT_BLOCK == at / KEPT_BLOCK ? s0 : s1;
    } else {  // across the halves, or the last ones
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const bool here = j < left, next = !here && col + j < 2 * hidden;
        const int c = here ? at + j : j - left;
        float f[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        gv[j] = 0.0f;
        if (here || next) {
          gv[j] = (float)g0[i * ldx + c];
          const uint8_t* const qj = here ? qi : q_up + i * pitch;
          const uint8_t* const ej = here ? ei : e_up + i * (pitch / KEPT_BLOCK);
          decode(qj[c], scale_up(ej[c / KEPT_BLOCK]), f);
        }
        d[j] = f[0];
      }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) v.v[j] = gv[j] * d[j];
  }
};
// 256 threads a tile, sixteen rows each, hold four tiles a unit (16-bit G); with 512
// a tile takes less time, but a unit holds fewer.
template <class G, bool ROW, bool COL, bool SR, int THREADS>
__global__ __launch_bounds__(THREADS, THREADS == 512 ? 4 : sizeof(G) == 2 ? 4 : 3) void gated_tile_kernel(GatedQuantParams p) {
  __shared__ __attribute__((aligned(16))) uint8_t turned[COL ? TILE * TILE : 16];
  const int64_t block = block_id();
  if (block >= fp8_blocks(p.q.rows) * fp8_blocks(p.q.cols)) return;
  quantize_tile<GatedSource<G, THREADS>, ROW, COL, false, SR>(p.q, (uint32_t)block, turned, p);
}
// With kept operands to lay out in the same launch, as above.
template <class G, bool SR, int THREADS>
__global__ __launch_bounds__(THREADS, THREADS == 512 ? 4 : sizeof(G) == 2 ? 4 : 3) void gated_tile_turn_kernel(GatedQuantParams p,
                                                                                                             TurnPlan t) {
  __shared__ __attribute__((aligned(16))) uint8_t room[sizeof(TurnLds) > TILE * TILE ? sizeof(TurnLds) : TILE * TILE];
  uint32_t block;
  if (t.turns_here<THREADS>(block, room)) return;
  quantize_tile<GatedSource<G, THREADS>, true, true, false, SR>(p.q, block, room, p);
}

hipError_t launch_gated_quantize(fqt_dtype type, const GatedQuantParams& p, const Fp8Turn& a, const Fp8Turn& b,
                                 hipStream_t s) {
  const int64_t tiles = fp8_blocks(p.q.rows) * fp8_blocks(p.q.cols), blocks = tiles + turn_blocks(a) + turn_blocks(b);
  if (tiles > 0x7FFFFFFF) return hipErrorInvalidValue;
  // 512 threads a tile / 256, whole backward with a width of 128, us: 256 tiles 25.5 / 26.2, 1032 (hidden off four)
  // 57.7 / 64.8, 1504 63.2 / 63.9, 2048 75 / 73, 4096 130 / 123; float32 1032 60 / 66, 4096 162 / 150
  const bool wide = tiles < 1536;
  auto with_threads = [&](auto f) { return wide ? f(std::integral_constant<int, 512>{}) : f(std::integral_constant<int, 256>{}); };
  if (blocks > tiles && p.q.q_row && p.q.q_col && blocks <= MOST_BLOCKS / 2) {
    return with_type(type, [&](auto e) {
      using T = decltype(e);
      return with_threads([&](auto threads) {
        constexpr int N = decltype(threads)::value;
        auto go = [&](auto kernel) {
          hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(N), 0, s, p, turn_plan(a, b, blocks));
          return hipGetLastError();
        };
        return p.q.stochastic ? go(gated_tile_turn_kernel<T, true, N>) : go(gated_tile_turn_kernel<T, false, N>);
      });
    });
  }
  hipError_t err = launch_fp8_turn(a, s);
  if (err == hipSuccess) err = launch_fp8_turn(b, s);
  if (err != hipSuccess) return err;
  return with_type(type, [&](auto e) {
    using T = decltype(e);
    auto go = [&](auto kernel, int threads) {
      hipLaunchKernelGGL(kernel, grid_of(tiles, threads), dim3(threads), 0, s, p);
      return hipGetLastError();
    };
    auto pick = [&](auto sr) {
      constexpr bool S = decltype(sr)::value;
      if (p.q.q_row && p.q.q_col)
        return with_threads([&](auto threads) {
          constexpr int N = decltype(threads)::value;
          return go(gated_tile_kernel<T, true, true, S, N>, N);
        });
      return p.q.q_row ? go(gated_tile_kernel<T, true, false, S, QT>, QT) : go(gated_tile_kernel<T, false, true, S, QT>, QT);
    };
    return p.q.stochastic ? pick(std::true_type{}) : pick(std::false_type{});
  });
}

}  // namespace fqt
