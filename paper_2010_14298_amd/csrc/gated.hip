// Gated layer in 8-bit floating point, forward:
//
//   a = Q(X) W_gate^T,  b = Q(X) W_up^T,  H = act(a) b
//   d_gate = Q8(b act'(a)),  d_up = Q8(act(a))    (kept for the backward)
#include "fp8_codes.h"
#include "gated_act.h"

namespace fqt {

// H and the checkpoints from a and b in memory: a thread four columns, eight
// threads a block of a checkpoint.
template <class T>
__global__ __launch_bounds__(256) void gated_finish_kernel(GatedParams p) {
  const int64_t quads = kept_pitch(p.hidden) / 4, i = block_id() * 256 + threadIdx.x;
  if (i >= p.N * quads) return;  // eight threads of a block leave together
  const int64_t row = i / quads, col = (i - row * quads) * 4, n = p.hidden - col;
  const float* const at = p.part + row * 2 * p.hidden + col;
  float a[4], b[4], h[4], dg[4], du[4];
  load_part<float, 4>(at, n, a);
  load_part<float, 4>(at + p.hidden, n, b);
  with_act(p.act, [&](auto act) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float slope;
      activate<decltype(act)::value>(a[j], du[j], slope);
      h[j] = du[j] * b[j];
      dg[j] = slope * b[j];
      if (j >= n) dg[j] = du[j] = 0.0f;
    }
  });
  store_part<T, 4>(static_cast<T*>(p.H) + row * p.ldh + col, n, h);
  auto keep = [&](const Kept& k, const float (&v)[4]) {
    if (!k.q) return;
    uint32_t key = 0u;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t m = __float_as_uint(v[j]) & 0x7fffffffu;
      key = key > m ? key : m;
    }
    auto larger = [](uint32_t x, uint32_t y) { return x > y ? x : y; };
    key = larger(key, dpp<0xB1>(key));
    key = larger(key, dpp<0x4E>(key));
    key = Quad<float>::key(larger(key, dpp<0x141>(key)));
    const uint32_t byte = scale_bytes(key) & 0xffffu;
    const Quad<float> x{{v[0], v[1], v[2], v[3]}};
    const int64_t o = row * quads * 4 + col;
    *reinterpret_cast<uint32_t*>(k.q + o) = key >= NAN_KEY ? 0x7f7f7f7fu : x.row_codes(scale_up(byte));
    if (col % KEPT_BLOCK == 0) k.e[o / KEPT_BLOCK] = stored_byte(key, byte);
  };
  keep(p.gate, dg);
  keep(p.up, du);
}

hipError_t launch_gated_finish(fqt_dtype type, const GatedParams& p, hipStream_t s) {
  return with_type(type, [&](auto e) {
    using T = decltype(e);
    const int64_t threads = p.N * (kept_pitch(p.hidden) / 4);
    hipLaunchKernelGGL((gated_finish_kernel<T>), grid_of((threads + 255) / 256, 256), dim3(256), 0, s, p);
    return hipGetLastError();
  });
}

}  // namespace fqt
