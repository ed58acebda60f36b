// rotate.hip -- rotary positions of rows, or the gradient through them (the transposed rotation: the angle negated).
//
// Eight lanes per row (rotary.hpp); a group of eight lanes forms the angles of a token once and walks over its heads.
#include "rotary.hpp"

namespace sparda {

namespace {

template <bool kBf16>
__global__ __launch_bounds__(256) void rotate_kernel(RotateArgs a, int64_t n_groups, int heads) {
  const int c = threadIdx.x & 7;
  const int64_t grp = (int64_t)blockIdx.x * 32 + (threadIdx.x >> 3);
  if (grp >= n_groups) return;
  const int64_t tokens = (int64_t)a.batch * a.n_tok;
  const int64_t tok = grp % tokens;
  const int h0 = (int)(grp / tokens) * heads, h1 = min(h0 + heads, a.n_heads);
  const int64_t b = tok / a.n_tok, t = tok % a.n_tok;
  Turns turn;
  rotary_turns(a.rope, c, a.pos[b * a.pos_ld + t], a.backward ? -1.f : 1.f, &turn);
  int ca, cb;
  rotary_chunks(a.rope, c, &ca, &cb);
  const int64_t x0 = b * a.x.ld_batch + t * a.x.ld_token, y0 = b * a.y.ld_batch + t * a.y.ld_token;
  for (int h = h0; h < h1; ++h) {
    if constexpr (kBf16) {
      const uint16_t* x = static_cast<const uint16_t*>(a.x.data) + x0 + h * a.x.ld_head;
      uint16_t* y = static_cast<uint16_t*>(a.y.data) + y0 + h * a.y.ld_head;
      uint4 wa = ld16(x + 8 * ca), wb = ld16(x + 8 * cb);
      rotary_row(a.rope, c, turn, &wa, &wb);
      *reinterpret_cast<uint4*>(y + 8 * ca) = wa;
      *reinterpret_cast<uint4*>(y + 8 * cb) = wb;
    } else {
      const float* x = static_cast<const float*>(a.x.data) + x0 + h * a.x.ld_head;
      float* y = static_cast<float*>(a.y.data) + y0 + h * a.y.ld_head;
      float v[16];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        *reinterpret_cast<float4*>(v + 4 * i) = *reinterpret_cast<const float4*>(x + 8 * ca + 4 * i);
        *reinterpret_cast<float4*>(v + 8 + 4 * i) = *reinterpret_cast<const float4*>(x + 8 * cb + 4 * i);
      }
      rotary_apply(a.rope, c, turn, v);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        *reinterpret_cast<float4*>(y + 8 * ca + 4 * i) = *reinterpret_cast<const float4*>(v + 4 * i);
        *reinterpret_cast<float4*>(y + 8 * cb + 4 * i) = *reinterpret_cast<const float4*>(v + 8 + 4 * i);
      }
    }
  }
}

}  // namespace

hipError_t launch_rotate(const RotateArgs& a, hipStream_t stream) {
  const int64_t tokens = (int64_t)a.batch * a.n_tok;
  // heads of a group of lanes: all of them while that leaves about eight wavefronts per SIMD, else fewer
  int64_t heads = tokens * a.n_heads / 65536;
  heads = heads < 1 ? 1 : heads > a.n_heads ? a.n_heads : heads;
  const int64_t groups = tokens * ((a.n_heads + heads - 1) / heads);
  const dim3 grid((unsigned)((groups + 31) / 32)), block(256);
  if (a.bf16)
    hipLaunchKernelGGL(rotate_kernel<true>, grid, block, 0, stream, a, groups, (int)heads);
  else
    hipLaunchKernelGGL(rotate_kernel<false>, grid, block, 0, stream, a, groups, (int)heads);
  return hipGetLastError();
}

}  // namespace sparda
