// rotate.hip -- rotary positions of rows, or the gradient through them (the transposed rotation: the angle negated).
//
// Eight lanes per row (rotary.hpp); a group of eight lanes forms the angles of a token once and walks over its heads, with
// the loads of several heads under way.  Rows are read and written once, past the caches.
//
// What bounds it: the memory's rate for a copy (32717 tokens of 32 heads: 536 MB in 101 us, 5.3 TB/s; a copy of as much takes
// 104 us; with ordinary loads and stores it was 114 us), for few rows the launch (2048 float32 rows: 4 us).
#include "rotary.hpp"

namespace sparda {

namespace {
__device__ __forceinline__ void st16_nt(void* p, uint4 w) {
  __builtin_nontemporal_store(__builtin_bit_cast(u32x4_t, w), reinterpret_cast<u32x4_t*>(p));
}

template <bool kBf16>
__global__ __launch_bounds__(256) void rotate_kernel(RotateArgs a, int64_t n_groups, int heads) {
  const int c = threadIdx.x & 7;
  const Chunks ch = rotary_chunks(a.rope, c);
  const int64_t grp = (int64_t)blockIdx.x * 32 + (threadIdx.x >> 3);
  if (grp >= n_groups) return;
  const int64_t tokens = (int64_t)a.batch * a.n_tok;
  const int64_t tok = grp % tokens;
  const int h0 = (int)(grp / tokens) * heads, h1 = min(h0 + heads, a.n_heads);
  const int64_t b = tok / a.n_tok, t = tok % a.n_tok;
  Turns turn;
  rotary_turns(a.rope, c, ch, a.pos[b * a.pos_ld + t], a.backward ? -1.f : 1.f, &turn);
  const int64_t x0 = b * a.x.ld_batch + t * a.x.ld_token, y0 = b * a.y.ld_batch + t * a.y.ld_token;
  // the loads of kAhead heads under way (those past the last repeat it)
  constexpr int kAhead = kBf16 ? 4 : 2;
  for (int h = h0; h < h1; h += kAhead) {
    if constexpr (kBf16) {
      const uint16_t* x = static_cast<const uint16_t*>(a.x.data) + x0;
      uint16_t* y = static_cast<uint16_t*>(a.y.data) + y0;
      uint4 wa[kAhead], wb[kAhead];
#pragma unroll
      for (int e = 0; e < kAhead; ++e) {
        const uint16_t* src = x + min(h + e, h1 - 1) * a.x.ld_head;
        wa[e] = ld16_nt(src + 8 * ch.a);
        wb[e] = ld16_nt(src + 8 * ch.b);
      }
#pragma unroll
      for (int e = 0; e < kAhead; ++e) {
        if (h + e >= h1) break;
        rotary_row(a.rope, ch, turn, wa[e], wb[e]);
        uint16_t* dst = y + (h + e) * a.y.ld_head;
        st16_nt(dst + 8 * ch.a, wa[e]);
        st16_nt(dst + 8 * ch.b, wb[e]);
      }
    } else {
      const float* x = static_cast<const float*>(a.x.data) + x0;
      float* y = static_cast<float*>(a.y.data) + y0;
      uint4 w[kAhead][4];
#pragma unroll
      for (int e = 0; e < kAhead; ++e) {
        const float* src = x + min(h + e, h1 - 1) * a.x.ld_head;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[e][i] = ld16_nt(src + 8 * (i < 2 ? ch.a : ch.b) + 4 * (i & 1));
      }
#pragma unroll
      for (int e = 0; e < kAhead; ++e) {
        if (h + e >= h1) break;
        float v[16];
#pragma unroll
        for (int i = 0; i < 4; ++i) *reinterpret_cast<uint4*>(v + 4 * i) = w[e][i];
        rotary_apply(a.rope, ch, turn, v);
        float* dst = y + (h + e) * a.y.ld_head;
#pragma unroll
        for (int i = 0; i < 4; ++i) st16_nt(dst + 8 * (i < 2 ? ch.a : ch.b) + 4 * (i & 1), *reinterpret_cast<const uint4*>(v + 4 * i));
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
  const int64_t parts = (a.n_heads + heads - 1) / heads;
  heads = (a.n_heads + parts - 1) / parts;
  const int64_t groups = tokens * ((a.n_heads + heads - 1) / heads);
  const dim3 grid((unsigned)((groups + 31) / 32)), block(256);
  if (a.bf16)
    hipLaunchKernelGGL(rotate_kernel<true>, grid, block, 0, stream, a, groups, (int)heads);
  else
    hipLaunchKernelGGL(rotate_kernel<false>, grid, block, 0, stream, a, groups, (int)heads);
  return hipGetLastError();
}

}  // namespace sparda
