// rotate.hip -- rotary positions of rows, or the gradient through them (the transposed rotation: the angle negated).
//
// Eight lanes per row (rotary.hpp); a group of eight lanes forms the angles of a token once and walks over its heads, with
// the loads of several heads under way.  Rows are read and written once, past the caches.
//
// What bounds it: the memory's rate for a copy (32717 tokens of 32 heads: 536 MB of bf16 in 101 us, 5.3 TB/s, 103 to 105 on
// inputs in turn; a copy of as much takes 104; with ordinary loads and stores it was 114; 1072 MB of float32 in 210, 5.1
// TB/s), for few rows the launch (2048 float32 rows: 4 us), for rows of one head the angles beside it (a million of bf16: 516
// MB in 120 us).
#include <type_traits>

#include "rotary.hpp"

namespace sparda {

namespace {
__device__ __forceinline__ void st16_nt(void* p, uint4 w) {
  __builtin_nontemporal_store(__builtin_bit_cast(u32x4_t, w), reinterpret_cast<u32x4_t*>(p));
}

template <bool kBf16>
__global__ __launch_bounds__(256) void rotate_kernel(RotateArgs a, int64_t n_groups, int heads, bool whole) {
  constexpr int E = kBf16 ? 8 : 4, kSlots = 8 / E, kAhead = kBf16 ? 4 : 2;
  const int c = threadIdx.x & 7;
  const int64_t grp = (int64_t)blockIdx.x * 32 + (threadIdx.x >> 3);
  if (grp >= n_groups) return;
  const int64_t tokens = (int64_t)a.batch * a.n_tok;
  const int64_t tok = grp % tokens;
  const int h0 = (int)(grp / tokens) * heads, h1 = min(h0 + heads, a.n_heads);
  const int64_t b = tok / a.n_tok, t = tok % a.n_tok;
  const int64_t x0 = b * a.x.ld_batch + t * a.x.ld_token, y0 = b * a.y.ld_batch + t * a.y.ld_token;
  typedef typename std::conditional<kBf16, uint16_t, float>::type T;
  const T* x = static_cast<const T*>(a.x.data) + x0;
  T* y = static_cast<T*>(a.y.data) + y0;
  Slot<E> slot[kSlots];
#pragma unroll
  for (int s = 0; s < kSlots; ++s) slot[s] = Slot<E>(a.rope, c + 8 * s);
  // the loads of kAhead heads under way, the first ones during the angles
  uint4 wa[kAhead][kSlots], wb[kAhead][kSlots];
  auto request = [&](int h) {
#pragma unroll
    for (int e = 0; e < kAhead; ++e) {
      if (h + e >= h1) break;
      const T* src = x + (h + e) * a.x.ld_head;
#pragma unroll
      for (int s = 0; s < kSlots; ++s) {
        wa[e][s] = ld16_nt(src + E * slot[s].a);
        wb[e][s] = ld16_nt(src + E * slot[s].b);
      }
    }
  };
  const int64_t p = a.pos[b * a.pos_ld + t];
  request(h0);
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int s = 0; s < kSlots; ++s) slot[s].angles(a.rope, p, a.backward ? -1.f : 1.f);
  for (int h = h0;;) {
#pragma unroll
    for (int e = 0; e < kAhead; ++e) {
      if (h + e >= h1) break;
      T* dst = y + (h + e) * a.y.ld_head;
#pragma unroll
      for (int s = 0; s < kSlots; ++s) {
        turn_pieces(a.rope, slot[s], wa[e][s], wb[e][s]);
        if (whole) {
          st16_nt(dst + E * slot[s].a, wa[e][s]);
          st16_nt(dst + E * slot[s].b, wb[e][s]);
        } else {
          *reinterpret_cast<uint4*>(dst + E * slot[s].a) = wa[e][s];
          *reinterpret_cast<uint4*>(dst + E * slot[s].b) = wb[e][s];
        }
      }
    }
    h += kAhead;
    if (h >= h1) return;
    request(h);
  }
}

}  // namespace

hipError_t launch_rotate(const RotateArgs& a, hipStream_t stream) {
  const int64_t tokens = (int64_t)a.batch * a.n_tok;
  const int64_t heads = rotary_heads(tokens * a.n_heads, a.n_heads);
  const int64_t groups = tokens * ((a.n_heads + heads - 1) / heads);
  // stores of whole lines pass the caches, parts of lines meet there
  const bool whole = a.rope.pairs || a.rope.rot_dim % 128 == 0;
  const dim3 grid((unsigned)((groups + 31) / 32)), block(256);
  if (a.bf16)
    hipLaunchKernelGGL(rotate_kernel<true>, grid, block, 0, stream, a, groups, (int)heads, whole);
  else
    hipLaunchKernelGGL(rotate_kernel<false>, grid, block, 0, stream, a, groups, (int)heads, whole);
  return hipGetLastError();
}

}  // namespace sparda
