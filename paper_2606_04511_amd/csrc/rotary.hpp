// rotary.hpp -- turning a row of a head by its position (rotate.hip, paged_append.hip).
//
// Eight lanes share a row of 128 elements: lane c holds two chunks of eight, A and B.  With P = rot_dim / 16 the
// lanes c < P hold pairs 8 c .. 8 c + 7 (chunks c and c + P where a pair lies half the rotated part apart, 2 c and
// 2 c + 1 where it is two neighbours), the others the elements that pass (2 c and 2 c + 1 in both layouts).
//
// The angle p freq is reduced in float64: at position 131072 a float32 angle is off by up to 2^-7.  Taken in turns,
// the reduction is a subtraction of the nearest whole number, and the rest, at most half a turn, keeps an
// absolute error below 2^-25 turns in float32.
#pragma once

#include "device_util.hpp"
#include "paged.hpp"

namespace sparda {

struct Turns {
  float cos[8], sin[8];
};

// The two chunks (of eight elements) that lane c of a row holds.
__device__ __forceinline__ void rotary_chunks(const Rope& r, int c, int* a, int* b) {
  const bool apart = !r.pairs && 16 * c < r.rot_dim;
  *a = apart ? c : 2 * c;
  *b = apart ? c + (r.rot_dim >> 4) : 2 * c + 1;
}

// cos and sin, scaled, of the lane's eight pairs at position p; sign -1 turns back.
__device__ __forceinline__ void rotary_turns(const Rope& r, int c, int64_t p, float sign, Turns* t) {
  if (16 * c >= r.rot_dim) return;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const double turns = (double)p * (r.freq[8 * c + i] * 0.15915494309189533577);  // 1 / (2 pi)
    const float rest = (float)(turns - rint(turns));
    float sn, cs;
    sincospif(2.f * rest, &sn, &cs);
    t->cos[i] = r.scale * cs;
    t->sin[i] = sign * r.scale * sn;
  }
}

// x: the lane's 16 elements, chunk A then chunk B.
__device__ __forceinline__ void rotary_apply(const Rope& r, int c, const Turns& t, float (&x)[16]) {
  if (16 * c >= r.rot_dim) return;
  if (r.pairs) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float a = x[2 * i], b = x[2 * i + 1];
      x[2 * i] = a * t.cos[i] - b * t.sin[i];
      x[2 * i + 1] = a * t.sin[i] + b * t.cos[i];
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float a = x[i], b = x[8 + i];
      x[i] = a * t.cos[i] - b * t.sin[i];
      x[8 + i] = a * t.sin[i] + b * t.cos[i];
    }
  }
}

__device__ __forceinline__ void unpack8(uint4 w, float* x) {
  x[0] = bf16lo(w.x); x[1] = bf16hi(w.x);
  x[2] = bf16lo(w.y); x[3] = bf16hi(w.y);
  x[4] = bf16lo(w.z); x[5] = bf16hi(w.z);
  x[6] = bf16lo(w.w); x[7] = bf16hi(w.w);
}
__device__ __forceinline__ uint4 pack8(const float* x) {
  return make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
}

// The bf16 row at src turned; *a and *b receive chunks A and B.  Lanes that pass keep their bits.
__device__ __forceinline__ void rotary_row(const Rope& r, int c, const Turns& t, uint4* a, uint4* b) {
  if (16 * c >= r.rot_dim) return;
  float x[16];
  unpack8(*a, x);
  unpack8(*b, x + 8);
  rotary_apply(r, c, t, x);
  *a = pack8(x);
  *b = pack8(x + 8);
}

}  // namespace sparda
