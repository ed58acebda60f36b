// rotary.hpp -- turning a row of a head by its position (rotate.hip, paged_append.hip).
//
// Eight lanes share a row of 128 elements: lane c holds two chunks of eight, A and B, such that an instruction of the eight
// lanes moves whole runs of 64 bytes at least.  Where a pair is two neighbours, A is chunk c and B chunk c + 8.  Where it
// lies half the rotated part apart, the lanes c < P = rot_dim / 16 hold both sides of pairs 8 c .. 8 c + 7 (chunks c and
// c + P), the others the elements that pass (c + P and c + 8).
//
// The angle p freq is reduced in float64: at position 131072 a float32 angle is off by up to 2^-7.  Taken in turns,
// the reduction is a subtraction of the nearest whole number of quarter turns, and the rest, at most half of one, keeps an
// absolute error below 2^-26 quarter turns in float32.
#pragma once

#include "device_util.hpp"
#include "paged.hpp"

namespace sparda {

struct Turns {
  float cos[8], sin[8];
};

// The two chunks (of eight elements) that lane c of a row holds, and whether they turn.
struct Chunks {
  int a, b;
  bool turn_a, turn_b;
};
__device__ __forceinline__ Chunks rotary_chunks(const Rope& r, int c) {
  const int p = r.rot_dim >> 4;  // (half: lanes that turn)
  Chunks ch;
  ch.turn_a = r.pairs ? 8 * c < r.rot_dim : c < p;
  ch.turn_b = r.pairs ? 8 * (c + 8) < r.rot_dim : c < p;
  ch.a = r.pairs || ch.turn_a ? c : c + p;
  ch.b = !r.pairs && ch.turn_a ? c + p : c + 8;
  return ch;
}

// cos and sin of x quarter turns, |x| <= 1/2: their Taylor series, whose next terms are below 2^-29 and 2^-32 here.
// (sincospif, which reduces its argument again and looks after special values, costs twice as much: the append of 13289
// tokens of 56 heads took 74.7 us with it.)
__device__ __forceinline__ void quarter_turns(float x, float* cs, float* sn) {
  const float y = x * x;
  *sn = x * (1.5707963268f + y * (-0.64596409751f + y * (0.079692626246f + y * (-0.0046817541353f + y * 0.00016044118479f))));
  *cs = 1.f + y * (-1.2337005501f + y * (0.25366950790f + y * (-0.020863480763f + y * (0.00091926027484f + y * -0.000025202042373f))));
}

// cos and sin, scaled, of the lane's eight pairs at position p (four of A, four of B where a pair is two neighbours);
// sign -1 turns back.
__device__ __forceinline__ void rotary_turns(const Rope& r, int c, const Chunks& ch, int64_t p, float sign, Turns* t) {
  if (!ch.turn_a) return;  // (then B passes too)
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int j = r.pairs ? 4 * (i < 4 || !ch.turn_b ? ch.a : ch.b) + (i & 3) : 8 * c + i;
    const double quarters = (double)p * (r.freq[j] * 0.63661977236758134308);  // 2 / pi
    const double whole = rint(quarters);
    float cs, sn;
    quarter_turns((float)(quarters - whole), &cs, &sn);
    const int k = (int)(uint32_t)(int64_t)whole;  // its last two bits: the quadrant
    const float x = k & 1 ? sn : cs, y = k & 1 ? cs : sn;
    t->cos[i] = (k + 1) & 2 ? -r.scale * x : r.scale * x;
    t->sin[i] = sign * (k & 2 ? -r.scale * y : r.scale * y);
  }
}

// x: the lane's 16 elements, chunk A then chunk B.  (B's turns are not used where it passes.)
__device__ __forceinline__ void rotary_apply(const Rope& r, const Chunks& ch, const Turns& t, float (&x)[16]) {
  if (!ch.turn_a) return;
  if (r.pairs) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float a = x[2 * i], b = x[2 * i + 1];
      const float ya = a * t.cos[i] - b * t.sin[i], yb = a * t.sin[i] + b * t.cos[i];
      x[2 * i] = i < 4 || ch.turn_b ? ya : a;
      x[2 * i + 1] = i < 4 || ch.turn_b ? yb : b;
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

// Chunks A and B of a bf16 row, turned.  A chunk that passes keeps its bits.
__device__ __forceinline__ void rotary_row(const Rope& r, const Chunks& ch, const Turns& t, uint4& a, uint4& b) {
  if (!ch.turn_a) return;
  float x[16];
  unpack8(a, x);
  unpack8(b, x + 8);
  rotary_apply(r, ch, t, x);
  a = pack8(x);
  const uint4 y = pack8(x + 8);
  b = make_uint4(ch.turn_b ? y.x : b.x, ch.turn_b ? y.y : b.y, ch.turn_b ? y.z : b.z, ch.turn_b ? y.w : b.w);
}

}  // namespace sparda
