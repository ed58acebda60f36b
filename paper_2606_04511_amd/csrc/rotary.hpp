// rotary.hpp -- turning a row of a head by its position (rotate.hip, paged_append.hip).
//
// Eight lanes share a row of 128 elements, which they move in pieces of 16 bytes (E elements: 8 of bf16, 4 of float32).
// A slot is two pieces, A and B, and holds E pairs: lane c has slot c, of float32 rows slot c + 8 too.  With n pieces in a
// row, slot q holds pieces q and q + n / 2 where a pair is two neighbours.  Where it lies half the rotated part apart, the
// slots q < T = rot_dim / (2 E) hold both sides of pairs E q .. E q + E - 1 (pieces q and q + T), the others pieces that pass
// (q + T and q + n / 2).  An instruction of the eight lanes moves one run of 128 bytes, or two where the turned slots end
// among them (halves apart, bf16: runs of rot_dim and 128 - rot_dim bytes).
//
// The angle p freq is reduced in float64: at position 131072 a float32 angle is off by up to 2^-7.  Taken in turns,
// the reduction is a subtraction of the nearest whole number, and the rest, at most half a turn, keeps an
// absolute error below 2^-25 turns in float32.
#pragma once

#include "device_util.hpp"
#include "paged.hpp"

namespace sparda {

// cos and sin of x quarter turns, |x| <= 1/2: their Taylor series, whose next terms are below 2^-29 and 2^-32 here.
// (sincospif reduces its argument again and looks after special values: the append of 13289 tokens of 56 heads took 74.7 us
// with it, 73.2 without.)
__device__ __forceinline__ void quarter_turns(float x, float* cs, float* sn) {
  const float y = x * x;
  *sn = x * (1.5707963268f + y * (-0.64596409751f + y * (0.079692626246f + y * (-0.0046817541353f + y * 0.00016044118479f))));
  *cs = 1.f + y * (-1.2337005501f + y * (0.25366950790f + y * (-0.020863480763f + y * (0.00091926027484f + y * -0.000025202042373f))));
}

template <int E>
struct Slot {
  static constexpr int kPieces = 128 / E;
  int a, b;             // the pieces
  bool turn_a, turn_b;  // (B passes where A does)
  int pairs_a, pairs_b; // the first pair of A, and of B where a pair is two neighbours
  float cos[E], sin[E];

  __device__ __forceinline__ Slot() {}
  __device__ __forceinline__ Slot(const Rope& r, int q) {
    const int t = r.rot_dim / (2 * E);
    turn_a = r.pairs ? E * q < r.rot_dim : q < t;
    turn_b = r.pairs ? E * (q + kPieces / 2) < r.rot_dim : q < t;
    a = r.pairs || turn_a ? q : q + t;
    b = !r.pairs && turn_a ? q + t : q + kPieces / 2;
    pairs_a = r.pairs ? E / 2 * a : E * q;
    pairs_b = turn_b ? E / 2 * b : pairs_a;
  }

  // cos and sin, scaled, of the slot's pairs at position p; sign -1 turns back.
  __device__ __forceinline__ void angles(const Rope& r, int64_t p, float sign) {
    if (!turn_a) return;
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const int j = r.pairs ? (i < E / 2 ? pairs_a + i : pairs_b + i - E / 2) : pairs_a + i;
      const double turns = (double)p * (r.freq[j] * 0.15915494309189533577);  // 1 / (2 pi)
      const float rest = 4.f * (float)(turns - rint(turns)), whole = rintf(rest);
      float cs, sn;
      quarter_turns(rest - whole, &cs, &sn);
      const int k = (int)whole;  // its last two bits: the quadrant
      const float x = k & 1 ? sn : cs, y = k & 1 ? cs : sn;
      cos[i] = (k + 1) & 2 ? -r.scale * x : r.scale * x;
      sin[i] = sign * (k & 2 ? -r.scale * y : r.scale * y);
    }
  }

  // x: A's elements, then B's.  (B's angles are not used where it passes.)
  __device__ __forceinline__ void apply(const Rope& r, float (&x)[2 * E]) const {
    if (!turn_a) return;
    if (r.pairs) {
#pragma unroll
      for (int i = 0; i < E; ++i) {
        const float u = x[2 * i], v = x[2 * i + 1];
        const float yu = u * cos[i] - v * sin[i], yv = u * sin[i] + v * cos[i];
        x[2 * i] = i < E / 2 || turn_b ? yu : u;
        x[2 * i + 1] = i < E / 2 || turn_b ? yv : v;
      }
    } else {
#pragma unroll
      for (int i = 0; i < E; ++i) {
        const float u = x[i], v = x[E + i];
        x[i] = u * cos[i] - v * sin[i];
        x[E + i] = u * sin[i] + v * cos[i];
      }
    }
  }
};

__device__ __forceinline__ void unpack8(uint4 w, float* x) {
  x[0] = bf16lo(w.x); x[1] = bf16hi(w.x);
  x[2] = bf16lo(w.y); x[3] = bf16hi(w.y);
  x[4] = bf16lo(w.z); x[5] = bf16hi(w.z);
  x[6] = bf16lo(w.w); x[7] = bf16hi(w.w);
}
__device__ __forceinline__ uint4 pack8(const float* x) {
  return make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
}

// A slot's pieces, turned.  A piece that passes keeps its bits.
__device__ __forceinline__ void turn_pieces(const Rope& r, const Slot<8>& t, uint4& a, uint4& b) {
  if (!t.turn_a) return;
  float x[16];
  unpack8(a, x);
  unpack8(b, x + 8);
  t.apply(r, x);
  a = pack8(x);
  const uint4 y = pack8(x + 8);
  b = make_uint4(t.turn_b ? y.x : b.x, t.turn_b ? y.y : b.y, t.turn_b ? y.z : b.z, t.turn_b ? y.w : b.w);
}
__device__ __forceinline__ void turn_pieces(const Rope& r, const Slot<4>& t, uint4& a, uint4& b) {
  float x[8] = {__uint_as_float(a.x), __uint_as_float(a.y), __uint_as_float(a.z), __uint_as_float(a.w),
                __uint_as_float(b.x), __uint_as_float(b.y), __uint_as_float(b.z), __uint_as_float(b.w)};
  t.apply(r, x);
  a = make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
  b = make_uint4(__float_as_uint(x[4]), __float_as_uint(x[5]), __float_as_uint(x[6]), __float_as_uint(x[7]));
}

// Heads that a group of eight lanes walks over, `rows` rows in all: enough that the angles weigh little, while the groups
// fill the chip (us with 65536 groups, 32768 and 16384, on inputs in turn: 18 heads of 5300 tokens in bf16 14.7, 11.7 and 11.4,
// in float32 21.6, 20.7 and 21.0; 40 heads of 4000 16.2, 14.8 and 18.1, 34.5, 32.0 and 37.9; an append of 500 tokens in 4
// sequences 19.1, 16.0 and 15.8, of 4001 86, 87 and 90).
constexpr int64_t kRotaryGroups = 32768;
inline int64_t rotary_heads(int64_t rows, int64_t n_heads) {
  int64_t heads = rows / kRotaryGroups;
  heads = heads < 1 ? 1 : heads > n_heads ? n_heads : heads;
  const int64_t parts = (n_heads + heads - 1) / heads;
  return (n_heads + parts - 1) / parts;
}

}  // namespace sparda
