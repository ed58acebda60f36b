// tree_verify.hip -- verification of drafted tokens against the target's probabilities from given
// random numbers (include/sparda.h states the rule).
//
// Every workgroup walks the tree of its sequence by itself: lane i of each wavefront holds node i's
// parent, token, random number and two probabilities, all requested at once, and the walk is scalar.  Only
// a second sibling's test after a rejection with q needs the sum of a whole row of remaining weights, which
// the workgroup then takes, with all rejections so far replayed (8 sequences of 50021 bf16 tokens: none 11 us, 2, 9 and 63
// siblings rejected in a row 21, 119 and 2916).  The workgroups of a sequence come to the same result, and their wavefronts
// share the final row: each sums the weights of pieces of 1024 tokens.  One wavefront then finds the
// piece in which the running sum passes u_0 times the total, and the token: in the same launch where one
// workgroup has all pieces, else in a second one.
//
// float64 throughout: a running sum over a vocabulary in float32 is off by more than most tokens weigh.
#include "device_util.hpp"
#include "launch.hpp"
#include "tree.hpp"

namespace sparda {

namespace {

// Wavefronts of a workgroup: with q more of them, for the sums of whole rows inside the walk.
template <bool kQ>
constexpr int kWalkWaves = kQ ? 16 : 8;
// Most pieces that one workgroup takes from walk to token (its wavefronts twice): the second launch costs the caller
// 2 us, further pieces in turn more (18 nodes of one sequence without q: 32 pieces 9.0 us against 8.4, 63 pieces 12.1).
template <bool kQ>
constexpr int kPickPieces = kQ ? 32 : 16;
constexpr int kPerLane = kVerifyPiece / 64;  // consecutive tokens of a piece that a lane holds

// What the walk leaves for the pick.
struct VerifyState {
  int32_t cur, rounds;   // the last accepted node (-1: none); rejections with q that stand there
  int32_t last;          // the node rejected last, or -1
  int32_t pad;
  uint64_t rejected;     // rejected children (q null)
};

struct VerifyWs {
  VerifyState* state;    // [batch]
  double* c;             // [batch][64]: c at each rejection with q
  double* sums;          // [batch][pieces][2]: with every rejection, and with the last one undone
};

__host__ __device__ inline VerifyWs verify_ws(void* ws, int64_t batch) {
  VerifyWs w;
  w.c = reinterpret_cast<double*>(ws);
  w.state = reinterpret_cast<VerifyState*>(w.c + batch * 64);
  w.sums = reinterpret_cast<double*>(w.state + batch);
  return w;
}
static_assert(sizeof(VerifyState) <= 64, "tree_verify_ws");

// A probability that is not a positive finite number counts as 0.  (Bits 1 .. 0x7f7fffff are the positive finite ones.)
__device__ __forceinline__ double weight_of(float x) {
  return (double)(__float_as_uint(x) - 1u < 0x7f7fffffu ? x : 0.f);
}

template <bool kBf16>
__device__ __forceinline__ double prob_at(const void* base, int64_t at) {
  if constexpr (kBf16) return weight_of(bf16_to_f32(static_cast<const uint16_t*>(base)[at]));
  return weight_of(static_cast<const float*>(base)[at]);
}

// Elements of a row before its first aligned group of four (a group is 16 bytes of float32, 8 of bf16).
template <bool kBf16>
__device__ __forceinline__ int row_shift(const void* base, int64_t at) {
  return (int)((reinterpret_cast<uintptr_t>(base) / (kBf16 ? 2 : 4) + (uintptr_t)at) & 3);
}

// The kPerLane elements of a row from e on as they lie in memory, 0 for those outside [0, vocab); e plus the row's
// shift is a multiple of 4.  They are converted by weight() afterwards, so that the loads of several rows are in flight
// together.
template <bool kBf16>
struct RawPiece {
  uint32_t w[kBf16 ? kPerLane / 2 : kPerLane];

  __device__ __forceinline__ void load(const void* base, int64_t row, int64_t e, int vocab) {
    if (e >= 0 && e + kPerLane <= vocab) {
      if constexpr (kBf16) {
        const uint2* src = reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(base) + row + e);
#pragma unroll
        for (int k = 0; k < kPerLane / 4; ++k) {
          const uint2 v = src[k];
          w[2 * k] = v.x;
          w[2 * k + 1] = v.y;
        }
      } else {
        const uint4* src = reinterpret_cast<const uint4*>(static_cast<const float*>(base) + row + e);
#pragma unroll
        for (int k = 0; k < kPerLane / 4; ++k) {
          const uint4 v = src[k];
          w[4 * k] = v.x;
          w[4 * k + 1] = v.y;
          w[4 * k + 2] = v.z;
          w[4 * k + 3] = v.w;
        }
      }
    } else {
      auto at = [&](int k) -> uint32_t {
        const bool in = e + k >= 0 && e + k < vocab;
        const int64_t from = row + (in ? e + k : 0);
        const uint32_t v = kBf16 ? (uint32_t) static_cast<const uint16_t*>(base)[from] : static_cast<const uint32_t*>(base)[from];
        return in ? v : 0u;
      };
#pragma unroll
      for (int k = 0; k < (kBf16 ? kPerLane / 2 : kPerLane); ++k) w[k] = kBf16 ? at(2 * k) | at(2 * k + 1) << 16 : at(k);
    }
  }
  __device__ __forceinline__ double weight(int k) const {
    if constexpr (kBf16) return weight_of(k & 1 ? bf16hi(w[k / 2]) : bf16lo(w[k / 2]));
    return weight_of(__uint_as_float(w[k]));
  }
};

// What `rounds` rejections with q leave of weight m; each product and difference is rounded by itself.
__device__ __forceinline__ double left_of(double m, double q, const double* c, int rounds) {
#pragma clang fp contract(off)
  for (int r = 0; r < rounds; ++r) {
    const double cut = c[r] * q;
    m = fmax(m - cut, 0.0);
  }
  return m;
}

__device__ __forceinline__ double readlane_d(double x, int lane) {
  const uint64_t u = (uint64_t)__double_as_longlong(x);
  const uint32_t lo = (uint32_t)readlane_i((int)(uint32_t)u, lane), hi = (uint32_t)readlane_i((int)(u >> 32), lane);
  return __longlong_as_double((long long)(((uint64_t)hi << 32) | lo));
}

template <int CTRL>
__device__ __forceinline__ double dpp_d(double x) {
  const uint64_t u = (uint64_t)__double_as_longlong(x);
  const uint32_t lo = (uint32_t)dpp_i<CTRL>((int)(uint32_t)u), hi = (uint32_t)dpp_i<CTRL>((int)(u >> 32));
  return __longlong_as_double((long long)(((uint64_t)hi << 32) | lo));
}

// Sum over the wavefront, the same bits in every lane: rotations inside the rows of 16 lanes, then the four rows.
__device__ __forceinline__ double wave_sum(double x) {
  x += dpp_d<0x128>(x);  // row_ror:8
  x += dpp_d<0x124>(x);
  x += dpp_d<0x122>(x);
  x += dpp_d<0x121>(x);
  return (readlane_d(x, 0) + readlane_d(x, 16)) + (readlane_d(x, 32) + readlane_d(x, 48));
}

// Sum over the workgroup, the same bits in every thread; `part` holds one double per wavefront.
template <int NW>
__device__ __forceinline__ double block_sum(double x, double* part) {
  x = wave_sum(x);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
  __syncthreads();
  double s = 0.0;
#pragma unroll
  for (int w = 0; w < NW; ++w) s += part[w];
  return s;
}

// Inclusive running sum over the wavefront's lanes.
__device__ __forceinline__ double wave_scan(double x) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const double y = __shfl_up(x, d, 64);
    if (lane >= d) x += y;
  }
  return x;
}

// A lane's kPerLane weights of a piece that begins at element e0 of the row (e0 plus the row's shift is a multiple of
// 4), after `rounds` rejections with q; *before (if given) gets their sum over the lane before the last of them.
template <bool kBf16, bool kQ>
__device__ __forceinline__ void piece_weights(const TreeVerifyArgs& a, int64_t row, int64_t e0, const double* c,
                                              int rounds, double* x, double* before) {
#pragma clang fp contract(off)
  const int lane = threadIdx.x & 63;
  auto sum = [&] {
    double s = 0.0;
#pragma unroll
    for (int k = 0; k < kPerLane; ++k) s += x[k];
    return s;
  };
  RawPiece<kBf16> rp, rq;
  if (kQ && rounds > 0) rq.load(a.q, row, e0 + kPerLane * lane, a.vocab);
  rp.load(a.p, row, e0 + kPerLane * lane, a.vocab);
#pragma unroll
  for (int k = 0; k < kPerLane; ++k) x[k] = rp.weight(k);
  if constexpr (kQ) {
    if (rounds > 0) {
      double y[kPerLane];
#pragma unroll
      for (int k = 0; k < kPerLane; ++k) y[k] = rq.weight(k);
#pragma unroll 1
      for (int r = 0; r < rounds; ++r) {
        if (before && r + 1 == rounds) *before = sum();
        const double cr = c[r];
#pragma unroll
        for (int k = 0; k < kPerLane; ++k) {
          const double cut = cr * y[k];
          x[k] = fmax(x[k] - cut, 0.0);
        }
      }
      return;
    }
  }
  if (before) *before = sum();
}

// The next token, by one wavefront: the pieces' sums, the piece, the token.  sums: [n_pieces][2], global or LDS.
template <bool kBf16, bool kQ>
__device__ __forceinline__ int pick_token(const TreeVerifyArgs& a, int b, const VerifyState& st, const double* c,
                                          const double* sums, int n_pieces) {
  const int lane = threadIdx.x & 63;
  double s1 = 0.0, s0 = 0.0;
  for (int i = lane; i < n_pieces; i += 64) {
    s1 += sums[2 * i];
    s0 += sums[2 * i + 1];
  }
  s1 = wave_sum(s1);
  s0 = wave_sum(s0);
  const int undone = s1 > 0.0 ? 0 : 1;  // the last rejection left nothing: it does not count
  const double total = undone ? s0 : s1;
  if (!(total > 0.0)) return -1;
  const double goal = (double)a.u[(int64_t)b * a.n] * total;
  // the first piece whose running sum exceeds the goal, else the last that weighs anything
  int piece = -1;
  double before = 0.0, carry = 0.0;
  for (int i0 = 0; i0 < n_pieces; i0 += 64) {
    const double x = i0 + lane < n_pieces ? sums[2 * (i0 + lane) + undone] : 0.0;
    const double run = carry + wave_scan(x);
    const uint64_t heavy = __ballot(x > 0.0), over = __ballot(x > 0.0 && run > goal);
    const int at = over ? (int)__builtin_ctzll(over) : heavy ? 63 - (int)__builtin_clzll(heavy) : -1;
    if (at >= 0) {
      piece = i0 + at;
      before = at == 0 ? carry : readlane_d(run, at - 1);
    }
    if (over) break;
    carry = readlane_d(run, 63);
  }
  const int64_t row = ((int64_t)b * a.n + st.cur) * a.ld;
  const int64_t e = (int64_t)piece * kVerifyPiece - row_shift<kBf16>(a.p, row) + kPerLane * lane;
  double x[kPerLane];
  piece_weights<kBf16, kQ>(a, row, e - kPerLane * lane, c, st.rounds - (st.rounds > 0 ? undone : 0), x, nullptr);
  if constexpr (!kQ) {
    uint64_t rejected = st.rejected;
    if (undone && st.last >= 0) rejected &= ~(1ull << st.last);
    for (; rejected; rejected &= rejected - 1) {
      const int64_t y = a.tokens[(int64_t)b * a.n + (int)__builtin_ctzll(rejected)];
#pragma unroll
      for (int k = 0; k < kPerLane; ++k) x[k] = e + k == y ? 0.0 : x[k];
    }
  }
  double own = 0.0;
#pragma unroll
  for (int k = 0; k < kPerLane; ++k) own += x[k];
  const double run = before + wave_scan(own), up = __shfl_up(run, 1, 64);
  double mine = lane == 0 ? before : up;
  int first = -1, last = -1;  // the lane's first token past the goal, and its last that weighs anything
#pragma unroll
  for (int k = 0; k < kPerLane; ++k) {
    mine += x[k];
    if (x[k] > 0.0) {
      last = (int)(e + k);
      if (first < 0 && mine > goal) first = last;
    }
  }
  const uint64_t hit = __ballot(first >= 0), any = __ballot(last >= 0);
  if (hit) return readlane_i(first, (int)__builtin_ctzll(hit));
  return any ? readlane_i(last, 63 - (int)__builtin_clzll(any)) : -1;
}

// kPick: one workgroup per sequence, which finds the token too.
template <bool kBf16, bool kQ, bool kPick>
__global__ __launch_bounds__(64 * kWalkWaves<kQ>) void tree_walk_kernel(TreeVerifyArgs a, int n_pieces) {
#pragma clang fp contract(off)
  constexpr int NW = kWalkWaves<kQ>;
  __shared__ double cs[NW][64];   // each wavefront's copy
  __shared__ double part[NW];
  __shared__ uint32_t gone[NW][kVerifyPiece / 32];
  __shared__ double piece_sums[kPick ? 2 * kPickPieces<kQ> : 2];
  __shared__ int slots[64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int b = blockIdx.y, n = a.n;
  const int64_t node0 = (int64_t)b * n;
  const uint64_t anc = tree_ancestors(a.parent + node0, n, lane);
  const int par = lane < n ? a.parent[node0 + lane] : -1;
  const int tok = lane < n ? a.tokens[node0 + lane] : -1;
  const double u = lane < n ? (double)a.u[node0 + lane] : 0.0;
  const bool cand = lane > 0 && anc != 0 && tok >= 0 && tok < a.vocab;
  const int64_t from = (node0 + (cand ? par : 0)) * a.ld + (cand ? tok : 0);
  const double pv = prob_at<kBf16>(a.p, from);
  double qv = 1.0;
  if constexpr (kQ) qv = prob_at<kBf16>(a.q, from);

  int cur = 0, rounds = 0, last = -1;
  uint64_t kept = 1ull, rejected = 0ull;
  double c = 1.0;
  bool pending = false;  // the sum after the last rejection with q is not known yet
  for (uint64_t kids = __ballot(cand && par == 0); kids;) {  // the untested children of cur, lowest node first
    const int i = (int)__builtin_ctzll(kids);
    kids &= kids - 1;
    double m = readlane_d(pv, i);
    double need = readlane_d(u, i);
    if constexpr (kQ) {
      if (pending) {
        const int64_t row = (node0 + cur) * a.ld;
        const int shift = row_shift<kBf16>(a.p, row);
        double s = 0.0;
        for (int piece = wave; piece < n_pieces; piece += NW) {
          double x[kPerLane];
          piece_weights<kBf16, true>(a, row, (int64_t)piece * kVerifyPiece - shift, cs[wave], rounds, x, nullptr);
#pragma unroll
          for (int k = 0; k < kPerLane; ++k) s += x[k];
        }
        s = block_sum<NW>(s, part);
        if (s > 0.0)
          c = s;
        else
          --rounds;  // nothing is left: the rejection is undone
        pending = false;
      }
      const double qx = readlane_d(qv, i);
      m = left_of(m, qx, cs[wave], rounds);
      need = need * c * qx;
    } else {
      if (__ballot(((rejected >> lane) & 1ull) && tok == readlane_i(tok, i))) m = 0.0;  // its weight is gone
      need = need * c;
    }
    if (need < m) {
      cur = i;
      kids = __ballot(cand && par == i);
      kept |= 1ull << i;
      rounds = 0;
      last = -1;
      rejected = 0ull;
      c = 1.0;
      pending = false;
    } else {
      last = i;
      if constexpr (kQ) {
        cs[wave][rounds++] = c;
        wave_lds_sync();
        pending = true;
      } else {
        rejected |= 1ull << i;
        c = c - m > 0.0 ? c - m : 0.0;
      }
    }
  }
  const bool present = readlane_i((int)(uint32_t)anc, 0) != 0;
  const VerifyWs ws = verify_ws(a.ws, a.batch);
  const VerifyState state = {present ? cur : -1, rounds, last, 0, rejected};
  if (blockIdx.x == 0 && wave == 0) {
    slots[lane] = -1;
    wave_lds_sync();
    if (present && ((kept >> lane) & 1ull)) slots[mbcnt64(kept)] = lane;
    wave_lds_sync();
    if (lane < n) a.path[node0 + lane] = slots[lane];
    if constexpr (kQ && !kPick) ws.c[(int64_t)b * 64 + lane] = cs[0][lane];
    if (lane == 0) {
      a.n_path[b] = present ? (int)__popcll(kept) : 0;
      if constexpr (!kPick) ws.state[b] = state;
      if (!present) a.next_token[b] = -1;
    }
  }
  if (!present) return;
  // ---- the final row's weights: a piece per wavefront at a time
  const int64_t row = (node0 + cur) * a.ld;
  const int shift = row_shift<kBf16>(a.p, row);
  double* const sums = kPick ? piece_sums : ws.sums + (int64_t)b * n_pieces * 2;
  for (int piece = blockIdx.x * NW + wave; piece < n_pieces; piece += gridDim.x * NW) {
    const int64_t e0 = (int64_t)piece * kVerifyPiece - shift;
    double x[kPerLane], s1 = 0.0, s0 = 0.0;
    piece_weights<kBf16, kQ>(a, row, e0, cs[wave], rounds, x, kQ ? &s0 : nullptr);
    if constexpr (kQ) {
#pragma unroll
      for (int k = 0; k < kPerLane; ++k) s1 += x[k];
      s0 = wave_sum(s0);
      s1 = wave_sum(s1);
    } else {
      if (rejected != 0ull) {  // rejected tokens of the piece weigh nothing
        if (lane < kVerifyPiece / 32) gone[wave][lane] = 0u;
        wave_lds_sync();
        const int64_t at = tok - e0;
        if (((rejected >> lane) & 1ull) && at >= 0 && at < kVerifyPiece) atomicOr(&gone[wave][at >> 5], 1u << (at & 31));
        wave_lds_sync();
        const uint32_t bits = gone[wave][lane * kPerLane / 32] >> (lane * kPerLane % 32);
#pragma unroll
        for (int k = 0; k < kPerLane; ++k) x[k] = (bits >> k) & 1u ? 0.0 : x[k];
      }
#pragma unroll
      for (int k = 0; k < kPerLane; ++k) s1 += x[k];
      s1 = s0 = wave_sum(s1);
      if (last >= 0) {  // the last rejected token, unless an earlier rejection took its weight
        const int y = readlane_i(tok, last);
        const uint64_t same = __ballot(((rejected >> lane) & 1ull) && tok == y);
        if (y - e0 >= 0 && y - e0 < kVerifyPiece && __popcll(same) == 1) s0 += readlane_d(pv, last);
      }
    }
    if (lane == 0) {
      sums[2 * piece] = s1;
      sums[2 * piece + 1] = s0;
    }
  }
  if constexpr (kPick) {
    __syncthreads();
    if (wave == 0) {
      const int token = pick_token<kBf16, kQ>(a, b, state, cs[0], piece_sums, n_pieces);
      if (lane == 0) a.next_token[b] = token;
    }
  }
}

template <bool kBf16, bool kQ>
__global__ __launch_bounds__(64) void tree_pick_kernel(TreeVerifyArgs a, int n_pieces) {
#pragma clang fp contract(off)
  __shared__ double cs[64];
  const int b = blockIdx.x, lane = threadIdx.x;
  const VerifyWs ws = verify_ws(a.ws, a.batch);
  const VerifyState st = ws.state[b];
  if constexpr (kQ) cs[lane] = ws.c[(int64_t)b * 64 + lane];
  if (st.cur < 0) return;
  __syncthreads();
  const int token = pick_token<kBf16, kQ>(a, b, st, cs, ws.sums + (int64_t)b * n_pieces * 2, n_pieces);
  if (lane == 0) a.next_token[b] = token;
}

template <bool kBf16, bool kQ>
hipError_t launch_verify(const TreeVerifyArgs& a, hipStream_t stream) {
  const int n_pieces = tree_verify_pieces(a.vocab);
  if (n_pieces <= kPickPieces<kQ>) {
    hipLaunchKernelGGL((tree_walk_kernel<kBf16, kQ, true>), dim3(1, (unsigned)a.batch), dim3(64 * kWalkWaves<kQ>), 0, stream, a,
                       n_pieces);
    return hipGetLastError();
  }
  // workgroups per sequence: a piece per wavefront while they fit the chip twice
  const int most = (n_pieces + kWalkWaves<kQ> - 1) / kWalkWaves<kQ>, want = 512 / a.batch;
  const int wgs = want < 1 ? 1 : want < most ? want : most;
  hipLaunchKernelGGL((tree_walk_kernel<kBf16, kQ, false>), dim3((unsigned)wgs, (unsigned)a.batch), dim3(64 * kWalkWaves<kQ>), 0,
                     stream, a, n_pieces);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((tree_pick_kernel<kBf16, kQ>), dim3((unsigned)a.batch), dim3(64), 0, stream, a, n_pieces);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_tree_verify(const TreeVerifyArgs& a, hipStream_t stream) {
  if (a.q) return a.bf16 ? launch_verify<true, true>(a, stream) : launch_verify<false, true>(a, stream);
  return a.bf16 ? launch_verify<true, false>(a, stream) : launch_verify<false, false>(a, stream);
}

}  // namespace sparda
