// tree_verify.hip -- verification of drafted tokens against the target's probabilities from given
// random numbers (include/sparda.h states the rule).
//
// Two launches.  Every workgroup of the first walks the tree of its sequence by itself: lane i of each
// wavefront holds node i's parent, token, random number and two probabilities, all requested at once,
// and the walk itself is scalar.  Only a second sibling's test after a rejection with q needs the sum of
// a whole row of remaining weights, which the workgroup then takes.  The workgroups of a sequence come
// to the same result, and each sums the final row's weights over its pieces of 4096 tokens.  The
// second launch finds the piece in which the running sum passes u_0 times the total, and the token.
//
// float64 throughout: a running sum over a vocabulary in float32 is off by more than most tokens weigh.
#include "device_util.hpp"
#include "launch.hpp"
#include "tree.hpp"

namespace sparda {

namespace {

constexpr int kWalkThreads = 512;
constexpr int kPickThreads = 1024;

// What the walk leaves in the workspace for the second launch.
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

__device__ __forceinline__ double weight_of(float x) { return x > 0.f && x < INFINITY ? (double)x : 0.0; }

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

// The row's elements e .. e + 3, of which those outside [0, vocab) are 0; e + its shift is a multiple of 4.
template <bool kBf16>
__device__ __forceinline__ void load4(const void* base, int64_t row, int64_t e, int vocab, double* x) {
  if (e >= 0 && e + 4 <= vocab) {
    if constexpr (kBf16) {
      const uint2 w = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(base) + row + e);
      x[0] = weight_of(bf16lo(w.x));
      x[1] = weight_of(bf16hi(w.x));
      x[2] = weight_of(bf16lo(w.y));
      x[3] = weight_of(bf16hi(w.y));
    } else {
      const float4 w = *reinterpret_cast<const float4*>(static_cast<const float*>(base) + row + e);
      x[0] = weight_of(w.x);
      x[1] = weight_of(w.y);
      x[2] = weight_of(w.z);
      x[3] = weight_of(w.w);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = e + i >= 0 && e + i < vocab ? prob_at<kBf16>(base, row + e + i) : 0.0;
  }
}

// What `rounds` rejections with q leave of weight m; each product and difference is rounded by itself.
__device__ __forceinline__ double left_of(double m, double q, const double* c, int rounds) {
#pragma clang fp contract(off)
  for (int r = 0; r < rounds; ++r) {
    const double cut = c[r] * q;
    m = m - cut > 0.0 ? m - cut : 0.0;
  }
  return m;
}

__device__ __forceinline__ double readlane_d(double x, int lane) {
  const uint64_t u = (uint64_t)__double_as_longlong(x);
  const uint32_t lo = (uint32_t)readlane_i((int)(uint32_t)u, lane), hi = (uint32_t)readlane_i((int)(u >> 32), lane);
  return __longlong_as_double((long long)(((uint64_t)hi << 32) | lo));
}

__device__ __forceinline__ double wave_sum(double x) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) x += __shfl_xor(x, d, 64);
  return x;
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

template <bool kBf16, bool kQ>
__global__ __launch_bounds__(kWalkThreads) void tree_walk_kernel(TreeVerifyArgs a, int n_pieces) {
#pragma clang fp contract(off)
  constexpr int NW = kWalkThreads / 64;
  __shared__ double cs[NW][64];   // each wavefront's copy
  __shared__ double part[NW];
  __shared__ uint32_t gone[kVerifyPiece / 32];
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
  for (uint64_t rest = __ballot(cand); rest; rest &= rest - 1) {
    const int i = (int)__builtin_ctzll(rest);
    if (readlane_i(par, i) != cur) continue;
    double m = readlane_d(pv, i);
    double need = readlane_d(u, i);
    if constexpr (kQ) {
      if (pending) {
        const int64_t row = (node0 + cur) * a.ld;
        const int shift = row_shift<kBf16>(a.p, row);
        double s = 0.0;
        for (int64_t e = 4 * (int)threadIdx.x - shift; e < a.vocab; e += 4 * kWalkThreads) {
          double x[4], y[4];
          load4<kBf16>(a.p, row, e, a.vocab, x);
          load4<kBf16>(a.q, row, e, a.vocab, y);
#pragma unroll
          for (int k = 0; k < 4; ++k) s += left_of(x[k], y[k], cs[wave], rounds);
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
  if (blockIdx.x == 0 && wave == 0) {
    slots[lane] = -1;
    wave_lds_sync();
    if (present && ((kept >> lane) & 1ull)) slots[mbcnt64(kept)] = lane;
    wave_lds_sync();
    if (lane < n) a.path[node0 + lane] = slots[lane];
    if constexpr (kQ) ws.c[(int64_t)b * 64 + lane] = cs[0][lane];
    if (lane == 0) {
      a.n_path[b] = present ? (int)__popcll(kept) : 0;
      ws.state[b] = {present ? cur : -1, rounds, last, 0, rejected};
    }
  }
  if (!present) return;
  // ---- the final row's weights, piece by piece
  const int64_t row = (node0 + cur) * a.ld;
  const int shift = row_shift<kBf16>(a.p, row);
  for (int piece = blockIdx.x; piece < n_pieces; piece += gridDim.x) {
    const int64_t e0 = (int64_t)piece * kVerifyPiece - shift;
    double s1 = 0.0, s0 = 0.0;
    if constexpr (!kQ) {
      __syncthreads();
      for (int i = threadIdx.x; i < kVerifyPiece / 32; i += kWalkThreads) gone[i] = 0u;
      __syncthreads();
      if (wave == 0 && ((rejected >> lane) & 1ull)) {
        const int64_t x = tok - e0;
        if (x >= 0 && x < kVerifyPiece) atomicOr(&gone[x >> 5], 1u << (x & 31));
      }
      __syncthreads();
    }
    for (int at = 4 * threadIdx.x; at < kVerifyPiece; at += 4 * kWalkThreads) {
      double x[4];
      load4<kBf16>(a.p, row, e0 + at, a.vocab, x);
      if constexpr (kQ) {
        double y[4];
        if (rounds > 0) load4<kBf16>(a.q, row, e0 + at, a.vocab, y);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const double w0 = rounds > 0 ? left_of(x[k], y[k], cs[wave], rounds - 1) : x[k];
          s0 += w0;
          s1 += rounds > 0 ? left_of(w0, y[k], cs[wave] + rounds - 1, 1) : w0;
        }
      } else {
        const uint32_t bits = gone[at >> 5] >> (at & 31);
#pragma unroll
        for (int k = 0; k < 4; ++k) s1 += (bits >> k) & 1u ? 0.0 : x[k];
      }
    }
    s1 = block_sum<NW>(s1, part);
    if constexpr (kQ) {
      s0 = block_sum<NW>(s0, part);
    } else {
      s0 = s1;
      if (last >= 0) {  // the last rejected token, unless an earlier rejection took its weight
        const int x = readlane_i(tok, last);
        const uint64_t same = __ballot(((rejected >> lane) & 1ull) && tok == x);
        if (x - e0 >= 0 && x - e0 < kVerifyPiece && __popcll(same) == 1) s0 += readlane_d(pv, last);
      }
    }
    if (threadIdx.x == 0) {
      double* out = ws.sums + ((int64_t)b * n_pieces + piece) * 2;
      out[0] = s1;
      out[1] = s0;
    }
  }
}

// Inclusive running sum over the workgroup's threads.
template <int NW>
__device__ __forceinline__ double block_scan(double x, double* part, double* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const double y = __shfl_up(x, d, 64);
    if (lane >= d) x += y;
  }
  __syncthreads();
  if (lane == 63) part[wave] = x;
  __syncthreads();
  double before = 0.0, all = 0.0;
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    before += w < wave ? part[w] : 0.0;
    all += part[w];
  }
  *total = all;
  return before + x;
}

template <bool kBf16, bool kQ>
__global__ __launch_bounds__(kPickThreads) void tree_pick_kernel(TreeVerifyArgs a, int n_pieces) {
#pragma clang fp contract(off)
  constexpr int NW = kPickThreads / 64;
  __shared__ double part[NW];
  __shared__ double cs[64];
  __shared__ double at_piece;
  __shared__ int found, spare;
  const int b = blockIdx.x, tid = threadIdx.x;
  const VerifyWs ws = verify_ws(a.ws, a.batch);
  const VerifyState st = ws.state[b];
  if (st.cur < 0) {
    if (tid == 0) a.next_token[b] = -1;
    return;
  }
  const double* sums = ws.sums + (int64_t)b * n_pieces * 2;
  if (kQ && tid < 64) cs[tid] = ws.c[(int64_t)b * 64 + tid];
  double s1 = 0.0, s0 = 0.0;
  for (int i = tid; i < n_pieces; i += kPickThreads) {
    s1 += sums[2 * i];
    s0 += sums[2 * i + 1];
  }
  s1 = block_sum<NW>(s1, part);
  s0 = block_sum<NW>(s0, part);
  const int undone = s1 > 0.0 ? 0 : 1;  // the last rejection left nothing: it does not count
  const double total = undone ? s0 : s1;
  if (!(total > 0.0)) {
    if (tid == 0) a.next_token[b] = -1;
    return;
  }
  const double goal = (double)a.u[(int64_t)b * a.n] * total;
  // ---- the piece: the first whose running sum exceeds the goal, else the last that weighs anything
  if (tid == 0) {
    found = 0x7fffffff;
    spare = -1;
  }
  double carry = 0.0;
  for (int i0 = 0; i0 < n_pieces; i0 += kPickThreads) {
    const int i = i0 + tid;
    const double x = i < n_pieces ? sums[2 * i + undone] : 0.0;
    double all;
    const double run = carry + block_scan<NW>(x, part, &all);
    if (x > 0.0) {
      if (run > goal) atomicMin(&found, i);
      atomicMax(&spare, i);
    }
    carry += all;
    __syncthreads();
    if (found != 0x7fffffff) break;
  }
  const int piece = found != 0x7fffffff ? found : spare;
  carry = 0.0;
  for (int i0 = 0; i0 < n_pieces; i0 += kPickThreads) {  // what lies before it
    const int i = i0 + tid;
    double all;
    const double x = i < n_pieces ? sums[2 * i + undone] : 0.0;
    const double run = carry + block_scan<NW>(x, part, &all);
    if (i == piece) at_piece = run - x;
    carry += all;
  }
  __syncthreads();
  const double before = at_piece;
  if (tid == 0) {
    found = 0x7fffffff;
    spare = -1;
  }
  __syncthreads();
  // ---- the token inside the piece: thread t holds four consecutive ones
  const int64_t row = ((int64_t)b * a.n + st.cur) * a.ld;
  const int64_t e = (int64_t)piece * kVerifyPiece - row_shift<kBf16>(a.p, row) + 4 * tid;
  double x[4];
  load4<kBf16>(a.p, row, e, a.vocab, x);
  if constexpr (kQ) {
    const int rounds = st.rounds - (st.rounds > 0 ? undone : 0);
    if (rounds > 0) {
      double y[4];
      load4<kBf16>(a.q, row, e, a.vocab, y);
#pragma unroll
      for (int k = 0; k < 4; ++k) x[k] = left_of(x[k], y[k], cs, rounds);
    }
  } else {
    uint64_t rejected = st.rejected;
    if (undone && st.last >= 0) rejected &= ~(1ull << st.last);
    for (; rejected; rejected &= rejected - 1) {
      const int64_t y = a.tokens[(int64_t)b * a.n + (int)__builtin_ctzll(rejected)];
#pragma unroll
      for (int k = 0; k < 4; ++k) x[k] = e + k == y ? 0.0 : x[k];
    }
  }
  double all;
  double run = before + block_scan<NW>(x[0] + x[1] + x[2] + x[3], part, &all) - (x[0] + x[1] + x[2] + x[3]);
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    run += x[k];
    if (x[k] > 0.0) {
      if (run > goal) atomicMin(&found, (int)(e + k));
      atomicMax(&spare, (int)(e + k));
    }
  }
  __syncthreads();
  if (tid == 0) a.next_token[b] = found != 0x7fffffff ? found : spare;
}

template <bool kBf16, bool kQ>
hipError_t launch_verify(const TreeVerifyArgs& a, hipStream_t stream) {
  const int n_pieces = (int)(((int64_t)a.vocab + 7 + kVerifyPiece - 1) / kVerifyPiece);
  hipLaunchKernelGGL((tree_walk_kernel<kBf16, kQ>), dim3(1, (unsigned)a.batch), dim3(kWalkThreads), 0, stream, a,
                     n_pieces);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((tree_pick_kernel<kBf16, kQ>), dim3((unsigned)a.batch), dim3(kPickThreads), 0, stream, a, n_pieces);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_tree_verify(const TreeVerifyArgs& a, hipStream_t stream) {
  if (a.q) return a.bf16 ? launch_verify<true, true>(a, stream) : launch_verify<false, true>(a, stream);
  return a.bf16 ? launch_verify<true, false>(a, stream) : launch_verify<false, false>(a, stream);
}

}  // namespace sparda
