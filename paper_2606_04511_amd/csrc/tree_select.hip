// tree_select.hip -- the attended block sets of the nodes of drafted-token trees (paper Sec. 4.1,
// Eq. 4 with Eq. 1), for sequences of different lengths.
//
// Node i of a sequence of t committed tokens is at p = t + |A(i)| - 1.  Forced blocks and candidates
// are those of a row at p; window scores F_i . K~_w (float32 accumulation) count for the windows
// complete within the t tokens; a block's score is the largest of the windows that overlap it.
// The scores go to the workspace, then one wavefront per node selects.
#include "device_util.hpp"
#include "launch.hpp"
#include "select_block.hpp"
#include "tree.hpp"

namespace sparda {

namespace {

// The tree's depth of every lane's node (0: absent) and the sequence's context.
struct SeqGeom {
  int64_t t;
  int depth;
};
__device__ __forceinline__ SeqGeom seq_geom(const TreeBatch& tb, int b, int lane) {
  const int64_t t = tree_context(tb, b);
  const uint64_t anc = tree_ancestors(tb.parent + (int64_t)b * tb.n, tb.n, lane);
  return {t, t < 0 ? 0 : (int)__popcll(anc)};
}

// Block scores of all nodes of a (batch, group) on MFMA: the keys are read once.  A = 16 nodes' Forecast
// rows (MT of them in registers), B = 16 keys, so consecutive candidates lie in consecutive lanes.  A step
// is 64 consecutive keys, which go from memory into 16 KiB of the wavefront's own LDS in whole rows (read as
// fragments of 64 bytes per row straight from memory the same launch is 7 us longer) and from there into
// registers, so that the next step's are under way during the products: 64 blocks on the one-key-per-block grid, 16
// blocks of the (32, 16) grid as four tiles, tile u holding window u of each block.  Window -1 of a block is window 3
// of the one before: the neighbouring lane's score, or for lane 0 that of the last step (at a wavefront's first step one
// more key).
//
// What bounds it: the memory's rate and what frames it.  16 nodes of 256 groups at 128K (134 MB of keys, 33 MB of
// scores): 29 us; the top-k of their 4096 rows another 17.
template <bool kBlocks, int MT>
__global__ __launch_bounds__(256) void tree_score_kernel(TreeSelectArgs a, int n_groups, int steps) {
  constexpr int kPerStep = kBlocks ? 64 : 16;  // candidates
  __shared__ __align__(16) char bufs[4][64 * 256];
  const int lane = threadIdx.x & 63, c = lane & 15, q = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t bm = blockIdx.x % n_groups;
  const int part = (int)(blockIdx.x / n_groups) * 4 + wave;
  const int n = a.tb.n;
  const int64_t t = tree_context(a.tb, (int)(bm / a.n_kv_heads));
  if (t < 0) return;
  // the candidates of the deepest node there can be: no other node has more
  const RowGeom g = row_geom(t + n - 1, a.n_init, a.n_local, a.k_total);
  if (g.n_take >= g.n_cand) return;
  const int x_end = min(g.n_cand, (part + 1) * steps * kPerStep);
  int x0 = part * steps * kPerStep;
  if (x0 >= x_end) return;
  const int32_t vis = grid_win_vis(a.grid, t - 1);
  const int32_t last_key = tree_last_key(a.grid, t, n, a.n_init, a.n_local, a.k_total);  // nothing past it is read
  bf16x8 fa[MT][4];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    const uint16_t* src = a.f + (bm * n + min(16 * mt + c, n - 1)) * kHeadDim + 8 * q;
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) fa[mt][ks] = as_bf16x8(ld16(src + 32 * ks));
  }
  const uint16_t* keys = a.kc + bm * a.nc_cap * kHeadDim + 8 * q;
  auto key_at = [&](int w) { return keys + (int64_t)tree_key_row(w, last_key) * kHeadDim; };
  auto products = [&](const uint4* kw, int mt) {
    f32x4 s = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) s = mfma16x16x32(fa[mt][ks], as_bf16x8(kw[ks]), s);
    return s;
  };
  float* const out = a.ws + bm * n * a.ws_stride;
  auto store = [&](int mt, int x, const f32x4& s) {  // element i: node 16 mt + 4 q + i, candidate x + c
    if (x + c >= g.n_cand) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int node = 16 * mt + 4 * q + i;
      if (node < n) out[node * a.ws_stride + x + c] = s[i];
    }
  };
  f32x4 carry[MT];
  if constexpr (!kBlocks) {
    const int w = 4 * (g.cand_lo + x0) - 1;
    uint4 kw[4];
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) kw[ks] = ld16(key_at(w) + 32 * ks);
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      carry[mt] = products(kw, mt);
      if (w < 0 || w > vis) carry[mt] = f32x4{-INFINITY, -INFINITY, -INFINITY, -INFINITY};
    }
  }
  // a step's 64 keys, 4 per instruction; piece y of key row z lies at y ^ c, c the lane column that reads the row
  const int r4 = lane >> 4;
  const uint32_t buf_at = __builtin_amdgcn_readfirstlane(lds_address(bufs[wave]));
  const uint16_t* const rows = a.kc + bm * a.nc_cap * kHeadDim;
  auto request = [&](int x) {
    const int w0 = kBlocks ? g.cand_lo + x : 4 * (g.cand_lo + x);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int z = 4 * i + r4, col = kBlocks ? z & 15 : i;
      lds_load16<true>(rows, (uint32_t)tree_key_row(w0 + z, last_key) * 256 + 16 * ((lane & 15) ^ col), buf_at + 1024 * i);
    }
  };
  request(x0);
  for (; x0 < x_end; x0 += kPerStep) {
    lds_loads_landed();
    uint4 kw[4][4];
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int ks = 0; ks < 4; ++ks)
        kw[u][ks] = *reinterpret_cast<const uint4*>(&bufs[wave][(kBlocks ? 16 * u + c : 4 * c + u) * 256 + 16 * ((4 * ks + q) ^ c)]);
    __asm__ __volatile__("s_waitcnt lgkmcnt(0)" ::: "memory");  // the keys are in registers
    if (x0 + kPerStep < x_end) request(x0 + kPerStep);
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      if constexpr (kBlocks) {
#pragma unroll
        for (int u = 0; u < 4; ++u) store(mt, x0 + 16 * u, products(kw[u], mt));
      } else {
        f32x4 best, s;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          s = products(kw[u], mt);
          if (4 * (g.cand_lo + x0 + c) + u > vis) s = f32x4{-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
          for (int i = 0; i < 4; ++i) best[i] = u == 0 ? s[i] : fmaxf(best[i], s[i]);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int before = __builtin_amdgcn_update_dpp(__float_as_int(carry[mt][i]), __float_as_int(s[i]), 0x111, 0xf, 0xf, false);
          best[i] = fmaxf(best[i], __int_as_float(before));  // row_shr:1, lane 0 keeps the carry
          carry[mt][i] = dpp_f<0x121>(s[i]);                 // row_ror:1: lane 15's to lane 0
        }
        store(mt, x0, best);
      }
    }
  }
}

template <bool kBlocks>
hipError_t launch_scores(const TreeSelectArgs& a, int C, hipStream_t stream) {
  const int groups = a.tb.batch * a.n_kv_heads;
  const int total = (C + (kBlocks ? 64 : 16) - 1) / (kBlocks ? 64 : 16);
  // steps per wavefront: one while the chip is not full, else about two wavefronts per SIMD; at most 16
  const int64_t all = (int64_t)groups * total;
  const int steps = (int)(all <= 2048 ? 1 : all >= 16 * 2048 ? 16 : all / 2048);
  const int parts = (total + steps - 1) / steps;
  const dim3 grid((unsigned)(groups * ((parts + 3) / 4))), block(256);
  switch ((a.tb.n + 15) / 16) {
    case 1: hipLaunchKernelGGL((tree_score_kernel<kBlocks, 1>), grid, block, 0, stream, a, groups, steps); break;
    case 2: hipLaunchKernelGGL((tree_score_kernel<kBlocks, 2>), grid, block, 0, stream, a, groups, steps); break;
    case 3: hipLaunchKernelGGL((tree_score_kernel<kBlocks, 3>), grid, block, 0, stream, a, groups, steps); break;
    default: hipLaunchKernelGGL((tree_score_kernel<kBlocks, 4>), grid, block, 0, stream, a, groups, steps);
  }
  return hipGetLastError();
}

// One wavefront's exact top-k over C <= 64 R scores in its registers (candidate 64 i + lane is x[i]; 0 < n < C; ties to
// the lower index), by value bins: 256 equal-width bins over the scores' range (a higher bin holds only larger scores),
// a histogram in LDS, the bin that holds the n-th largest by a scan from the top, that bin's scores ranked one per lane.
// Returns false, with nothing written, where the bins cannot rank: a range that is empty or not finite, a NaN (also past
// C: x repeats the last score there), or more than 64 scores in that bin.  lds: 256 uint32.  Against the counting search (reg_topk_emit), whose every threshold
// costs a count over all the scores: 4096 rows of 2045 candidates 17.4 us and 25, 1344 rows of 508 6.6 and 12.
template <int R>
__device__ __forceinline__ bool bin_topk_emit(const float (&x)[R], int C, int n, int cand_lo,
                                              int16_t* out, uint32_t* lds) {
  const int lane = threadIdx.x & 63;
  float hi = -INFINITY, lo = INFINITY;
  bool odd = false;
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const bool in = 64 * i + lane < C;
    odd |= x[i] != x[i];
    hi = in ? fmaxf(hi, x[i]) : hi;
    lo = in ? fminf(lo, x[i]) : lo;
  }
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    hi = fmaxf(hi, __shfl_xor(hi, d, 64));
    lo = fminf(lo, __shfl_xor(lo, d, 64));
  }
  const float scale = 256.f / (hi - lo);
  if (__ballot(odd) != 0ull || !(hi > lo) || !(hi < INFINITY) || !(lo > -INFINITY) || !(scale < INFINITY)) return false;
  auto bin = [&](float v) { return min((int)((v - lo) * scale), 255); };
  *reinterpret_cast<uint4*>(&lds[4 * lane]) = make_uint4(0u, 0u, 0u, 0u);
  wave_lds_sync();
#pragma unroll
  for (int i = 0; i < R; ++i)
    if (64 * i + lane < C) atomicAdd(&lds[255 - bin(x[i])], 1u);  // slot 0: the highest bin
  wave_lds_sync();
  const uint4 c = *reinterpret_cast<const uint4*>(&lds[4 * lane]);
  const int mine = (int)(c.x + c.y + c.z + c.w), incl = wave_incl_scan_dpp(mine);
  const int at = (int)__builtin_ctzll(__ballot(incl >= n));  // n < C: there is one
  int above = readlane_i(incl - mine, at), slot = 4 * at;    // scores in the bins before slot
  const int c0 = readlane_i((int)c.x, at), c1 = readlane_i((int)c.y, at), c2 = readlane_i((int)c.z, at), c3 = readlane_i((int)c.w, at);
  int count = c0;
  if (above + count < n) { above += count; count = c1; ++slot; }
  if (above + count < n) { above += count; count = c2; ++slot; }
  if (above + count < n) { above += count; count = c3; ++slot; }
  if (count > 64) return false;
  wave_lds_sync();
  // the bin's scores, one per lane, in index order
  const int tb = 255 - slot;
  int base = 0;
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const bool hit = 64 * i + lane < C && bin(x[i]) == tb;
    const uint64_t b = __ballot(hit);
    if (b == 0ull) continue;
    if (hit) {
      const int z = base + mbcnt64(b);
      lds[z] = __float_as_uint(x[i]);
      lds[64 + z] = (uint32_t)(64 * i + lane);
    }
    base += (int)__popcll(b);
  }
  wave_lds_sync();
  const float k = __uint_as_float(lds[min(lane, count - 1)]);
  const int idx = (int)lds[64 + min(lane, count - 1)];
  int rank = 0;  // scores of the bin that come first: larger, or equal at a lower index (lanes are in index order)
  for (int j = 0; j < count; ++j) {
    const float o = readlane_f(k, j);
    rank += o > k || (o == k && j < lane) ? 1 : 0;
  }
  const int last = (int)__builtin_ctzll(__ballot(lane < count && rank == n - above - 1));
  const float kk = readlane_f(k, last);
  const int ki = readlane_i(idx, last);
  // everything above (kk, ki), in index order
  int done = 0;
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const bool pick = 64 * i + lane < C && (x[i] > kk || (x[i] == kk && 64 * i + lane <= ki));
    const uint64_t b = __ballot(pick);
    if (b == 0ull) continue;
    if (pick) out[done + mbcnt64(b)] = (int16_t)(cand_lo + 64 * i + lane);
    done += (int)__popcll(b);
  }
  return true;
}

// One wavefront per node: forced blocks, padding, count, and the exact top-k over its block scores, in
// registers up to 64 R candidates (R = 0: radix passes over the workspace).
template <int R>
__global__ __launch_bounds__(256, R <= 32 ? 4 : 2) void tree_topk_kernel(TreeSelectArgs a, int64_t n_rows) {
  __shared__ __align__(16) uint32_t lds[4][R == 1 ? 64 : 256];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int64_t row = (int64_t)blockIdx.x * 4 + wave;
  if (row >= n_rows) return;
  const SeqGeom s = seq_geom(a.tb, (int)(row / ((int64_t)a.tb.n * a.n_kv_heads)), lane);
  const int depth = readlane_i(s.depth, (int)(row % a.tb.n));
  int16_t* out = a.sel + row * a.k_total;
  if (depth == 0) {  // an absent node
    for (int i = lane; i < a.k_total; i += kWave) out[i] = (int16_t)-1;
    if (lane == 0) a.cnt[row] = 0;
    return;
  }
  const RowGeom g = row_geom(s.t + depth - 1, a.n_init, a.n_local, a.k_total);
  emit_forced(out, g, a.k_total, lane);
  if (lane == 0) a.cnt[row] = (int16_t)(g.n_forced + g.n_take);
  out += g.init_hi;
  const int C = g.n_cand, n = g.n_take;
  if (n >= C) {
    for (int i = lane; i < C; i += kWave) out[i] = (int16_t)(g.cand_lo + i);
    return;
  }
  if (n <= 0) return;
  const float* sc = a.ws + row * a.ws_stride;
  if constexpr (R == 0) {
    wave_topk_emit([&](int i) { return score_key(sc[i]); }, C, n, g.cand_lo, lds[wave], out);
  } else {
    // slots past the candidates repeat the last; the loads are requested before the first is waited for (the empty
    // asm keeps each out of a branch of its own)
    float x[R];
#pragma unroll
    for (int i = 0; i < R; ++i) x[i] = sc[min(64 * i + lane, C - 1)];
#pragma unroll
    for (int i = 0; i < R; ++i) __asm__ __volatile__("" : "+v"(x[i]));
    if constexpr (R == 1) {
      lane_topk_emit(lane < C ? score_key(x[0]) : 0u, C, n, g.cand_lo, out);
    } else if (!bin_topk_emit<R>(x, C, n, g.cand_lo, out, lds[wave])) {
      uint32_t key[R];  // 0, below every score, past the candidates
#pragma unroll
      for (int i = 0; i < R; ++i) key[i] = 64 * i + lane < C ? score_key(x[i]) : 0u;
      reg_topk_emit<R, true>(key, C, n, g.cand_lo, out, lds[wave]);
    }
  }
}

}  // namespace

hipError_t launch_tree_select(const TreeSelectArgs& a, hipStream_t stream) {
  const int64_t rows = (int64_t)a.tb.batch * a.n_kv_heads * a.tb.n;
  const int C = row_geom(a.tb.t_max + a.tb.n - 1, a.n_init, a.n_local, a.k_total).n_cand;
  if (C > 0) {
    const hipError_t e = grid_is_blocks(a.grid) ? launch_scores<true>(a, C, stream) : launch_scores<false>(a, C, stream);
    if (e != hipSuccess) return e;
  }
  const dim3 grid((unsigned)((rows + 3) / 4)), block(256);
  if (C <= 64)
    hipLaunchKernelGGL(tree_topk_kernel<1>, grid, block, 0, stream, a, rows);
  else if (C <= 128)
    hipLaunchKernelGGL(tree_topk_kernel<2>, grid, block, 0, stream, a, rows);
  else if (C <= 256)
    hipLaunchKernelGGL(tree_topk_kernel<4>, grid, block, 0, stream, a, rows);
  else if (C <= 512)
    hipLaunchKernelGGL(tree_topk_kernel<8>, grid, block, 0, stream, a, rows);
  else if (C <= 1024)
    hipLaunchKernelGGL(tree_topk_kernel<16>, grid, block, 0, stream, a, rows);
  else if (C <= 2048)
    hipLaunchKernelGGL(tree_topk_kernel<32>, grid, block, 0, stream, a, rows);
  else if (C <= 4096)
    hipLaunchKernelGGL(tree_topk_kernel<64>, grid, block, 0, stream, a, rows);
  else
    hipLaunchKernelGGL(tree_topk_kernel<0>, grid, block, 0, stream, a, rows);
  return hipGetLastError();
}

}  // namespace sparda
