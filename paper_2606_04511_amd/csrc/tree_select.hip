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

// Block scores of one node, 16 candidates per workgroup: 16 lanes per candidate, 8 dims each.
__global__ __launch_bounds__(256) void tree_score_kernel(TreeSelectArgs a) {
  const int64_t row = blockIdx.x;
  const int i = (int)(row % a.tb.n);
  const int64_t bm = row / a.tb.n;
  const int b = (int)(bm / a.n_kv_heads);
  const int lane = threadIdx.x & 63;
  const SeqGeom s = seq_geom(a.tb, b, lane);
  const int depth = readlane_i(s.depth, i);
  if (depth == 0) return;
  const RowGeom g = row_geom(s.t + depth - 1, a.n_init, a.n_local, a.k_total);
  if (g.n_take >= g.n_cand) return;
  const int32_t vis = grid_win_vis(a.grid, s.t - 1);
  const int c = threadIdx.x & 15;
  const int x = blockIdx.y * 16 + (threadIdx.x >> 4);
  if (x >= g.n_cand) return;
  const uint4 fw = ld16(a.f + row * kHeadDim + c * 8);
  const float fv[8] = {bf16lo(fw.x), bf16hi(fw.x), bf16lo(fw.y), bf16hi(fw.y),
                       bf16lo(fw.z), bf16hi(fw.z), bf16lo(fw.w), bf16hi(fw.w)};
  const int lo = grid_win_lo(a.grid, g.cand_lo + x), hi = min(grid_win_hi(a.grid, g.cand_lo + x), vis);
  float best = -INFINITY;
  for (int w = lo; w <= hi; ++w) {
    const uint4 kw = ld16(a.kc + (bm * a.nc_cap + w) * kHeadDim + c * 8);
    const float kv[8] = {bf16lo(kw.x), bf16hi(kw.x), bf16lo(kw.y), bf16hi(kw.y),
                         bf16lo(kw.z), bf16hi(kw.z), bf16lo(kw.w), bf16hi(kw.w)};
    float d = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) d = fmaf(fv[e], kv[e], d);
    best = fmaxf(best, row16_sum(d));
  }
  if (c == 0) a.ws[row * a.ws_stride + x] = best;
}

// One wavefront per node: forced blocks, padding, count, and the exact top-k over its block scores, in
// registers up to 64 R candidates (R = 0: radix passes over the workspace).
template <int R>
__global__ __launch_bounds__(256) void tree_topk_kernel(TreeSelectArgs a, int64_t n_rows) {
  __shared__ __align__(16) uint32_t lds[4][R == 0 ? 256 : 64];
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
    // slots past the candidates: key 0, below every score; the loads are requested before the first is
    // waited for (the empty asm keeps each out of a branch of its own)
    uint32_t key[R];
    constexpr int kBatch = R < 16 ? R : 16;
#pragma unroll
    for (int i0 = 0; i0 < R; i0 += kBatch) {
      float x[kBatch];
#pragma unroll
      for (int i = 0; i < kBatch; ++i) x[i] = sc[min(64 * (i0 + i) + lane, C - 1)];
#pragma unroll
      for (int i = 0; i < kBatch; ++i) {
        __asm__ __volatile__("" : "+v"(x[i]));
        key[i0 + i] = 64 * (i0 + i) + lane < C ? score_key(x[i]) : 0u;
      }
    }
    if constexpr (R == 1)
      lane_topk_emit(key[0], C, n, g.cand_lo, out);
    else
      reg_topk_emit<R, true>(key, C, n, g.cand_lo, out, lds[wave]);
  }
}

}  // namespace

hipError_t launch_tree_select(const TreeSelectArgs& a, hipStream_t stream) {
  const int64_t rows = (int64_t)a.tb.batch * a.n_kv_heads * a.tb.n;
  const int C = row_geom(a.tb.t_max + a.tb.n - 1, a.n_init, a.n_local, a.k_total).n_cand;
  if (C > 0) {
    hipLaunchKernelGGL(tree_score_kernel, dim3((unsigned)rows, (unsigned)((C + 15) / 16)), dim3(256), 0, stream, a);
    const hipError_t e = hipGetLastError();
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
