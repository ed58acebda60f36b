// paged_select.hip -- the attended block set of every sequence's newest token (paper Sec. 4.1, Eq. 4 with Eq. 1), for
// sequences of different lengths whose compressed keys lie in pages.
//
// A row (sequence, KV head) is at p = t - 1.  Its windows score F . K~_w (float32 accumulation) where they are complete
// within the t tokens; a block's score is the largest of the windows that overlap it.  The scores go to the workspace,
// then one wavefront per row selects.
#include "device_util.hpp"
#include "launch.hpp"
#include "paged.hpp"
#include "select_block.hpp"

namespace sparda {

namespace {

__device__ __forceinline__ int64_t paged_context(const int32_t* t_ctx, int b, int64_t t_max) {
  const int64_t t = t_ctx[b];
  return t > t_max ? t_max : t;
}

// Scores of 64 windows per step and wavefront: 64 blocks on the one-key-per-block grid, 16 blocks of the (32, 16) grid.
// Sixteen lanes read a key of 256 bytes, so a load instruction brings four; the lane of key 4 c + z that keeps its score
// is lane c of the z-th sixteen.  On the (32, 16) grid z is the window within block c, so a block's four scores meet
// across the sixteens; its fifth, window -1, is window 3 of the block before: the neighbouring lane's, or for the first
// block the last step's (at a wavefront's first step one more key).
template <bool kBlocks>
__global__ __launch_bounds__(256) void paged_score_kernel(PagedSelectArgs a, int n_rows, int steps) {
  constexpr int kPerStep = kBlocks ? 64 : 16, kLog = kBlocks ? 6 : 4;
  const int lane = threadIdx.x & 63, c = lane & 15, z = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row = blockIdx.x % n_rows;
  const int part = (int)(blockIdx.x / n_rows) * 4 + wave;
  const int b = row / a.n_kv_heads, h = row % a.n_kv_heads;
  const int64_t t = paged_context(a.t_ctx, b, a.t_max);
  if (t <= 0) return;
  const RowGeom g = row_geom(t - 1, a.n_init, a.n_local, a.k_total);
  if (g.n_take >= g.n_cand) return;
  const int x_end = min(g.n_cand, (part + 1) * steps * kPerStep);
  int x0 = part * steps * kPerStep;
  if (x0 >= x_end) return;
  const int32_t vis = grid_win_vis(a.grid, t - 1);  // no window past it is read
  const int32_t* table = a.pg.table + b * a.pg.table_ld;
  float f[8];
  {
    const uint4 w = ld16(a.f + (int64_t)row * kHeadDim + 8 * c);
    f[0] = bf16lo(w.x); f[1] = bf16hi(w.x); f[2] = bf16lo(w.y); f[3] = bf16hi(w.y);
    f[4] = bf16lo(w.z); f[5] = bf16hi(w.z); f[6] = bf16lo(w.w); f[7] = bf16hi(w.w);
  }
  auto page_at = [&](int w) {  // of window w, -1: not to be scored
    return w >= 0 && w <= vis ? page_of(a.pg, table, (int64_t)w << kLog) : -1;
  };
  auto load = [&](int w, int page) {
    return ld16_nt(a.pg.kc + key_at(a.pg, page < 0 ? 0 : page, a.n_kv_heads, h, (int64_t)(w < 0 ? 0 : w) << kLog, kLog) + 8 * c);
  };
  auto dot = [&](uint4 k) {
    float s = bf16lo(k.x) * f[0];
    s = fmaf(bf16hi(k.x), f[1], s);
    s = fmaf(bf16lo(k.y), f[2], s);
    s = fmaf(bf16hi(k.y), f[3], s);
    s = fmaf(bf16lo(k.z), f[4], s);
    s = fmaf(bf16hi(k.z), f[5], s);
    s = fmaf(bf16lo(k.w), f[6], s);
    s = fmaf(bf16hi(k.w), f[7], s);
    return row16_sum(s);
  };
  float* const out = a.ws + (int64_t)row * a.ws_stride;
  float carry = -INFINITY;
  if constexpr (!kBlocks) {
    const int w = 4 * (g.cand_lo + x0) - 1, page = page_at(w);
    const float s = dot(load(w, page));
    if (page >= 0) carry = s;
  }
  for (; x0 < x_end; x0 += kPerStep) {
    const int w0 = kBlocks ? g.cand_lo + x0 : 4 * (g.cand_lo + x0);
    const int pages = page_at(w0 + lane);
    uint4 k[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) k[j] = load(w0 + 4 * j + z, __shfl(pages, 4 * j + z, 64));
    float mine = 0.f;
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      const float s = dot(k[j]);
      mine = c == j ? s : mine;
    }
    if (__shfl(pages, 4 * c + z, 64) < 0) mine = -INFINITY;
    if constexpr (kBlocks) {
      const int x = x0 + 4 * c + z;
      if (x < g.n_cand) out[x] = mine;
    } else {
      float best = fmaxf(mine, __shfl_xor(mine, 16, 64));
      best = fmaxf(best, __shfl_xor(best, 32, 64));
      const float last = __shfl(mine, 48 + c, 64);  // window 3 of block c
      const float before = __shfl_up(last, 1, 16);
      best = fmaxf(best, c == 0 ? carry : before);
      carry = __shfl(last, 15, 64);
      if (z == 0 && x0 + c < g.n_cand) out[x0 + c] = best;
    }
  }
}

template <int R>
__global__ __launch_bounds__(256, R <= 32 ? 4 : 2) void paged_topk_kernel(PagedSelectArgs a, int n_rows) {
  __shared__ __align__(16) uint32_t lds[4][R == 1 ? 64 : 256];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int row = (int)blockIdx.x * 4 + wave;
  if (row >= n_rows) return;
  const int64_t t = paged_context(a.t_ctx, row / a.n_kv_heads, a.t_max);
  int16_t* out = a.sel + (int64_t)row * a.k_total;
  if (t <= 0) {
    for (int i = lane; i < a.k_total; i += kWave) out[i] = (int16_t)-1;
    if (lane == 0) a.cnt[row] = 0;
    return;
  }
  const RowGeom g = row_geom(t - 1, a.n_init, a.n_local, a.k_total);
  emit_forced(out, g, a.k_total, lane);
  if (lane == 0) a.cnt[row] = (int16_t)(g.n_forced + g.n_take);
  out += g.init_hi;
  const int C = g.n_cand, n = g.n_take;
  if (n >= C) {
    for (int i = lane; i < C; i += kWave) out[i] = (int16_t)(g.cand_lo + i);
    return;
  }
  if (n <= 0) return;
  scores_topk_emit<R>(a.ws + (int64_t)row * a.ws_stride, C, n, g.cand_lo, out, lds[wave]);
}

}  // namespace

hipError_t launch_paged_select(const PagedSelectArgs& a, hipStream_t stream) {
  const int rows = a.batch * a.n_kv_heads;
  const RowGeom g = row_geom(a.t_max - 1, a.n_init, a.n_local, a.k_total);
  const int C = g.n_cand;
  const bool blocks = grid_is_blocks(a.grid);
  if (C > g.n_take) {  // shorter contexts take every candidate where the longest does
    const int total = (C + (blocks ? 63 : 15)) / (blocks ? 64 : 16);
    // steps per wavefront: one while the chip is not full, else about two wavefronts per SIMD; at most 16
    const int64_t all = (int64_t)rows * total;
    const int steps = (int)(all <= 2048 ? 1 : all >= 16 * 2048 ? 16 : all / 2048);
    const int parts = (total + steps - 1) / steps;
    const dim3 grid((unsigned)(rows * ((parts + 3) / 4))), block(256);
    if (blocks)
      hipLaunchKernelGGL(paged_score_kernel<true>, grid, block, 0, stream, a, rows, steps);
    else
      hipLaunchKernelGGL(paged_score_kernel<false>, grid, block, 0, stream, a, rows, steps);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  const dim3 grid((unsigned)((rows + 3) / 4)), block(256);
  if (C <= 64)
    hipLaunchKernelGGL(paged_topk_kernel<1>, grid, block, 0, stream, a, rows);
  else if (C <= 256)
    hipLaunchKernelGGL(paged_topk_kernel<4>, grid, block, 0, stream, a, rows);
  else if (C <= 512)
    hipLaunchKernelGGL(paged_topk_kernel<8>, grid, block, 0, stream, a, rows);
  else if (C <= 1024)
    hipLaunchKernelGGL(paged_topk_kernel<16>, grid, block, 0, stream, a, rows);
  else if (C <= 2048)
    hipLaunchKernelGGL(paged_topk_kernel<32>, grid, block, 0, stream, a, rows);
  else if (C <= 4096)
    hipLaunchKernelGGL(paged_topk_kernel<64>, grid, block, 0, stream, a, rows);
  else
    hipLaunchKernelGGL(paged_topk_kernel<0>, grid, block, 0, stream, a, rows);
  return hipGetLastError();
}

}  // namespace sparda
