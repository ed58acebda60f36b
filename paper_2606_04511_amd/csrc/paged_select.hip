// paged_select.hip -- the attended block set of every sequence's newest token (paper Sec. 4.1, Eq. 4 with Eq. 1), for
// sequences of different lengths whose compressed keys lie in pages.
//
// A row (sequence, KV head) is at p = t - 1.  Its windows score F . K~_w (float32 accumulation) where they are complete
// within the t tokens; a block's score is the largest of the windows that overlap it.  A workgroup per row selects, and
// forms the scores itself where that is faster (launch has the choice); elsewhere a launch before it does.
//
// What bounds it: the memory's rate for many rows (256 rows of 128K: 126 MB in 24 us, of which the top-k is about 5);
// below, the chain length -> pages -> keys -> top-k, 5.3 us for a row of 4K.
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

// A row's scores.  A step is 64 windows of one wavefront: 64 blocks on the one-key-per-block grid, 16 blocks of the (32, 16)
// grid.  Sixteen lanes read a key of 256 bytes, so a load instruction brings four; lane (z, c) keeps the score of key
// 4 c + z.  On the (32, 16) grid z is the window within block c, so a block's four scores meet across the sixteens; its
// fifth, window -1, is window 3 of the block before: the neighbouring lane's, or for the first block the last step's (at a
// wavefront's first step one more key).  A key of the next step is requested when its register is free, so sixteen are
// under way at all times; pages are looked up two steps ahead.  put(x, score) takes the score of candidate x, on some lanes of the wavefront.
template <bool kBlocks>
struct RowScores {
  static constexpr int kPerStep = kBlocks ? 64 : 16, kLog = kBlocks ? 6 : 4;
  const PagedSelectArgs& a;
  const RowGeom g;
  const int32_t* table;
  int h, lane, c, z;
  int32_t vis;  // no window past it is read
  float f[8];

  __device__ RowScores(const PagedSelectArgs& args, const RowGeom& geom, int row, int64_t t)
      : a(args), g(geom), table(args.pg.table + (int64_t)(row / args.n_kv_heads) * args.pg.table_ld),
        h(row % args.n_kv_heads), lane(threadIdx.x & 63), c(lane & 15), z(lane >> 4), vis(grid_win_vis(args.grid, t - 1)) {
    const uint4 w = ld16(a.f + (int64_t)row * kHeadDim + 8 * c);
    f[0] = bf16lo(w.x); f[1] = bf16hi(w.x); f[2] = bf16lo(w.y); f[3] = bf16hi(w.y);
    f[4] = bf16lo(w.z); f[5] = bf16hi(w.z); f[6] = bf16lo(w.w); f[7] = bf16hi(w.w);
  }
  __device__ int first_window(int x) const { return kBlocks ? g.cand_lo + x : 4 * (g.cand_lo + x); }
  // Window w's key as a row of the pool (a pool of 2^32 rows would be 1 TB), kNone: not to be scored.
  static constexpr uint32_t kNone = 0xffffffffu;
  __device__ uint32_t row_at(int w) const {
    const int page = w >= 0 && w <= vis ? page_of(a.pg, table, (int64_t)w << kLog) : -1;
    return page < 0 ? kNone : (uint32_t)(key_at(a.pg, page, a.n_kv_heads, h, (int64_t)w << kLog, kLog) >> 7);
  }
  __device__ uint4 load(uint32_t row) const {
    return ld16_nt(a.pg.kc + (uint64_t)(row == kNone ? 0u : row) * kHeadDim + 8 * c);
  }
  __device__ float dot(uint4 k) const {
    float s = bf16lo(k.x) * f[0];
    s = fmaf(bf16hi(k.x), f[1], s);
    s = fmaf(bf16lo(k.y), f[2], s);
    s = fmaf(bf16hi(k.y), f[3], s);
    s = fmaf(bf16lo(k.z), f[4], s);
    s = fmaf(bf16hi(k.z), f[5], s);
    s = fmaf(bf16lo(k.w), f[6], s);
    s = fmaf(bf16hi(k.w), f[7], s);
    return row16_sum(s);
  }
  // The score of key 4 c + z of the step at x; candidates before x1.
  template <class Put>
  __device__ void finish(float mine, int x, int x1, uint32_t rows, float& carry, Put& put) const {
    if (!(__ballot(rows != kNone) >> (4 * c + z) & 1ull)) mine = -INFINITY;
    if constexpr (kBlocks) {
      if (x + 4 * c + z < x1) put(x + 4 * c + z, mine);
    } else {
      float best = fmaxf(mine, __shfl_xor(mine, 16, 64));
      best = fmaxf(best, __shfl_xor(best, 32, 64));
      const float last = __shfl(mine, 48 + c, 64);  // window 3 of block c
      const float before = __shfl_up(last, 1, 16);
      best = fmaxf(best, c == 0 ? carry : before);
      carry = __shfl(last, 15, 64);
      if (z == 0 && x + c < x1) put(x + c, best);
    }
  }
  // Candidates [x, x1), x1 > x.
  template <class Put>
  __device__ void run(int x, int x1, Put put) const {
    uint4 k[16];
    uint32_t here = row_at(first_window(x) + lane), next = row_at(first_window(x + kPerStep) + lane);
    auto request = [&](int j, uint32_t rows) { k[j] = load((uint32_t)__shfl((int)rows, 4 * j + z, 64)); };
    float carry = -INFINITY, mine = 0.f;
    auto products = [&](int j) {
      const float s = dot(k[j]);
      mine = c == j ? s : mine;
    };
    uint4 edge = make_uint4(0u, 0u, 0u, 0u);
    uint32_t edge_row = kNone;
    if constexpr (!kBlocks) {
      edge_row = row_at(first_window(x) - 1);
      edge = load(edge_row);
    }
#pragma unroll
    for (int j = 0; j < 16; ++j) request(j, here);
    if constexpr (!kBlocks) {
      const float s = dot(edge);
      if (edge_row != kNone) carry = s;
    }
    for (; x + kPerStep < x1; x += kPerStep) {  // a register's next key is requested as soon as it is free
      const uint32_t behind = row_at(first_window(x + 2 * kPerStep) + lane);
#pragma unroll
      for (int j = 0; j < 16; j += 4) {
#pragma unroll
        for (int e = 0; e < 4; ++e) products(j + e);
#pragma unroll
        for (int e = 0; e < 4; ++e) request(j + e, next);
        __builtin_amdgcn_sched_barrier(0);
      }
      finish(mine, x, x1, here, carry, put);
      here = next;
      next = behind;
    }
#pragma unroll
    for (int j = 0; j < 16; ++j) products(j);
    finish(mine, x, x1, here, carry, put);
  }
};

// The scores of all rows to the workspace.
template <bool kBlocks>
__global__ __launch_bounds__(256) void paged_score_kernel(PagedSelectArgs a, int n_rows, int steps) {
  constexpr int kPerStep = RowScores<kBlocks>::kPerStep;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row = blockIdx.x % n_rows;
  const int part = (int)(blockIdx.x / n_rows) * 4 + wave;
  const int64_t t = paged_context(a.t_ctx, row / a.n_kv_heads, a.t_max);
  if (t <= 0) return;
  const RowGeom g = row_geom(t - 1, a.n_init, a.n_local, a.k_total);
  if (g.n_take >= g.n_cand) return;
  const int x0 = part * steps * kPerStep, x1 = min(g.n_cand, x0 + steps * kPerStep);
  if (x0 >= x1) return;
  float* const out = a.ws + (int64_t)row * a.ws_stride;
  RowScores<kBlocks>(a, g, row, t).run(x0, x1, [&](int x, float s) { out[x] = s; });
}

// A row's set by one workgroup of kDecThreads.  kScores: it forms the scores itself, in LDS; otherwise they are in the
// workspace, and come to LDS where `lds` holds as many floats.
template <bool kBlocks, bool kScores>
__global__ __launch_bounds__(kDecThreads) void paged_row_kernel(PagedSelectArgs a, int lds) {
  extern __shared__ __align__(16) float scores[];
  __shared__ __align__(16) uint32_t hist[kTopkLds];
  __shared__ int wave_cnt[kDecThreads / 64], pick[3];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int row = blockIdx.x;
  const int64_t t = paged_context(a.t_ctx, row / a.n_kv_heads, a.t_max);
  int16_t* out = a.sel + (int64_t)row * a.k_total;
  if (t <= 0) {
    for (int i = tid; i < a.k_total; i += kDecThreads) out[i] = (int16_t)-1;
    if (tid == 0) a.cnt[row] = 0;
    return;
  }
  const RowGeom g = row_geom(t - 1, a.n_init, a.n_local, a.k_total);
  const int C = g.n_cand, n = g.n_take;
  uint32_t kmin = 0xffffffffu, kmax = 0u;
  auto keep = [&](int x, float s) {
    scores[x] = s;
    const uint32_t key = score_key(s);
    kmin = min(kmin, key);
    kmax = max(kmax, key);
  };
  const bool ranked = n > 0 && n < C, staged = kScores || C <= lds;
  if (ranked && staged) {
    topk_clear(hist);
    if constexpr (kScores) {
      constexpr int kPerStep = RowScores<kBlocks>::kPerStep, kWaves = kDecThreads / 64;
      const int each = ((C + kPerStep - 1) / kPerStep + kWaves - 1) / kWaves;
      const int x0 = wave * each * kPerStep, x1 = min(C, x0 + each * kPerStep);
      if (x0 < x1) RowScores<kBlocks>(a, g, row, t).run(x0, x1, keep);
    } else {
      const float* src = a.ws + (int64_t)row * a.ws_stride;
      for (int x0 = 0; x0 < C; x0 += 8 * kDecThreads) {  // eight loads under way
        float s[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) s[e] = src[min(x0 + e * kDecThreads + tid, C - 1)];
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (x0 + e * kDecThreads + tid < C) keep(x0 + e * kDecThreads + tid, s[e]);
      }
    }
    topk_publish_extremes(kmin, kmax, hist);
  }
  if (wave == kDecThreads / 64 - 1) emit_forced(out, g, a.k_total, lane);  // (the last wavefront has the fewest scores)
  if (tid == 0) a.cnt[row] = (int16_t)(g.n_forced + n);
  out += g.init_hi;
  if (!ranked) {
    for (int i = tid; i < n; i += kDecThreads) out[i] = (int16_t)(g.cand_lo + i);
    return;
  }
  __syncthreads();
  block_topk_emit(staged ? scores : a.ws + (int64_t)row * a.ws_stride, C, n, g.cand_lo, out, hist, wave_cnt, pick, staged);
}

template <bool kBlocks>
hipError_t launch(const PagedSelectArgs& a, hipStream_t stream) {
  constexpr int kPerStep = RowScores<kBlocks>::kPerStep;
  const int rows = a.batch * a.n_kv_heads;
  const RowGeom g = row_geom(a.t_max - 1, a.n_init, a.n_local, a.k_total);
  const int C = g.n_cand, total = (C + kPerStep - 1) / kPerStep;
  // One launch, whose workgroup reads a row's keys alone (a CU brings about 50 GB/s), or the scores by as many wavefronts as
  // fill the chip and a second launch.  Measured in graphs (us, one launch and two), a key per block: 1 row of 4K 5.3 and
  // 6.9, of 64K 8.7 and 8.7, of 128K 13.1 and 8.7; 64 rows of 128K 13.9 and 10.6; 128 rows of 128K 18.1 and 16.6; 192 rows
  // 22.4 and 25.5; 256 rows 26.0 and 29.8.  (32, 16): 1 row of 4K 6.2 and 7.5, of 12K 9.1 and 9.0, of 32K 15.6 and 9.0; 128
  // rows of 64K 33 and 28; 192 rows 37 and 42; 256 rows 46 and 52.
  const bool one = C <= 8192 && (total <= (kBlocks ? 16 : 12) || rows >= 192);
  // (shorter contexts take every candidate where the longest does; a budget of the forced blocks alone takes none of any)
  if (one || C <= g.n_take || g.n_take == 0) {
    const size_t lds = (size_t)(C > 64 ? C : 64) * sizeof(float);
    hipLaunchKernelGGL((paged_row_kernel<kBlocks, true>), dim3((unsigned)rows), dim3(kDecThreads), one ? lds : 256, stream, a, 0);
    return hipGetLastError();
  }
  // steps per wavefront: one while the chip is not full, else about two wavefronts per SIMD; at most 16
  const int64_t all = (int64_t)rows * total;
  const int steps = (int)(all <= 2048 ? 1 : all >= 16 * 2048 ? 16 : all / 2048);
  const int parts = (total + steps - 1) / steps;
  hipLaunchKernelGGL(paged_score_kernel<kBlocks>, dim3((unsigned)(rows * ((parts + 3) / 4))), dim3(256), 0, stream, a, rows, steps);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int lds = C <= 16384 ? C : 0;  // (64 KiB)
  hipLaunchKernelGGL((paged_row_kernel<kBlocks, false>), dim3((unsigned)rows), dim3(kDecThreads), (size_t)lds * sizeof(float), stream,
                     a, lds);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_select(const PagedSelectArgs& a, hipStream_t stream) {
  return grid_is_blocks(a.grid) ? launch<true>(a, stream) : launch<false>(a, stream);
}

}  // namespace sparda
