// tree_commit.hip -- the accepted path's K and V packed into the caches behind the context, and the
// compressed keys of the windows they complete (paper Alg. 2's append and incremental K~ update, for
// several tokens and layers at once; Sec. 3, Eq. 2).
//
// One workgroup per (layer, batch, group).  Its rows are 256 bytes: 16 lanes move a row of K and the
// same row of V.  A completed window's keys come from the cache up to the context and from the
// drafted rows behind it, so nothing waits for the copies; float64 sums of at most 64 bf16 keys are
// exact, so the mean has the bits of sparda_compress_keys.
#include "device_util.hpp"
#include "launch.hpp"
#include "tree.hpp"

namespace sparda {

namespace {

__global__ __launch_bounds__(256) void tree_commit_kernel(TreeCommitArgs a) {
  const int tid = threadIdx.x, lane = tid & 63;
  const int groups = a.batch * a.n_kv_heads;
  const int layer = blockIdx.x / groups;
  const int64_t bm = blockIdx.x % groups;
  const int b = (int)(bm / a.n_kv_heads);
  const int64_t t = a.t_ctx[b];
  // entries up to the first one that names no node or lies past the cache
  const int listed = a.n_path[b];
  const int mine = lane < a.n ? a.path[(int64_t)b * a.n + lane] : -1;
  const bool good = t >= 0 && lane < a.n && lane < listed && mine >= 0 && mine < a.n && t + lane < a.t_cap;
  const uint64_t bad = ~__ballot(good);
  const int cnt = bad ? (int)__builtin_ctzll(bad) : 64;
  if (a.t_new && layer == 0 && bm % a.n_kv_heads == 0 && tid == 0) a.t_new[b] = (int32_t)(t + cnt);
  constexpr int kPieces = kHeadDim * 2 / 16;
  const int c = tid % kPieces, r = tid / kPieces;
  const uint4* kt = reinterpret_cast<const uint4*>(a.kt[layer] + bm * a.n * kHeadDim);
  const uint4* vt = reinterpret_cast<const uint4*>(a.vt[layer] + bm * a.n * kHeadDim);
  uint4* k = reinterpret_cast<uint4*>(a.k[layer] + bm * a.t_cap * kHeadDim);
  uint4* v = reinterpret_cast<uint4*>(a.v[layer] + bm * a.t_cap * kHeadDim);
  for (int i0 = 0; i0 < cnt; i0 += 16) {
    const int i = i0 + r;
    const int node = __shfl(mine, i & 63, 64);
    if (i < cnt) {
      const uint4 x = kt[node * kPieces + c], y = vt[node * kPieces + c];
      k[(t + i) * kPieces + c] = x;
      v[(t + i) * kPieces + c] = y;
    }
  }
  if (a.kc[layer] == nullptr || cnt == 0) return;
  const int64_t w0 = grid_win_vis(a.grid, t - 1) + 1;
  int64_t w1 = grid_win_vis(a.grid, t + cnt - 1) + 1;
  if (w1 > a.nc_cap) w1 = a.nc_cap;
  const uint16_t* keys = a.k[layer] + bm * a.t_cap * kHeadDim;
  const uint16_t* drafted = a.kt[layer] + bm * a.n * kHeadDim;
  for (int64_t w = w0 + (tid >> 7); w < w1; w += 2) {
    double sum = 0.0;
    for (int x = 0; x < a.grid.l; ++x) {
      const int64_t tok = w * a.grid.s + x;
      const uint16_t* row = tok < t ? keys + tok * kHeadDim
                                    : drafted + (int64_t)a.path[(int64_t)b * a.n + (tok - t)] * kHeadDim;
      sum += (double)bf16_to_f32(row[tid & 127]);
    }
    a.kc[layer][(bm * a.nc_cap + w) * kHeadDim + (tid & 127)] = f64_to_bf16(sum / a.grid.l);
  }
}

}  // namespace

hipError_t launch_tree_commit(const TreeCommitArgs& a, hipStream_t stream) {
  const int64_t wgs = (int64_t)a.n_layers * a.batch * a.n_kv_heads;
  hipLaunchKernelGGL(tree_commit_kernel, dim3((unsigned)wgs), dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace sparda
