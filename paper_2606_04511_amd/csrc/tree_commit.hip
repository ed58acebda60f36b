// tree_commit.hip -- the accepted path's K and V packed into the caches behind the context, and the
// compressed keys of the windows they complete (paper Alg. 2's append and incremental K~ update, for
// several tokens and layers at once; Sec. 3, Eq. 2).
//
// One workgroup per (layer, batch, group).  Its rows are 256 bytes: 16 lanes move a row of K and the
// same row of V.  A completed window's keys come from the cache up to the context and from the
// drafted rows behind it, so nothing waits for the copies, and the keys of up to two windows are requested
// together with the rows.  The float64 sums run in the order of compress_kernel (compress.hip: rows r + 16 x by one
// thread, then the 16 threads' sums in turn) and have to, for the mean to have the bits of sparda_compress_keys: only for
// keys within 39 binades of each other are they exact and free of any order.
//
// What bounds it: latency (a dependent chain of the path's loads, the rows and the stores) for few groups, the
// memory's rate for scattered rows of 256 bytes for many.
#include "device_util.hpp"
#include "launch.hpp"
#include "tree.hpp"

namespace sparda {

namespace {

template <int L>  // tokens of a window
__global__ __launch_bounds__(256) void tree_commit_kernel(TreeCommitArgs a) {
  __shared__ double part[16][144];
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
  if (cnt == 0) return;
  // ---- windows [w0, w1) that the tokens complete
  const int64_t w0 = a.kc[layer] ? grid_win_vis(a.grid, t - 1) + 1 : 0;
  int64_t w1 = a.kc[layer] ? grid_win_vis(a.grid, t + cnt - 1) + 1 : 0;
  if (w1 > a.nc_cap) w1 = a.nc_cap;
  // row rr of window w: in the cache, or drafted (the path's nodes are in the lanes of every wavefront)
  auto key_row = [&](int64_t w, int rr) {
    const int64_t tok = w * a.grid.s + rr;
    const int node = __shfl(mine, (int)(tok < t ? 0 : tok - t) & 63, 64);
    return tok < t ? k[tok * kPieces + c] : kt[node * kPieces + c];
  };
  constexpr int kRows = L / 16;  // of a window that a thread sums
  uint4 first[kRows];
  if (w0 < w1) {
#pragma unroll
    for (int x = 0; x < kRows; ++x) first[x] = key_row(w0, r + 16 * x);
  }
  for (int i0 = 0; i0 < cnt; i0 += 16) {
    const int i = i0 + r;
    const int node = __shfl(mine, i & 63, 64);
    if (i < cnt) {
      const uint4 x = kt[node * kPieces + c], y = vt[node * kPieces + c];
      k[(t + i) * kPieces + c] = x;
      v[(t + i) * kPieces + c] = y;
    }
  }
  // ---- the windows' means: dims 8 c + e at 9 c + e of a thread's row of partial sums (no bank conflicts)
  for (int64_t w = w0; w < w1; ++w) {
    double acc[8] = {};
#pragma unroll
    for (int x = 0; x < kRows; ++x) {
      const uint4 y = first[x];
      acc[0] += bf16lo(y.x); acc[1] += bf16hi(y.x);
      acc[2] += bf16lo(y.y); acc[3] += bf16hi(y.y);
      acc[4] += bf16lo(y.z); acc[5] += bf16hi(y.z);
      acc[6] += bf16lo(y.w); acc[7] += bf16hi(y.w);
    }
    if (w + 1 < w1) {
#pragma unroll
      for (int x = 0; x < kRows; ++x) first[x] = key_row(w + 1, r + 16 * x);
    }
    __syncthreads();  // the last window's sums have been read
#pragma unroll
    for (int e = 0; e < 8; ++e) part[r][c * 9 + e] = acc[e];
    __syncthreads();
    if (tid < kHeadDim) {
      double sum = 0.0;
#pragma unroll
      for (int g = 0; g < 16; ++g) sum += part[g][(tid >> 3) * 9 + (tid & 7)];
      a.kc[layer][(bm * a.nc_cap + w) * kHeadDim + tid] = f64_to_bf16(sum * (1.0 / L));  // exact: L is a power of 2
    }
  }
}

}  // namespace

hipError_t launch_tree_commit(const TreeCommitArgs& a, hipStream_t stream) {
  const int64_t wgs = (int64_t)a.n_layers * a.batch * a.n_kv_heads;
  if (a.grid.l == 64)
    hipLaunchKernelGGL(tree_commit_kernel<64>, dim3((unsigned)wgs), dim3(256), 0, stream, a);
  else
    hipLaunchKernelGGL(tree_commit_kernel<32>, dim3((unsigned)wgs), dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace sparda
