// tree.hpp -- launchers, sizes and device helpers of the operators over trees of drafted tokens
// (tree_select.hip, tree_attention.hip, tree_verify.hip, tree_commit.hip; private to the library).
//
// A tree has at most 64 nodes, one per lane of a wavefront.  Node 0 is the last sampled token; the
// parent of node i > 0 is a lower node.  A(i), the node and its ancestors, is a 64-bit mask.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "launch.hpp"

namespace sparda {

constexpr int kTreeMaxNodes = 64;

// Where the contexts and the trees of a call's sequences come from.
struct TreeBatch {
  const int32_t* t_ctx;   // [batch]: committed tokens; negative: an absent sequence
  const int32_t* parent;  // [batch][n]
  int32_t batch, n;
  int64_t t_max;          // no sequence is longer
};

struct TreeSelectArgs {
  TreeBatch tb;
  const uint16_t* f;
  const uint16_t* kc;
  int16_t* sel;
  int16_t* cnt;
  float* ws;           // block scores: row stride ws_stride, the first candidate at slot 0
  int64_t ws_stride;
  int32_t n_kv_heads;
  int64_t nc_cap;
  int32_t n_init, n_local, k_total;
  WinGrid grid;
};

struct TreeAttnArgs {
  TreeBatch tb;
  const uint16_t* q;
  const uint16_t* k;
  const uint16_t* v;
  const uint16_t* kt;  // drafted K and V: [batch][n_kv_heads][n][128]
  const uint16_t* vt;
  const int16_t* sel;  // [batch][n_kv_heads][n_sel][k_total]
  const int16_t* cnt;
  uint16_t* o;
  float* ws;           // split partials
  int32_t n_kv_heads, group_size, n_sel, k_total;
  int64_t t_cap;
  float sm_scale;
  int32_t width, n_splits;  // the plan
  uint64_t k_recip;       // ceil(2^36 / k_total)
  uint64_t groups_recip;  // ceil(2^36 / (batch * n_kv_heads))
  uint32_t ns_recip;   // ceil(2^20 / n_splits)
  uint32_t g_recip;    // ceil(2^16 / group_size)
};

struct TreeVerifyArgs {
  const void* p;          // [batch][n][ld]
  const void* q;          // the same, or null
  const int32_t* tokens;  // [batch][n]
  const int32_t* parent;
  const float* u;         // [batch][n]
  int32_t* path;          // [batch][n]
  int32_t* n_path;
  int32_t* next_token;
  void* ws;
  int64_t ld;
  int32_t batch, n, vocab, bf16;
};

// The caches of up to this many layers travel in one launch's arguments.
constexpr int kCommitLayers = 32;

struct TreeCommitArgs {
  const uint16_t* kt[kCommitLayers];  // [batch][n_kv_heads][n][128]
  const uint16_t* vt[kCommitLayers];
  uint16_t* k[kCommitLayers];         // [batch][n_kv_heads][t_cap][128]
  uint16_t* v[kCommitLayers];
  uint16_t* kc[kCommitLayers];        // [batch][n_kv_heads][nc_cap][128], or null
  const int32_t* t_ctx;
  const int32_t* path;
  const int32_t* n_path;
  int32_t* t_new;                     // null: another launch of the call writes it
  int32_t n_layers, batch, n_kv_heads, n;
  int64_t t_cap, nc_cap;
  WinGrid grid;
};

// Floats per row of the selection's workspace: the candidates of the longest context.
inline int64_t tree_select_stride(int64_t t_max, int32_t n, int32_t n_init, int32_t n_local) {
  const int64_t c = (t_max + n - 1) / 64 - n_local - n_init + 1;
  return c > 0 ? (c + 3) & ~(int64_t)3 : 0;
}
inline size_t tree_select_ws(int64_t groups, int64_t t_max, int32_t n, int32_t n_init, int32_t n_local) {
  return (size_t)groups * n * (size_t)tree_select_stride(t_max, n, n_init, n_local) * sizeof(float);
}

// The last compressed key that the selection of a context of t tokens reads: of the windows that overlap a candidate of
// the deepest node there can be, the last one complete within t.  -1: no key is read.  It does not fall as t grows.
__host__ __device__ inline int32_t tree_last_key(const WinGrid& grid, int64_t t, int32_t n, int32_t n_init,
                                                 int32_t n_local, int32_t k_total) {
  const RowGeom g = row_geom(t + n - 1, n_init, n_local, k_total);
  if (g.n_cand <= 0) return -1;
  const int32_t hi = grid_win_hi(grid, g.cand_lo + g.n_cand - 1), vis = grid_win_vis(grid, t - 1);
  return hi < vis ? hi : vis;
}
// The row read for window w: those before the first and past the last are requested too (a step is 64 keys).
__host__ __device__ inline int32_t tree_key_row(int32_t w, int32_t last) {
  const int32_t x = w < last ? w : last;
  return x > 0 ? x : 0;
}

// How an attention call is cut into workgroups, one of which fits a CU.
struct TreeAttnPlan {
  int32_t width;     // columns (node, query head) of a workgroup: 16 or 32, whose wavefronts stream blocks of
                     // their own, or 64, 128 or 256, whose wavefronts share them
  int32_t n_splits;  // of a (batch, group)'s blocks
  size_t ws_bytes;   // partials of the splits
};

// Above 32 columns a narrow tile (32) reads the blocks that its own nodes list, in as many workgroups as there are tiles;
// a wide one reads a block once for all its columns, but its wavefronts wait for each other at every block, also those
// whose nodes do not list it.  Widths between 32 and the narrowest that holds all columns (at most 256) are nowhere more
// than 4 % below the better of the two.  Measured (us), 32 columns against the widest; 32K, 64 blocks per list unless said.
// One list for all nodes: every wavefront works on every block, and the wide form wins once the narrow tiles need a
// second round of the 256 CUs.  16 nodes of 4 heads (2 tiles): 128 groups 52 and 58, 144 groups 90 and 83; 32 nodes (4):
// 64 groups 38 and 50, 80 groups 70 and 58; 64 nodes (8): 32 groups 39 and 51, 48 groups 70 and 63, 128 groups 158 and
// 130; 27 nodes of 8 heads (7): 64 groups 74 and 71; 8 nodes of 16 heads (4): 64 groups 38 and 50, 128 groups 84 and 77;
// 64 nodes of 16 heads (32): 16 groups 72 and 69, 64 groups 276 and 199.
// A list per node: the nodes of a tree list about 3 times a list's blocks between them.  Up to 128 columns the wide form
// wins from about 200 MB on.  27 nodes of 4 heads: 24, 32, 40, 64 and 128 groups 50 and 54, 63 and 62, 83 and 75, 131
// and 101, 250 and 187; 13 nodes: 24, 32 and 128 groups 36 and 37, 45 and 41, 168 and 126; 27 nodes of 2 heads, 32
// groups 51 and 46; 8 nodes of 8 heads, 32 and 64 groups 37 and 39, 68 and 63.  With lists of 16 blocks, 27 nodes of 4
// heads: 96, 128 and 256 groups 67 and 85, 79 and 87, 164 and 143; of 32: 48 and 64 groups 55 and 60, 73 and 71; of 160
// at 64K: 8, 16 and 24 groups 37 and 49, 73 and 70, 121 and 96.  Beyond 128 columns too many wavefronts wait, and the
// narrow form is within 13 % or faster, often by much: 64 nodes of 4 heads: 32, 48, 64 and 128 groups 82 and 109, 155 and 154, 177 and 184,
// 347 and 341; 40 nodes: 48, 64, 96 and 256 groups 101 and 132, 180 and 159, 204 and 295, 534 and 567; 64 nodes of 8
// heads, 64 groups 250 and 290; 64 nodes of 16 heads with 96 blocks at 64K: 8, 16 and 48 groups 60 and 95, 119 and 166,
// 385 and 581.
// With fewer workgroups than CUs the blocks are split over them: at least half a block per wavefront, or three blocks
// per workgroup where the wavefronts share them (one each: 19 -> 24 us for 22 nodes of 3 groups of 4 heads, 55 blocks).
// The second launch reads up to 8 splits at once: beyond 16 the finer split of lists that differ by node costs what it
// saves (7 nodes of 4 groups, 64 blocks: 16 splits 18.9 us, 33 20.1).
inline TreeAttnPlan tree_attn_plan(int64_t groups, int32_t n, int32_t group_size, int32_t k_total, int64_t t_max,
                                   bool one_list) {
  TreeAttnPlan p;
  const int cols = n * group_size;
  const int64_t most_blocks = (t_max + 63) / 64;
  auto at_most = [&](int64_t x) { return most_blocks < x ? most_blocks : x; };
  const int64_t narrow_wgs = groups * ((cols + 31) / 32), bytes = groups * at_most(3 * (int64_t)k_total) * (2 * 64 * 128 * 2);
  const bool share = one_list ? narrow_wgs > 256 : cols <= 128 && bytes >= ((int64_t)192 << 20);
  p.width = cols <= 16 ? 16 : cols <= 32 || !share ? 32 : cols <= 64 ? 64 : cols <= 128 ? 128 : 256;
  const int64_t wgs = groups * ((cols + p.width - 1) / p.width), blocks = at_most(k_total);
  int64_t ns = 256 / wgs;
  int64_t most = p.width <= 32 ? (2 * blocks + 2 + 7) / 8 : (blocks + 1 + 2) / 3;
  if (p.width <= 32 && !one_list && n > 1) {  // about twice the blocks: up to 16 splits for them
    const int64_t twice = (2 * at_most(2 * (int64_t)k_total) + 2 + 7) / 8, some = twice < 16 ? twice : 16;
    most = most > some ? most : some;
  }
  ns = ns < most ? ns : most;
  ns = ns > 64 ? 64 : ns < 1 ? 1 : ns;
  p.n_splits = (int32_t)ns;
  p.ws_bytes = ns == 1 ? 0 : (size_t)groups * cols * (size_t)ns * (128 + 4) * sizeof(float);
  return p;
}
// The workspace covers both kinds of lists.
inline size_t tree_attn_ws(int64_t groups, int32_t n, int32_t group_size, int32_t k_total, int64_t t_max) {
  const size_t a = tree_attn_plan(groups, n, group_size, k_total, t_max, true).ws_bytes;
  const size_t b = tree_attn_plan(groups, n, group_size, k_total, t_max, false).ws_bytes;
  return a > b ? a : b;
}

// Workspace of the verification: per sequence the state that the walk left and the sums of the
// row's pieces.
constexpr int kVerifyPiece = 1024;
inline int32_t tree_verify_pieces(int32_t vocab) {  // a row may begin up to 3 elements past a piece's first
  return (int32_t)(((int64_t)vocab + 3 + kVerifyPiece - 1) / kVerifyPiece);
}
inline size_t tree_verify_ws(int64_t batch, int32_t vocab) {
  return (size_t)batch * (64 * sizeof(double) + 2 * (size_t)tree_verify_pieces(vocab) * sizeof(double) + 64);
}

hipError_t launch_tree_select(const TreeSelectArgs& a, hipStream_t stream);
hipError_t launch_tree_attn(const TreeAttnArgs& a, hipStream_t stream);
hipError_t launch_tree_verify(const TreeVerifyArgs& a, hipStream_t stream);
hipError_t launch_tree_commit(const TreeCommitArgs& a, hipStream_t stream);

// ---- device helpers ------------------------------------------------------------------------------

// A(lane) of a tree of n nodes whose parents are at `parent`; 0 for an absent node: one past n, a
// parent that is not a lower node, or an ancestor that is absent.  Pointer doubling: after step x a
// lane's mask covers 2^x nodes of its path and its pointer names the next one, so six steps reach
// the root.  Every lane of the wavefront must call it.
__device__ __forceinline__ uint64_t tree_ancestors(const int32_t* parent, int n, int lane) {
  const int par = lane < n ? parent[lane] : -2;
  int up = lane == 0 ? (par == -1 ? -1 : -2) : (par >= 0 && par < lane ? par : -2);  // -1: past the root
  uint64_t mask = 1ull << lane;
#pragma unroll
  for (int s = 0; s < 6; ++s) {
    const int src = up < 0 ? lane : up;
    const uint32_t lo = (uint32_t)__shfl((int)(uint32_t)mask, src, 64);
    const uint32_t hi = (uint32_t)__shfl((int)(uint32_t)(mask >> 32), src, 64);
    const int next = __shfl(up, src, 64);
    if (up >= 0) {
      mask |= ((uint64_t)hi << 32) | lo;
      up = next;
    }
  }
  return up == -1 ? mask : 0ull;
}

// Committed tokens of sequence b: -1 for an absent one.
__device__ __forceinline__ int64_t tree_context(const TreeBatch& tb, int b) {
  const int64_t t = tb.t_ctx[b];
  return t < 0 ? -1 : (t > tb.t_max ? tb.t_max : t);
}

}  // namespace sparda
