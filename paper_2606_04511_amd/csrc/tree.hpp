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
  int32_t n_splits;
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

// Splits of a (batch, group)'s blocks and the bytes of their partials.
struct TreeAttnPlan {
  int32_t n_splits;
  size_t ws_bytes;
};
// Columns (node, query head) that one workgroup takes.
inline int tree_attn_cols(int32_t n, int32_t group_size) {
  const int cols = n * group_size;
  return cols <= 16 ? 16 : cols <= 32 ? 32 : cols <= 64 ? 64 : cols <= 128 ? 128 : 256;
}
// With fewer workgroups than CUs (one fits a CU) the blocks are split over them, at least half a block
// per wavefront each.
inline TreeAttnPlan tree_attn_plan(int64_t groups, int32_t n, int32_t group_size, int32_t k_total, int64_t t_max) {
  const int cols = n * group_size, width = tree_attn_cols(n, group_size);
  const int64_t wgs = groups * ((cols + width - 1) / width);
  const int64_t blocks = (t_max + 63) / 64 < k_total ? (t_max + 63) / 64 : k_total;
  int64_t ns = 1;
  if (wgs < 256) {
    const int64_t want = (256 + wgs - 1) / wgs, most = (2 * blocks + 2 + 7) / 8;
    ns = want < most ? want : most;
    if (ns > 64) ns = 64;
  }
  const size_t bytes = ns == 1 ? 0 : (size_t)groups * cols * (size_t)ns * (128 + 4) * sizeof(float);
  return {(int32_t)ns, bytes};
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
