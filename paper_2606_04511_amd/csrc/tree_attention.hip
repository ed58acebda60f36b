// tree_attention.hip -- attention of the nodes of drafted-token trees over their blocks of the cache
// and their ancestors (paper Sec. 4.1, Eq. 5 over the set of Eq. 1):
//   o_i = softmax(sm_scale q_i K^T) V over {t' < t in the blocks of node i} U A(i).
//
// Work unit: a tile of columns (column c is query head c % G of node c / G) of one (batch, group), and a
// split of the blocks that any of the tile's nodes lists, on one workgroup of 8 wavefronts.  One pass over
// K and V serves all columns of the tile, with the running maximum and sum of the softmax in registers.
//   1. The lists of the tile's nodes become a table in LDS, one 64-bit mask of nodes per block (entries
//      outside the context are dropped, a repeated one sets its bit again), and the blocks with a mask
//      an ascending list.  Split s takes every n_splits-th of them.  The drafted tokens are one more
//      entry.  Contexts of more than 2048 blocks are walked in windows of 2048.
//   2. K and V go from memory straight into LDS.  Up to 32 columns (tree_attn_kernel) each wavefront takes
//      halves of blocks (32 tokens, 8 KiB of K and of V) in turn into two buffers of its own, the next
//      half's K in flight from the moment the products of this one have read K, its V from the moment O
//      has read V; it waits for its own loads by count, and no barrier joins the wavefronts until the
//      merge.  64 to 256 columns (tree_attn_shared_kernel): a ring of four blocks for all wavefronts, each
//      of which has 16 or 32 columns; one barrier per block.  tree_attn_plan chooses, with figures.
//   3. Per half and 16 columns: S^T = K Q^T on v_mfma_f32_16x16x32_bf16 (lane (c, g) holds column c's
//      scores of tokens 16 tt + 4 g + i); masks; P = 2^(z - m) with a reference m that moves only when a
//      score exceeds it by more than 2^8; O^T += V^T P^T on the same MFMA, V read through the transposing
//      LDS read.  P enters the product as two bf16 numbers, itself rounded and what that rounding took, so
//      a weight is off by at most 2^-16 of itself; the denominators sum it in float32.  With the rounded
//      one alone (2^-8) the products take half the instructions (27 nodes of 64 groups below: 88 us instead
//      of 99; 16 nodes of 256 groups 90 and 92-95), but a step over a tree would be less exact than the
//      decode steps it stands for.
//   4. The wavefronts' states merge through LDS; with splits their float32 partials go to the workspace
//      and a second launch merges them.
//
// What bounds it.  16 nodes of 256 groups of 4 heads at 128K, 64 blocks (537 MB): 92 us, 5.9 TB/s, the memory's rate
// with prologue and merge.  27 nodes of 64 groups with lists of their own at 32K (400 MB): 99 us, of which 9 before the
// first product, 3 after the last; each of the 48 blocks of a workgroup takes 1.8 us, three blocks' loads in flight.
// 64 nodes of 16 groups of 16 heads at 64K (168 MB, 51 GFLOP): 124 us, a block read from L2 once per two nodes
// (256 columns per workgroup: 166, the wavefronts waiting for the one whose nodes list the block).  8 nodes at 4K: 14 us,
// of which 4 merge the splits, a chain of latencies.
#include <math.h>

#include "device_util.hpp"
#include "launch.hpp"
#include "tree.hpp"

namespace sparda {

namespace {

constexpr float kLog2eT = 1.4426950408889634f;
constexpr float kHeadroom = 8.f;                     // log2 by which a score may exceed its column's reference
constexpr int kTaWaves = 8;
constexpr int kTaThreads = 64 * kTaWaves;
constexpr int kTaHalf = 32;                          // tokens per half block
constexpr int kTaBuf = kTaHalf * kHeadDim * 2;       // bytes of a half's K or V
constexpr int kTaSlot = 4 * kTaBuf;                  // bytes of a block's K, then its V
constexpr int kTaRing = 4;                           // blocks in LDS at once (shared form)
constexpr int kTaWindow = 2048;                      // blocks per window of the table
constexpr int kTaTree = 0x7fff;                      // the list's entry of the drafted tokens (others: 0 .. 2047)
constexpr int kTaTreeBlock = 0x10000;                // as a block's number, past every block's: from here on
constexpr int kTaPitch = kHeadDim + 4;               // floats per merged row: 16 rows of 16 bytes touch every bank once
constexpr int kTaPartial = kHeadDim + 4;             // floats of a split's partial: m, l, two unused, the sums
constexpr int kCombineThreads = 256;

struct TreeAttnLds {
  char kv[kTaRing * kTaSlot];
  uint64_t table[kTaWindow];
  int16_t list[kTaWindow + 1];
  int count[kTaWaves];
};
static_assert(sizeof(TreeAttnLds) <= 160 * 1024, "LDS of one CU");
static_assert(sizeof(float) * kTaWaves * 16 * (kTaPitch + 2) <= kTaRing * kTaSlot, "a merge round of the private form fits in the buffers");
static_assert(sizeof(float) * 4 * 32 * (kTaPitch + 2) <= kTaRing * kTaSlot, "the merge of the shared form fits in the ring");

// Column c's node, c / G: c < 1024 and G <= 16.
__device__ __forceinline__ int node_of(const TreeAttnArgs& a, int c) { return (int)(((uint32_t)c * a.g_recip) >> 16); }

// What a workgroup works on: a tile of columns of one (batch, group) and a split of its blocks.
struct TreeUnit {
  int64_t bm;
  int split, tile;
  int first_node, last_node;  // of the tile
  uint64_t anc;               // A(lane)
  uint64_t present;           // nodes that are there
  int t;                      // committed tokens
};

// The tile's list entries, window by window.  The first two entries of each thread are requested before
// anything else is waited for.
struct TreeLists {
  static constexpr int kAhead = 2;
  int rows, n_listed;
  int64_t row0;
  int ahead[kAhead];

  // e / k_total: at most 64 k_total entries, and 64 k_total^2 < 2^36
  __device__ __forceinline__ int row_of(const TreeAttnArgs& a, int e) const { return (int)(((uint64_t)e * a.k_recip) >> 36); }
  __device__ __forceinline__ int entry(const TreeAttnArgs& a, int e) const {  // the block, or -1
    const int r = row_of(a, e), j = a.sel[row0 * a.k_total + e], c = a.cnt[row0 + r];
    return e - r * a.k_total < c ? j : -1;
  }
  __device__ __forceinline__ void request(const TreeAttnArgs& a, int64_t bm, int first_node, int last_node) {
    rows = a.n_sel == 1 ? 1 : last_node - first_node + 1;
    row0 = a.n_sel == 1 ? bm : bm * a.tb.n + first_node;
    n_listed = rows * a.k_total;
#pragma unroll
    for (int i = 0; i < kAhead; ++i) ahead[i] = entry(a, min((int)threadIdx.x + kTaThreads * i, n_listed - 1));
  }

  // The window of blocks from w0 on: table[j] = the tile's nodes that list block w0 + j, and this split's share of
  // the blocks with a node, ascending, in list, the drafted tokens behind the last window's.  Returns the share's
  // size; *tree_here says whether it holds the drafted tokens.  Every thread must call it.
  __device__ __forceinline__ int window(const TreeAttnArgs& a, const TreeUnit& u, int w0, int nb, TreeAttnLds& lds,
                                        bool* tree_here) const {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, ns = a.n_splits;
    const int wn = min(kTaWindow, nb - w0);
    __syncthreads();  // the last window's are no longer read
    for (int i = tid; i < wn; i += kTaThreads) lds.table[i] = 0ull;
    __syncthreads();
    auto mark = [&](int e, int block) {
      const int j = block - w0, r = row_of(a, e);
      if (block < 0 || j < 0 || j >= wn) return;
      if (a.n_sel == 1)
        lds.table[j] = ~0ull;
      else if ((u.present >> (u.first_node + r)) & 1ull)
        atomicOr(reinterpret_cast<unsigned long long*>(&lds.table[j]), 1ull << r);
    };
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      if (tid + kTaThreads * i < n_listed) mark(tid + kTaThreads * i, ahead[i]);
    for (int e = tid + kTaThreads * kAhead; e < n_listed; e += kTaThreads) mark(e, entry(a, e));
    __syncthreads();
    constexpr int kRounds = kTaWindow / kTaThreads;
    uint64_t listed[kRounds];
    int mine = 0;
#pragma unroll
    for (int i = 0; i < kRounds; ++i) {
      const int j = (wave * kRounds + i) * 64 + lane;
      listed[i] = __ballot(j < wn && lds.table[j] != 0ull);
      mine += (int)__popcll(listed[i]);
    }
    if (lane == 0) lds.count[wave] = mine;
    __syncthreads();
    int pos = 0, total = 0;
#pragma unroll
    for (int w = 0; w < kTaWaves; ++w) {
      pos += w < wave ? lds.count[w] : 0;
      total += lds.count[w];
    }
#pragma unroll
    for (int i = 0; i < kRounds; ++i) {
      const int at = pos + mbcnt64(listed[i]);
      const int share = (int)(((uint32_t)at * a.ns_recip) >> 20);  // at / ns: at < 2048, ns <= 64
      if (((listed[i] >> lane) & 1ull) && at - share * ns == u.split)
        lds.list[share] = (int16_t)((wave * kRounds + i) * 64 + lane);
      pos += (int)__popcll(listed[i]);
    }
    const int whole = (int)(((uint32_t)total * a.ns_recip) >> 20), over = total - whole * ns;
    const int n_blocks = whole + (u.split < over ? 1 : 0);
    *tree_here = w0 + kTaWindow >= nb && u.present != 0ull && over == u.split;
    if (*tree_here && tid == 0) lds.list[n_blocks] = (int16_t)kTaTree;
    __syncthreads();
    return n_blocks + (*tree_here ? 1 : 0);
  }
};

// A wavefront's 16 NT columns: lane (hh, grp) is column hh of every tile, k-chunk and token group grp.
template <int NT>
struct TreeCols {
  uint64_t anc[NT];   // A(node) of the lane's columns
  int node[NT];       // from the tile's first node
  bf16x8 q[NT][4];
  float m[NT], off[NT], l[NT];  // the softmax reference, -m once there is one (else 0), the lane's sum
  f32x4 o[NT][8];               // dims 16 dt + 4 grp + e
  float zscale;
  // 64 entries of the list, one per lane, and which of them each column's node lists
  int jv, chunk;
  uint64_t mine[NT];

  // Columns c0 + 16 nt + hh (those past n_cols repeat the last).
  __device__ __forceinline__ void load(const TreeAttnArgs& a, const TreeUnit& u, int c0) {
    const int lane = threadIdx.x & 63, hh = lane & 15, grp = lane >> 4, n = a.tb.n, G = a.group_size;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int c = min(c0 + 16 * nt + hh, n * G - 1), x = node_of(a, c);
      node[nt] = x - u.first_node;
      anc[nt] = ((uint64_t)(uint32_t)__shfl((int)(u.anc >> 32), x, 64) << 32) | (uint32_t)__shfl((int)(uint32_t)u.anc, x, 64);
      const uint16_t* qrow = a.q + ((u.bm * G + (c - x * G)) * n + x) * kHeadDim + 8 * grp;
#pragma unroll
      for (int ks = 0; ks < 4; ++ks) q[nt][ks] = as_bf16x8(ld16(qrow + 32 * ks));
      m[nt] = -INFINITY;
      off[nt] = l[nt] = 0.f;
#pragma unroll
      for (int dt = 0; dt < 8; ++dt) o[nt][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    // z = zscale (q . k) with zscale > 0, so that the largest q . k has the largest z: a negative scale moves into the
    // query's sign bits (exact), a scale of zero becomes the smallest positive one, so that masked scores (-inf) keep
    // weight 0
    zscale = a.sm_scale * kLog2eT;
    if (zscale < 0.f) {
      zscale = -zscale;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
          uint4 w = __builtin_bit_cast(uint4, q[nt][ks]);
          w.x ^= 0x80008000u;
          w.y ^= 0x80008000u;
          w.z ^= 0x80008000u;
          w.w ^= 0x80008000u;
          q[nt][ks] = as_bf16x8(w);
        }
    }
    if (zscale == 0.f) zscale = __FLT_MIN__;
  }

  // Entry e of the list: the block from the window's first on, or kTaTree.
  __device__ __forceinline__ int entry(const TreeAttnLds& lds, int e) const {
    return e >> 6 == chunk ? readlane_i(jv, e & 63) : __builtin_amdgcn_readfirstlane((int)lds.list[e]);
  }
  // Takes up the 64 entries around e of n_list.
  __device__ __forceinline__ void scan(const TreeAttnArgs& a, const TreeAttnLds& lds, int e, int n_list) {
    const int lane = threadIdx.x & 63;
    chunk = e >> 6;
    const int at = chunk * 64 + lane;
    jv = lds.list[min(at, n_list - 1)];
    const uint64_t nodes = at < n_list && jv != kTaTree ? lds.table[jv] : 0ull;
    if (a.n_sel == 1) {
      const uint64_t x = __ballot(nodes != 0ull);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) mine[nt] = anc[nt] ? x : 0ull;
    } else {
      const int lo = readlane_i(node[0], 0), hi = readlane_i(node[NT - 1], 15);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) mine[nt] = 0ull;
      for (int r = lo; r <= hi; ++r) {
        const uint64_t x = __ballot(((nodes >> r) & 1ull) != 0ull);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) mine[nt] = node[nt] == r ? x : mine[nt];
      }
    }
  }

  // One half block: K rows at kbuf, V rows at vbuf (rows of 256 bytes, 16-byte piece x of token t at x ^ (t % 16) for K
  // and x ^ 2 (t % 8) for V).  valid: its tokens that hold a V; they are the context's, or the drafted ones from node
  // 32 hf on.  k_read runs once K has been read, v_ready before V is; kVFirst: V is there already and is read before the
  // softmax.
  template <bool kVFirst, class KRead, class VReady>
  __device__ __forceinline__ void half(const char* kbuf, const char* vbuf, bool tree, int hf, int e, uint32_t valid,
                                       KRead k_read, VReady v_ready) {
    const int lane = threadIdx.x & 63, hh = lane & 15, grp = lane >> 4;
    // operand addresses: K row 16 tt + hh, piece (4 ks + grp) ^ hh; V rows 16 x + 4 grp + hh / 4, dims
    // 16 dt + 4 (hh % 4) .. + 3
    const uint32_t ka = hh * 256 + 16 * (grp ^ hh);
    const int vt = 4 * grp + (hh >> 2);
    const uint32_t va = vt * 256 + 16 * (((hh >> 1) & 1) ^ (2 * (vt & 7))) + 8 * (hh & 1);
    uint32_t vis[NT];
    bool on[NT], part[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      vis[nt] = tree ? (uint32_t)(anc[nt] >> (hf * kTaHalf)) : (mine[nt] >> (e & 63)) & 1ull ? valid : 0u;
      on[nt] = __ballot(vis[nt] != 0u) != 0ull;
      part[nt] = __ballot(vis[nt] != ~0u) != 0ull;
    }
    bf16x8 kf[2][4];
#pragma unroll
    for (int ks = 0; ks < 4; ++ks)
#pragma unroll
      for (int tt = 0; tt < 2; ++tt)
        kf[tt][ks] = as_bf16x8(*reinterpret_cast<const uint4*>(kbuf + 4096 * tt + (ka ^ (ks << 6))));
    f32x4 st[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      st[nt][0] = st[nt][1] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (!on[nt]) continue;
#pragma unroll
      for (int ks = 0; ks < 4; ++ks)
#pragma unroll
        for (int tt = 0; tt < 2; ++tt) st[nt][tt] = mfma16x16x32(kf[tt][ks], q[nt][ks], st[nt][tt]);
    }
    k_read();
    bf16x8 vf[8];
    auto read_v = [&] {
#pragma unroll
      for (int dt = 0; dt < 8; ++dt) {
        const uint2 v0 = lds_read_tr16(vbuf + (va ^ (dt << 5))), v1 = lds_read_tr16(vbuf + 4096 + (va ^ (dt << 5)));
        vf[dt] = as_bf16x8(make_uint4(v0.x, v0.y, v1.x, v1.y));
      }
    };
    if constexpr (kVFirst) read_v();  // under way during the softmax
    float top[NT];
    bool ask = false;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      top[nt] = -INFINITY;
      if (!on[nt]) continue;
      if (part[nt]) {
        const uint32_t bits = vis[nt] >> (4 * grp);
#pragma unroll
        for (int tt = 0; tt < 2; ++tt)
#pragma unroll
          for (int i = 0; i < 4; ++i) st[nt][tt][i] = (bits >> (16 * tt + i)) & 1u ? st[nt][tt][i] : -INFINITY;
      }
#pragma unroll
      for (int tt = 0; tt < 2; ++tt)
        top[nt] = fmaxf(top[nt], fmaxf(fmaxf(st[nt][tt][0], st[nt][tt][1]), fmaxf(st[nt][tt][2], st[nt][tt][3])));
      top[nt] *= zscale;
      ask |= top[nt] > m[nt] + kHeadroom;  // also on a column's first scores
    }
    if (__ballot(ask) != 0ull) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        float x = top[nt];
        x = fmaxf(x, __shfl_xor(x, 16, 64));
        x = fmaxf(x, __shfl_xor(x, 32, 64));
        if (x > m[nt] + kHeadroom) {
          const float alpha = __builtin_amdgcn_exp2f(m[nt] - x);
          m[nt] = x;
          off[nt] = -x;
          l[nt] *= alpha;
#pragma unroll
          for (int dt = 0; dt < 8; ++dt) o[nt][dt] *= alpha;
        }
      }
    }
    bf16x8 pb[NT], pr[NT];  // the weights rounded to bf16, and what the rounding took, rounded likewise
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      if (!on[nt]) continue;
      uint32_t big[4], rest[4];
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        float p[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          p[i] = __builtin_amdgcn_exp2f(fmaf(st[nt][x >> 1][2 * (x & 1) + i], zscale, off[nt]));
          l[nt] += p[i];
        }
        big[x] = pack_bf16(p[0], p[1]);
        rest[x] = pack_bf16(p[0] - bf16lo(big[x]), p[1] - bf16hi(big[x]));
      }
      pb[nt] = as_bf16x8(make_uint4(big[0], big[1], big[2], big[3]));
      pr[nt] = as_bf16x8(make_uint4(rest[0], rest[1], rest[2], rest[3]));
    }
    if constexpr (!kVFirst) {
      v_ready();
      read_v();
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      if (!on[nt]) continue;
#pragma unroll
      for (int dt = 0; dt < 8; ++dt) o[nt][dt] = mfma16x16x32(vf[dt], pr[nt], o[nt][dt]);
#pragma unroll
      for (int dt = 0; dt < 8; ++dt) o[nt][dt] = mfma16x16x32(vf[dt], pb[nt], o[nt][dt]);
    }
  }

  __device__ __forceinline__ float row_sum(int nt) const {  // l over the column's four lanes
    float x = l[nt];
    x += __shfl_xor(x, 16, 64);
    x += __shfl_xor(x, 32, 64);
    return x;
  }
};

// The tokens of a half block that hold a V.
__device__ __forceinline__ uint32_t half_valid(const TreeUnit& u, bool tree, int j, int hf) {
  if (tree) return (uint32_t)(u.present >> (hf * kTaHalf));
  const int left = u.t - (j * kBlock + hf * kTaHalf);  // committed tokens from the half's first on
  return left >= kTaHalf ? ~0u : left > 0 ? (1u << left) - 1u : 0u;
}

// 1 / den; 0 for a column without a token, whose den is 0.  NaN stays NaN.
__device__ __forceinline__ float inverse_of(float den) { return den == 0.f ? 0.f : 1.f / den; }

// Four dims of a finished column, or of a split's partial.
__device__ __forceinline__ void store_dims(const TreeAttnArgs& a, const TreeUnit& u, int c, int d, float m, float den,
                                           f32x4 num) {
  const int node = node_of(a, c);
  const int64_t row = (u.bm * a.group_size + (c - node * a.group_size)) * a.tb.n + node;
  if (a.n_splits == 1) {
    const float inv = inverse_of(den);
    uint2 w;
    w.x = (uint32_t)f32_to_bf16(num[0] * inv) | ((uint32_t)f32_to_bf16(num[1] * inv) << 16);
    w.y = (uint32_t)f32_to_bf16(num[2] * inv) | ((uint32_t)f32_to_bf16(num[3] * inv) << 16);
    *reinterpret_cast<uint2*>(a.o + row * kHeadDim + d) = w;
  } else {
    float* pp = a.ws + (row * a.n_splits + u.split) * kTaPartial;
    if (d == 0) *reinterpret_cast<float2*>(pp) = make_float2(m, den);
    *reinterpret_cast<f32x4*>(pp + 4 + d) = num;
  }
}

// The workgroup's unit; false: none.  Grid x = 8 n_tiles, y = (groups x splits) / 8: workgroups 8 apart run on the same
// XCD, so the tiles of a (group, split) share its L2, and few groups still spread over all XCDs.
__device__ __forceinline__ bool tree_unit(const TreeAttnArgs& a, int n_groups, int tile_cols, TreeUnit* u, TreeLists* lists) {
  const int lane = threadIdx.x & 63, n = a.tb.n, G = a.group_size;
  const int unit = blockIdx.y * 8 + (blockIdx.x & 7);
  if (unit >= n_groups * a.n_splits) return false;
  u->tile = blockIdx.x >> 3;
  u->split = a.n_splits == 1 ? 0 : (int)(((uint64_t)unit * a.groups_recip) >> 36);  // with splits: below 2^14 units
  u->bm = unit - u->split * n_groups;
  const int c0 = u->tile * tile_cols;
  u->first_node = node_of(a, c0);
  u->last_node = node_of(a, min(c0 + tile_cols, n * G) - 1);
  lists->request(a, u->bm, u->first_node, u->last_node);
  const int b = (int)(u->bm / a.n_kv_heads);
  const int64_t ctx = tree_context(a.tb, b);
  u->anc = tree_ancestors(a.tb.parent + (int64_t)b * n, n, lane);
  if (ctx < 0) u->anc = 0ull;
  u->t = ctx < 0 ? 0 : (int)ctx;
  u->present = __ballot(u->anc != 0ull);
  return true;
}

// ---- up to 32 columns: every wavefront streams halves of its own -------------------------------------

template <int NT, bool kOnce>
__global__ __launch_bounds__(kTaThreads) void tree_attn_kernel(TreeAttnArgs a, int n_groups) {
  __shared__ __align__(16) TreeAttnLds lds;
  const int tid = threadIdx.x, lane = tid & 63, hh = lane & 15, grp = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = a.tb.n, c0_tile = 16 * NT;
  TreeUnit u;
  TreeLists lists;
  if (!tree_unit(a, n_groups, c0_tile, &u, &lists)) return;
  const int c0 = u.tile * c0_tile;
  TreeCols<NT> cols;
  cols.load(a, u, c0);

  char* const kbuf = lds.kv + wave * 2 * kTaBuf;
  char* const vbuf = kbuf + kTaBuf;
  const uint32_t k_at = __builtin_amdgcn_readfirstlane(lds_address(kbuf)), v_at = k_at + kTaBuf;
  // staging: instruction i brings token rows 4 i + r4
  const int r4 = lane >> 4;
  const uint32_t k_off = r4 * 256 + 16 * ((lane & 15) ^ r4), v_off = r4 * 256 + 16 * ((lane & 15) ^ (2 * r4));
  auto issue = [&](const uint16_t* cache, const uint16_t* drafted, int j, int hf, uint32_t off0, int flip, int by,
                   uint32_t dst) {
    if (j < kTaTreeBlock) {
      const char* src = reinterpret_cast<const char*>(cache + (u.bm * a.t_cap + (int64_t)j * kBlock + hf * kTaHalf) * kHeadDim);
#pragma unroll
      for (int i = 0; i < 8; ++i) lds_load16<kOnce>(src + 1024 * i, off0 ^ ((i & flip) << by), dst + 1024 * i);
    } else {  // rows past the last node repeat it
      const char* src = reinterpret_cast<const char*>(drafted + u.bm * n * kHeadDim);
#pragma unroll 1
      for (int i = 0; i < 8; ++i) {
        const int row = min(hf * kTaHalf + 4 * i + r4, n - 1);
        lds_load16<kOnce>(src, row * 256 + ((off0 ^ ((i & flip) << by)) & 255), dst + 1024 * i);
      }
    }
  };
  auto issue_k = [&](int j, int hf) { issue(a.k, a.kt, j, hf, k_off, 3, 6, k_at); };
  auto issue_v = [&](int j, int hf) { issue(a.v, a.vt, j, hf, v_off, 1, 7, v_at); };

  const int nb = (u.t + kBlock - 1) / kBlock;
  for (int w0 = 0; w0 == 0 || w0 < nb; w0 += kTaWindow) {
    bool tree_here;
    const int n_list = lists.window(a, u, w0, nb, lds, &tree_here);
    const int n_items = 2 * n_list - (tree_here && n <= kTaHalf ? 1 : 0);
    auto block_of = [&](int j) { return j + (j == kTaTree ? kTaTreeBlock : w0); };
    cols.chunk = -1;
    int x = wave;
    int j = 0;
    if (x < n_items) {
      j = block_of(cols.entry(lds, x >> 1));
      issue_k(j, x & 1);
      issue_v(j, x & 1);
    }
    lds_loads_landed();  // the first half and the queries: from here on the loads are counted
    while (x < n_items) {
      const int e = x >> 1, hf = x & 1, x2 = x + kTaWaves;
      const bool more = x2 < n_items, tree = j >= kTaTreeBlock;
      if (e >> 6 != cols.chunk) cols.scan(a, lds, e, n_list);
      const int j2 = more ? block_of(cols.entry(lds, x2 >> 1)) : 0;
      const uint32_t valid = half_valid(u, tree, j, hf);
      __asm__ __volatile__("s_waitcnt vmcnt(8)" ::: "memory");  // this half's K (its V may be under way)
      cols.template half<false>(
          kbuf, vbuf, tree, hf, e, valid,
          [&] {
            __asm__ __volatile__("s_waitcnt lgkmcnt(0)" ::: "memory");  // K has been read
            if (more) issue_k(j2, x2 & 1);
          },
          [&] {
            if (more)
              __asm__ __volatile__("s_waitcnt vmcnt(8)" ::: "memory");  // this half's V (the next K may be under way)
            else
              __asm__ __volatile__("s_waitcnt vmcnt(0)" ::: "memory");
            if (valid != ~0u) {  // rows that no column may see: whatever lies there becomes zeros
              for (int r = r4; r < kTaHalf; r += 4)
                if (!((valid >> r) & 1u)) *reinterpret_cast<uint4*>(vbuf + r * 256 + 16 * (lane & 15)) = make_uint4(0u, 0u, 0u, 0u);
              wave_lds_sync();
            }
          });
      __asm__ __volatile__("s_waitcnt lgkmcnt(0)" ::: "memory");  // V has been read
      if (more) issue_v(j2, x2 & 1);
      x = x2;
      j = j2;
    }
  }

  // the wavefronts' states, 16 columns at a time, through the buffers' space
  float* st_m = reinterpret_cast<float*>(lds.kv);  // [waves][16]
  float* st_l = st_m + kTaWaves * 16;              // [waves][16]
  float* st_o = st_l + kTaWaves * 16;              // [waves][16][kTaPitch]
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    __syncthreads();
    const float l = cols.row_sum(nt);
    if (grp == 0) {
      st_m[wave * 16 + hh] = cols.m[nt];
      st_l[wave * 16 + hh] = l;
    }
#pragma unroll
    for (int dt = 0; dt < 8; ++dt)
      *reinterpret_cast<f32x4*>(&st_o[(wave * 16 + hh) * kTaPitch + 16 * dt + 4 * grp]) = cols.o[nt][dt];
    __syncthreads();
    const int cl = tid >> 5, d = 4 * (tid & 31), c = c0 + 16 * nt + cl;  // 16 columns x 32 quads of dims
    if (c < n * a.group_size) {
      float m = -INFINITY;
#pragma unroll
      for (int w = 0; w < kTaWaves; ++w) m = fmaxf(m, st_m[w * 16 + cl]);
      // a wavefront without a score has m = -inf and weighs nothing; one whose scores are all NaN has m = -inf too, and
      // sums of NaN that reach the result
      const float ref = m > -INFINITY ? m : 0.f;
      float den = 0.f;
      f32x4 num = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < kTaWaves; ++w) {
        const float sc = __builtin_amdgcn_exp2f(st_m[w * 16 + cl] - ref);
        den = fmaf(st_l[w * 16 + cl], sc, den);
        num += *reinterpret_cast<const f32x4*>(&st_o[(w * 16 + cl) * kTaPitch + d]) * sc;
      }
      store_dims(a, u, c, d, m, den, num);
    }
  }
}

// ---- more columns: the wavefronts share the blocks ------------------------------------------------------

// kOnce: no other workgroup reads the blocks, so they bypass the caches (16 nodes of 256 groups of 4 heads at 128K
// 108 -> 93 us).  WC groups of 16 NT columns; with WC = 4 two wavefronts take a group, one half of every block each.
template <int NT, int WC, bool kOnce>
__global__ __launch_bounds__(kTaThreads) void tree_attn_shared_kernel(TreeAttnArgs a, int n_groups) {
  constexpr int WT = kTaWaves / WC;
  static_assert(WT == 1 || WT == 2, "a wavefront takes whole blocks or halves");
  __shared__ __align__(16) TreeAttnLds lds;
  const int tid = threadIdx.x, lane = tid & 63, hh = lane & 15, grp = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int cg = wave % WC, th = wave / WC;
  const int n = a.tb.n;
  TreeUnit u;
  TreeLists lists;
  if (!tree_unit(a, n_groups, 16 * NT * WC, &u, &lists)) return;
  const int c0 = (u.tile * WC + cg) * 16 * NT;
  const bool live = c0 < n * a.group_size;  // the last tile may leave wavefronts without columns: they only load
  TreeCols<NT> cols;
  cols.load(a, u, c0);

  // staging: a wavefront brings token rows 8 wave .. + 7 of K and of V, 4 rows per instruction
  const int r4 = lane >> 4;
  const uint32_t ring_at = __builtin_amdgcn_readfirstlane(lds_address(lds.kv)) + wave * 2048;
  auto issue = [&](int j, int slot) {
    const uint32_t dst = ring_at + slot * kTaSlot;
    const bool tree = j >= kTaTreeBlock;
    const int64_t at = (tree ? u.bm * n : u.bm * a.t_cap + (int64_t)j * kBlock) * kHeadDim;
    const uint16_t* const kp = (tree ? a.kt : a.k) + at;
    const uint16_t* const vp = (tree ? a.vt : a.v) + at;
    const int last = tree ? n - 1 : kBlock - 1;  // rows past the last node repeat it
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int row = 8 * wave + 4 * i + r4;
      const uint32_t from = min(row, last) * 256;
      lds_load16<kOnce>(kp, from + 16 * ((lane & 15) ^ (row & 15)), dst + 1024 * i);
      lds_load16<kOnce>(vp, from + 16 * ((lane & 15) ^ (2 * (row & 7))), dst + 2 * kTaBuf + 1024 * i);
    }
  };

  const int nb = (u.t + kBlock - 1) / kBlock;
  for (int w0 = 0; w0 == 0 || w0 < nb; w0 += kTaWindow) {
    bool tree_here;
    const int n_list = lists.window(a, u, w0, nb, lds, &tree_here);
    auto block_of = [&](int j) { return j + (j == kTaTree ? kTaTreeBlock : w0); };
    cols.chunk = -1;
    lds_loads_landed();  // the queries: from here on the loads are counted, 4 per block
#pragma unroll 1
    for (int s = 0; s < kTaRing - 1; ++s)
      if (s < n_list) issue(block_of(cols.entry(lds, s)), s);
    for (int s = 0; s < n_list; ++s) {
      if (s >> 6 != cols.chunk) cols.scan(a, lds, s, n_list);
      const int j = block_of(cols.entry(lds, s));
      const bool tree = j >= kTaTreeBlock;
      char* const kslot = lds.kv + (s % kTaRing) * kTaSlot;
      char* const vslot = kslot + 2 * kTaBuf;
      // this wavefront's rows of block s have landed (two more blocks may be under way), the rows of V that no column
      // may see become zeros, and its reads of block s - 1 have returned; then everybody's have
      if (s + 2 < n_list)
        __asm__ __volatile__("s_waitcnt vmcnt(8)" ::: "memory");
      else if (s + 1 < n_list)
        __asm__ __volatile__("s_waitcnt vmcnt(4)" ::: "memory");
      else
        __asm__ __volatile__("s_waitcnt vmcnt(0)" ::: "memory");
      const uint64_t valid = half_valid(u, tree, j, 0) | (uint64_t)half_valid(u, tree, j, 1) << 32;
      if (valid != ~0ull) {
        for (int r = 8 * wave + r4; r < 8 * wave + 8; r += 4)
          if (!((valid >> r) & 1ull)) *reinterpret_cast<uint4*>(vslot + r * 256 + 16 * (lane & 15)) = make_uint4(0u, 0u, 0u, 0u);
      }
      __asm__ __volatile__("s_waitcnt lgkmcnt(0)" ::: "memory");
      __builtin_amdgcn_s_barrier();
      __asm__ __volatile__("" ::: "memory");
      if (s + kTaRing - 1 < n_list) issue(block_of(cols.entry(lds, s + kTaRing - 1)), (s + kTaRing - 1) % kTaRing);
      if (!live) continue;
#pragma unroll 1
      for (int h = WT == 2 ? th : 0; h < (WT == 2 ? th + 1 : 2); ++h) {
        cols.template half<true>(kslot + h * kTaBuf, vslot + h * kTaBuf, tree, h, s, (uint32_t)(valid >> (h * kTaHalf)), [] {}, [] {});
      }
    }
    __asm__ __volatile__("s_waitcnt lgkmcnt(0)" ::: "memory");
  }

  if constexpr (WT == 2) {  // the second half's states, through the ring's space
    __syncthreads();
    float* st_m = reinterpret_cast<float*>(lds.kv);  // [WC][16 NT]
    float* st_l = st_m + WC * 16 * NT;
    float* st_o = st_l + WC * 16 * NT;               // [WC][16 NT][kTaPitch]
    const int at = cg * 16 * NT + hh;
    if (th == 1) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        if (grp == 0) st_m[at + 16 * nt] = cols.m[nt];
        const float l = cols.row_sum(nt);
        if (grp == 0) st_l[at + 16 * nt] = l;
#pragma unroll
        for (int dt = 0; dt < 8; ++dt)
          *reinterpret_cast<f32x4*>(&st_o[(at + 16 * nt) * kTaPitch + 16 * dt + 4 * grp]) = cols.o[nt][dt];
      }
    }
    __syncthreads();
    if (th == 1) return;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const float m1 = st_m[at + 16 * nt], m = fmaxf(cols.m[nt], m1), ref = m > -INFINITY ? m : 0.f;
      const float s0 = __builtin_amdgcn_exp2f(cols.m[nt] - ref), s1 = __builtin_amdgcn_exp2f(m1 - ref);
      cols.l[nt] = cols.row_sum(nt) * s0 + st_l[at + 16 * nt] * s1;
      cols.m[nt] = m;
#pragma unroll
      for (int dt = 0; dt < 8; ++dt)
        cols.o[nt][dt] = cols.o[nt][dt] * s0 + *reinterpret_cast<const f32x4*>(&st_o[(at + 16 * nt) * kTaPitch + 16 * dt + 4 * grp]) * s1;
    }
  }
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const float l = WT == 2 ? cols.l[nt] : cols.row_sum(nt);
    const int c = c0 + 16 * nt + hh;
    if (c >= n * a.group_size) continue;
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) store_dims(a, u, c, 16 * dt + 4 * grp, cols.m[nt], l, cols.o[nt][dt]);
  }
}

// Merge the splits' partials of one (node, query head): one wavefront, two head dims per lane, up to 8
// splits requested at once.
__global__ __launch_bounds__(kCombineThreads) void tree_combine_kernel(TreeAttnArgs a, int64_t n_rows) {
  const int lane = threadIdx.x & 63;
  const int64_t row = (int64_t)blockIdx.x * (kCombineThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (row >= n_rows) return;
  constexpr int kStride = kTaPartial;
  const float* base = a.ws + row * a.n_splits * kStride;
  float m = -INFINITY, l = 0.f, o0 = 0.f, o1 = 0.f;
  for (int s0 = 0; s0 < a.n_splits; s0 += 8) {
    float2 ml[8], po[8];
    float top = m;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float* src = base + min(s0 + i, a.n_splits - 1) * kStride;
      ml[i] = *reinterpret_cast<const float2*>(src);
      po[i] = *reinterpret_cast<const float2*>(src + 4 + 2 * lane);
      if (s0 + i >= a.n_splits) ml[i].x = -INFINITY;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) top = fmaxf(top, ml[i].x);
    const float ref = top > -INFINITY ? top : 0.f;  // as in the merge of the wavefronts
    const float keep = __builtin_amdgcn_exp2f(m - ref);
    l *= keep;
    o0 *= keep;
    o1 *= keep;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float w = __builtin_amdgcn_exp2f(ml[i].x - ref);
      l = fmaf(ml[i].y, w, l);
      o0 = fmaf(po[i].x, w, o0);
      o1 = fmaf(po[i].y, w, o1);
    }
    m = top;
  }
  const float inv = inverse_of(l);
  reinterpret_cast<uint32_t*>(a.o + row * kHeadDim)[lane] = (uint32_t)f32_to_bf16(o0 * inv) | ((uint32_t)f32_to_bf16(o1 * inv) << 16);
}

template <class Kernel>
hipError_t launch_tiles(Kernel kernel, const TreeAttnArgs& a, int tile_cols, hipStream_t stream) {
  const int groups = a.tb.batch * a.n_kv_heads;
  const int n_tiles = (a.tb.n * a.group_size + tile_cols - 1) / tile_cols;
  hipLaunchKernelGGL(kernel, dim3((unsigned)(8 * n_tiles), (unsigned)((groups * a.n_splits + 7) / 8)), dim3(kTaThreads), 0,
                     stream, a, groups);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_tree_attn(const TreeAttnArgs& a, hipStream_t stream) {
  const int cols = a.tb.n * a.group_size;
  const int width = a.width;
  const bool once = cols <= width;  // one tile: every block is read once
  const hipError_t e = width == 16    ? launch_tiles(tree_attn_kernel<1, true>, a, width, stream)
                       : width == 32  ? launch_tiles(once ? tree_attn_kernel<2, true> : tree_attn_kernel<2, false>, a, width, stream)
                       : width == 64  ? launch_tiles(tree_attn_shared_kernel<1, 4, true>, a, width, stream)
                       : width == 128 ? launch_tiles(tree_attn_shared_kernel<2, 4, true>, a, width, stream)
                                      : launch_tiles(once ? tree_attn_shared_kernel<2, 8, true> : tree_attn_shared_kernel<2, 8, false>, a, width, stream);
  if (e != hipSuccess || a.n_splits == 1) return e;
  const int64_t rows = (int64_t)a.tb.batch * a.n_kv_heads * a.group_size * a.tb.n;
  hipLaunchKernelGGL(tree_combine_kernel, dim3((unsigned)((rows + 3) / 4)), dim3(kCombineThreads), 0, stream, a, rows);
  return hipGetLastError();
}

}  // namespace sparda
