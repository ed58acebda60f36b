// tree_attention.hip -- attention of the nodes of drafted-token trees over their blocks of the cache
// and their ancestors (paper Sec. 4.1, Eq. 5 over the set of Eq. 1):
//   o_i = softmax(sm_scale q_i K^T) V over {t' < t in the blocks of node i} U A(i).
//
// Work unit: a tile of up to 16 NT columns (column c is query head c % G of node c / G) of one (batch,
// group), and a split of the blocks that any of the tile's nodes lists.  One pass over K and V serves all
// columns of the tile, with the running maximum and sum of the softmax in registers.
//   1. The lists of the tile's nodes become a table in LDS, one 64-bit mask of nodes per block (entries
//      outside the context are dropped, a repeated one sets its bit again), and the blocks with a mask
//      an ascending list.  Split s takes every n_splits-th of them.  The drafted tokens are one more
//      entry.  Contexts of more than 2048 blocks are walked in windows of 2048.
//   2. Each of the 8 wavefronts takes halves of blocks (32 tokens, 8 KiB of K and of V) in turn.  They go
//      from memory straight into two LDS buffers of its own, the next half's K in flight from the moment
//      the products of this one have read K, its V from the moment O has read V; the wavefront waits for
//      its own loads by count, and no barrier joins the wavefronts until the merge.
//   3. Per half and 16 columns: S^T = K Q^T on v_mfma_f32_16x16x32_bf16 (lane (c, g) holds column c's
//      scores of tokens 16 tt + 4 g + i); masks; P = 2^(z - m) with a reference m that moves only when a
//      score exceeds it by more than 2^8; O^T += V^T P^T on the same MFMA, V read through the transposing
//      LDS read.  The denominators sum P in float32, before it is rounded to bf16 for the product (a
//      weight is off by at most 2^-8 of itself).
//   4. The wavefronts' states merge through LDS; with splits their float32 partials go to the workspace
//      and a second launch merges them.
#include <math.h>

#include "device_util.hpp"
#include "launch.hpp"
#include "tree.hpp"

namespace sparda {

namespace {

constexpr float kLog2eT = 1.4426950408889634f;
constexpr int kTaWaves = 8;
constexpr int kTaThreads = 64 * kTaWaves;
constexpr int kTaHalf = 32;                          // tokens per half block
constexpr int kTaBuf = kTaHalf * kHeadDim * 2;       // bytes of a half's K or V
constexpr int kTaWindow = 2048;                      // blocks per window of the table
constexpr int kTaTree = 0x7fff;                      // the list's entry of the drafted tokens
constexpr int kTaPitch = kHeadDim + 4;               // floats per merged row: 16 rows of 16 bytes touch every bank once
constexpr int kCombineThreads = 256;

struct TreeAttnLds {
  char kv[kTaWaves][2][kTaBuf];
  uint64_t table[kTaWindow];
  int16_t list[kTaWindow + 1];
  int count[kTaWaves];
};
static_assert(sizeof(float) * kTaWaves * 16 * (kTaPitch + 2) <= sizeof(char) * kTaWaves * 2 * kTaBuf, "a merge round fits in the buffers");
static_assert(sizeof(TreeAttnLds) <= 160 * 1024, "LDS of one CU");

template <int NT>
__global__ __launch_bounds__(kTaThreads) void tree_attn_kernel(TreeAttnArgs a, int n_tiles, int n_groups) {
  __shared__ __align__(16) TreeAttnLds lds;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = a.tb.n, G = a.group_size, ns = a.n_splits;
  // workgroups 8 apart run on the same XCD: the tiles of a (group, split) share its L2
  const int unit = (int)(blockIdx.x / (8 * n_tiles)) * 8 + (int)(blockIdx.x % 8);
  const int tile = (int)(blockIdx.x / 8) % n_tiles;
  if (unit >= n_groups * ns) return;
  const int64_t bm = unit % n_groups;
  const int split = unit / n_groups;
  const int b = (int)(bm / a.n_kv_heads);
  const int hh = lane & 15, grp = lane >> 4;
  const int n_cols = n * G, c0 = tile * 16 * NT;
  const int first_node = c0 / G, last_node = (min(c0 + 16 * NT, n_cols) - 1) / G;
  // The tile's list entries: the first two of each thread are requested before anything is waited for.
  const int rows = a.n_sel == 1 ? 1 : last_node - first_node + 1;
  const int64_t row0 = a.n_sel == 1 ? bm : bm * n + first_node;
  const int n_listed = rows * a.k_total;
  auto list_row = [&](int e) { return e / a.k_total; };
  auto list_entry = [&](int e) {  // the block, or -1; the count and the entry are requested together
    const int r = list_row(e), j = a.sel[row0 * a.k_total + e], c = a.cnt[row0 + r];
    return e - r * a.k_total < c ? j : -1;
  };
  constexpr int kAhead = 2;
  int ahead[kAhead];
#pragma unroll
  for (int i = 0; i < kAhead; ++i) ahead[i] = list_entry(min(tid + kTaThreads * i, n_listed - 1));
  const int64_t ctx = tree_context(a.tb, b);
  uint64_t anc = tree_ancestors(a.tb.parent + (int64_t)b * n, n, lane);
  if (ctx < 0) anc = 0ull;
  const int t = ctx < 0 ? 0 : (int)ctx;
  const uint64_t present = __ballot(anc != 0ull);

  // ---- the lane's columns (those past the last repeat it) and their queries
  uint64_t col_anc[NT];
  int col_node[NT];  // from the tile's first node
  bf16x8 qb[NT][4];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int c = min(c0 + 16 * nt + hh, n_cols - 1), node = c / G;
    col_node[nt] = node - first_node;
    col_anc[nt] = ((uint64_t)(uint32_t)__shfl((int)(anc >> 32), node, 64) << 32) | (uint32_t)__shfl((int)(uint32_t)anc, node, 64);
    const uint16_t* qrow = a.q + ((bm * G + c % G) * n + node) * kHeadDim + 8 * grp;
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) qb[nt][ks] = as_bf16x8(ld16(qrow + 32 * ks));
  }
  // z = zscale (q . k) with zscale > 0, so that the largest q . k has the largest z: a negative scale moves
  // into the query's sign bits (exact), a scale of zero becomes the smallest positive one, so that masked
  // scores (-inf) keep weight 0
  float zscale = a.sm_scale * kLog2eT;
  if (zscale < 0.f) {
    zscale = -zscale;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int ks = 0; ks < 4; ++ks) {
        uint4 w = __builtin_bit_cast(uint4, qb[nt][ks]);
        w.x ^= 0x80008000u;
        w.y ^= 0x80008000u;
        w.z ^= 0x80008000u;
        w.w ^= 0x80008000u;
        qb[nt][ks] = as_bf16x8(w);
      }
  }
  if (zscale == 0.f) zscale = __FLT_MIN__;
  constexpr float kHeadroom = 8.f;
  float m_run[NT], off[NT], l_run[NT];  // off: -m_run once there is one
  f32x4 o[NT][8];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    m_run[nt] = -INFINITY;
    off[nt] = 0.f;
    l_run[nt] = 0.f;
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) o[nt][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  const char* kbuf = lds.kv[wave][0];
  const char* vbuf = lds.kv[wave][1];
  const uint32_t k_at = __builtin_amdgcn_readfirstlane(lds_address(kbuf));
  const uint32_t v_at = k_at + kTaBuf;
  // staging: instruction i brings token rows 4 i + r4; piece x of token t lies at x ^ (t % 16) for K and at
  // x ^ 2 (t % 8) for V
  const int r4 = lane >> 4;
  const uint32_t k_off = r4 * 256 + 16 * ((lane & 15) ^ r4), v_off = r4 * 256 + 16 * ((lane & 15) ^ (2 * r4));
  auto issue = [&](const uint16_t* cache, const uint16_t* drafted, int j, int hf, uint32_t off0, int flip, int by,
                   uint32_t dst) {
    if (j != kTaTree) {
      const char* src = reinterpret_cast<const char*>(cache + (bm * a.t_cap + (int64_t)j * kBlock + hf * kTaHalf) * kHeadDim);
#pragma unroll
      for (int i = 0; i < 8; ++i) lds_load16(src + 1024 * i, off0 ^ ((i & flip) << by), dst + 1024 * i);
    } else {  // rows past the last node repeat it
      const char* src = reinterpret_cast<const char*>(drafted + bm * n * kHeadDim);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int row = min(hf * kTaHalf + 4 * i + r4, n - 1);
        lds_load16(src, row * 256 + ((off0 ^ ((i & flip) << by)) & 255), dst + 1024 * i);
      }
    }
  };
  auto issue_k = [&](int j, int hf) { issue(a.k, a.kt, j, hf, k_off, 3, 6, k_at); };
  auto issue_v = [&](int j, int hf) { issue(a.v, a.vt, j, hf, v_off, 1, 7, v_at); };
  // operand addresses: K row 16 tt + hh, piece (4 ks + grp) ^ hh; V rows 16 x + 4 grp + hh / 4, dims
  // 16 dt + 4 (hh % 4) .. + 3
  const uint32_t ka = hh * 256 + 16 * (grp ^ hh);
  const int vt = 4 * grp + (hh >> 2);
  const uint32_t va = vt * 256 + 16 * (((hh >> 1) & 1) ^ (2 * (vt & 7))) + 8 * (hh & 1);

  const int nb = (t + kBlock - 1) / kBlock;
  for (int w0 = 0; w0 == 0 || w0 < nb; w0 += kTaWindow) {
    const int wn = min(kTaWindow, nb - w0);
    const bool final_window = w0 + kTaWindow >= nb;
    // ---- 1. the window's table and list
    __syncthreads();  // the last window's are no longer read
    for (int i = tid; i < wn; i += kTaThreads) lds.table[i] = 0ull;
    __syncthreads();
    auto mark = [&](int e, int block) {
      const int j = block - w0, r = list_row(e);
      if (block < 0 || j < 0 || j >= wn) return;
      if (a.n_sel == 1)
        lds.table[j] = ~0ull;
      else if ((present >> (first_node + r)) & 1ull)
        atomicOr(reinterpret_cast<unsigned long long*>(&lds.table[j]), 1ull << r);
    };
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      if (tid + kTaThreads * i < n_listed) mark(tid + kTaThreads * i, ahead[i]);
    for (int e = tid + kTaThreads * kAhead; e < n_listed; e += kTaThreads) mark(e, list_entry(e));
    __syncthreads();
    constexpr int kRounds = kTaWindow / kTaThreads;
    uint64_t listed[kRounds];
    int mine_n = 0;
#pragma unroll
    for (int i = 0; i < kRounds; ++i) {
      const int j = (wave * kRounds + i) * 64 + lane;
      listed[i] = __ballot(j < wn && lds.table[j] != 0ull);
      mine_n += (int)__popcll(listed[i]);
    }
    if (lane == 0) lds.count[wave] = mine_n;
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
      if (((listed[i] >> lane) & 1ull) && at % ns == split) lds.list[at / ns] = (int16_t)((wave * kRounds + i) * 64 + lane);
      pos += (int)__popcll(listed[i]);
    }
    const bool tree_here = final_window && present != 0ull && total % ns == split;
    const int n_entries = (total - split + ns - 1) / ns;
    if (tree_here && tid == 0) lds.list[n_entries] = (int16_t)kTaTree;
    const int n_items = 2 * n_entries + (tree_here ? (n > kTaHalf ? 2 : 1) : 0);
    __syncthreads();

    // ---- 2. and 3.
    int jv = 0, chunk = -1;      // 64 entries of the list, one per lane
    uint64_t mine[NT];           // which of them the column's node lists
    auto entry = [&](int e) { return e >> 6 == chunk ? readlane_i(jv, e & 63) : __builtin_amdgcn_readfirstlane((int)lds.list[e]); };
    auto scan = [&](int e) {
      chunk = e >> 6;
      const int at = chunk * 64 + lane, last = n_entries + (tree_here ? 1 : 0) - 1;
      jv = lds.list[min(at, last)];
      const uint64_t nodes = at <= last && jv != kTaTree ? lds.table[jv] : 0ull;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) mine[nt] = 0ull;
      if (a.n_sel == 1) {
        const uint64_t x = __ballot(nodes != 0ull);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) mine[nt] = col_anc[nt] ? x : 0ull;
      } else {
        for (int r = 0; r <= last_node - first_node; ++r) {
          const uint64_t x = __ballot(((nodes >> r) & 1ull) != 0ull);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) mine[nt] = col_node[nt] == r ? x : mine[nt];
        }
      }
    };
    auto block_of = [&](int j) { return j == kTaTree ? j : j + w0; };
    int x = wave;
    int j = 0;
    if (x < n_items) {
      j = block_of(entry(x >> 1));
      issue_k(j, x & 1);
      issue_v(j, x & 1);
    }
    lds_loads_landed();  // the first half and the queries: from here on the loads are counted
    while (x < n_items) {
      const int e = x >> 1, hf = x & 1, x2 = x + kTaWaves;
      const bool more = x2 < n_items;
      if (e >> 6 != chunk) scan(e);
      const int j2 = more ? block_of(entry(x2 >> 1)) : 0;
      // which tokens of the half hold a V, and which of them each column sees
      const bool tree = j == kTaTree;
      const int left = t - (j * kBlock + hf * kTaHalf);  // committed tokens from the half's first on
      const uint32_t valid = tree ? (uint32_t)(present >> (hf * kTaHalf)) : left >= kTaHalf ? ~0u : left > 0 ? (1u << left) - 1u : 0u;
      uint32_t vis[NT];
      bool on[NT], part[NT];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        vis[nt] = tree ? (uint32_t)(col_anc[nt] >> (hf * kTaHalf)) : (mine[nt] >> (e & 63)) & 1ull ? valid : 0u;
        on[nt] = __ballot(vis[nt] != 0u) != 0ull;
        part[nt] = __ballot(vis[nt] != ~0u) != 0ull;
      }
      __asm__ __volatile__("s_waitcnt vmcnt(8)" ::: "memory");  // this half's K (its V may be under way)
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
          for (int tt = 0; tt < 2; ++tt) st[nt][tt] = mfma16x16x32(kf[tt][ks], qb[nt][ks], st[nt][tt]);
      }
      __asm__ __volatile__("s_waitcnt lgkmcnt(0)" ::: "memory");  // K has been read
      if (more) issue_k(j2, x2 & 1);
      float bmax[NT];
      bool ask = false;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        if (!on[nt]) {
          bmax[nt] = -INFINITY;
          continue;
        }
        if (part[nt]) {
          const uint32_t bits = vis[nt] >> (4 * grp);
#pragma unroll
          for (int tt = 0; tt < 2; ++tt)
#pragma unroll
            for (int i = 0; i < 4; ++i) st[nt][tt][i] = (bits >> (16 * tt + i)) & 1u ? st[nt][tt][i] : -INFINITY;
        }
        float top = -INFINITY;
#pragma unroll
        for (int tt = 0; tt < 2; ++tt)
          top = fmaxf(top, fmaxf(fmaxf(st[nt][tt][0], st[nt][tt][1]), fmaxf(st[nt][tt][2], st[nt][tt][3])));
        bmax[nt] = top * zscale;
        ask |= bmax[nt] > m_run[nt] + kHeadroom;  // also on a column's first scores
      }
      if (__ballot(ask) != 0ull) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          float m = bmax[nt];
          m = fmaxf(m, __shfl_xor(m, 16, 64));
          m = fmaxf(m, __shfl_xor(m, 32, 64));
          if (m > m_run[nt] + kHeadroom) {
            const float alpha = __builtin_amdgcn_exp2f(m_run[nt] - m);
            m_run[nt] = m;
            off[nt] = -m;
            l_run[nt] *= alpha;
#pragma unroll
            for (int dt = 0; dt < 8; ++dt) o[nt][dt] *= alpha;
          }
        }
      }
      bf16x8 pb[NT];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        if (!on[nt]) continue;
        float p[2][4];
#pragma unroll
        for (int tt = 0; tt < 2; ++tt)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            p[tt][i] = __builtin_amdgcn_exp2f(fmaf(st[nt][tt][i], zscale, off[nt]));
            l_run[nt] += p[tt][i];
          }
        pb[nt] = as_bf16x8(make_uint4(pack_bf16(p[0][0], p[0][1]), pack_bf16(p[0][2], p[0][3]),
                                      pack_bf16(p[1][0], p[1][1]), pack_bf16(p[1][2], p[1][3])));
      }
      if (more)
        __asm__ __volatile__("s_waitcnt vmcnt(8)" ::: "memory");  // this half's V (the next K may be under way)
      else
        __asm__ __volatile__("s_waitcnt vmcnt(0)" ::: "memory");
      if (valid != ~0u) {  // rows that no column may see: whatever lies there becomes zeros
        for (int r = r4; r < kTaHalf; r += 4)
          if (!((valid >> r) & 1u))
            *reinterpret_cast<uint4*>(&lds.kv[wave][1][r * 256 + 16 * (lane & 15)]) = make_uint4(0u, 0u, 0u, 0u);
        wave_lds_sync();
      }
      bf16x8 vf[8];
#pragma unroll
      for (int dt = 0; dt < 8; ++dt) {
        const uint2 v0 = lds_read_tr16(vbuf + (va ^ (dt << 5))), v1 = lds_read_tr16(vbuf + 4096 + (va ^ (dt << 5)));
        vf[dt] = as_bf16x8(make_uint4(v0.x, v0.y, v1.x, v1.y));
      }
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        if (!on[nt]) continue;
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) o[nt][dt] = mfma16x16x32(vf[dt], pb[nt], o[nt][dt]);
      }
      __asm__ __volatile__("s_waitcnt lgkmcnt(0)" ::: "memory");  // V has been read
      if (more) issue_v(j2, x2 & 1);
      x = x2;
      j = j2;
    }
  }

  // ---- 4. the wavefronts' states, 16 columns at a time, through the buffers' space
  float* st_m = reinterpret_cast<float*>(&lds.kv[0][0][0]);  // [waves][16]
  float* st_l = st_m + kTaWaves * 16;                        // [waves][16]
  float* st_o = st_l + kTaWaves * 16;                        // [waves][16][kTaPitch]
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    __syncthreads();
    float l = l_run[nt];
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    if (grp == 0) {
      st_m[wave * 16 + hh] = m_run[nt];
      st_l[wave * 16 + hh] = l;
    }
#pragma unroll
    for (int dt = 0; dt < 8; ++dt)
      *reinterpret_cast<f32x4*>(&st_o[(wave * 16 + hh) * kTaPitch + 16 * dt + 4 * grp]) = o[nt][dt];
    __syncthreads();
    const int cl = tid >> 5, d = 4 * (tid & 31), c = c0 + 16 * nt + cl;  // 16 columns x 32 quads of dims
    if (c < n_cols) {
      float m = -INFINITY;
#pragma unroll
      for (int w = 0; w < kTaWaves; ++w) m = fmaxf(m, st_m[w * 16 + cl]);
      float den = 0.f;
      f32x4 num = f32x4{0.f, 0.f, 0.f, 0.f};
      if (m != -INFINITY) {
#pragma unroll
        for (int w = 0; w < kTaWaves; ++w) {
          const float sc = __builtin_amdgcn_exp2f(st_m[w * 16 + cl] - m);  // 0 for a wavefront without a score
          den = fmaf(st_l[w * 16 + cl], sc, den);
          num += *reinterpret_cast<const f32x4*>(&st_o[(w * 16 + cl) * kTaPitch + d]) * sc;
        }
      }
      const int64_t row = (bm * G + c % G) * n + c / G;
      if (ns == 1) {
        const float inv = den > 0.f ? 1.f / den : 0.f;
        uint2 w;
        w.x = (uint32_t)f32_to_bf16(num[0] * inv) | ((uint32_t)f32_to_bf16(num[1] * inv) << 16);
        w.y = (uint32_t)f32_to_bf16(num[2] * inv) | ((uint32_t)f32_to_bf16(num[3] * inv) << 16);
        *reinterpret_cast<uint2*>(a.o + row * kHeadDim + d) = w;
      } else {
        float* pp = a.ws + (row * ns + split) * (kHeadDim + 4);
        if (d == 0) *reinterpret_cast<float2*>(pp) = make_float2(m, den);
        *reinterpret_cast<f32x4*>(pp + 4 + d) = num;
      }
    }
  }
}

// Merge the splits' partials of one (node, query head): one wavefront, two head dims per lane, up to 8
// splits requested at once.
__global__ __launch_bounds__(kCombineThreads) void tree_combine_kernel(TreeAttnArgs a, int64_t n_rows) {
  const int lane = threadIdx.x & 63;
  const int64_t row = (int64_t)blockIdx.x * (kCombineThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (row >= n_rows) return;
  constexpr int kStride = kHeadDim + 4;
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
    if (top == -INFINITY) continue;
    const float keep = __builtin_amdgcn_exp2f(m - top);
    l *= keep;
    o0 *= keep;
    o1 *= keep;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (ml[i].x == -INFINITY) continue;  // a split without a score weighs nothing
      const float w = __builtin_amdgcn_exp2f(ml[i].x - top);
      l = fmaf(ml[i].y, w, l);
      o0 = fmaf(po[i].x, w, o0);
      o1 = fmaf(po[i].y, w, o1);
    }
    m = top;
  }
  const float inv = l > 0.f ? 1.f / l : 0.f;
  reinterpret_cast<uint32_t*>(a.o + row * kHeadDim)[lane] = (uint32_t)f32_to_bf16(o0 * inv) | ((uint32_t)f32_to_bf16(o1 * inv) << 16);
}

template <int NT>
hipError_t launch_tiles(const TreeAttnArgs& a, hipStream_t stream) {
  const int groups = a.tb.batch * a.n_kv_heads, units = groups * a.n_splits;
  const int n_tiles = (a.tb.n * a.group_size + 16 * NT - 1) / (16 * NT);
  hipLaunchKernelGGL(tree_attn_kernel<NT>, dim3((unsigned)((units + 7) / 8 * 8 * n_tiles)), dim3(kTaThreads), 0, stream, a,
                     n_tiles, groups);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_tree_attn(const TreeAttnArgs& a, hipStream_t stream) {
  const int nt = tree_attn_tiles(a.tb.n, a.group_size);
  const hipError_t e = nt == 1   ? launch_tiles<1>(a, stream)
                       : nt == 2 ? launch_tiles<2>(a, stream)
                                 : launch_tiles<4>(a, stream);
  if (e != hipSuccess || a.n_splits == 1) return e;
  const int64_t rows = (int64_t)a.tb.batch * a.n_kv_heads * a.group_size * a.tb.n;
  hipLaunchKernelGGL(tree_combine_kernel, dim3((unsigned)((rows + 3) / 4)), dim3(kCombineThreads), 0, stream, a, rows);
  return hipGetLastError();
}

}  // namespace sparda
