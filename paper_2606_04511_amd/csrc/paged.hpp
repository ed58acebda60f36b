// paged.hpp -- launchers, sizes and device helpers of the rotary positions and the operators over paged
// caches (rotate.hip, paged_append.hip, paged_select.hip, paged_attention.hip; private to the library).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "launch.hpp"

namespace sparda {

struct Rows {  // strided rows of 128 elements (strides in elements)
  void* data;
  int64_t ld_batch, ld_head, ld_token;
};

struct Rope {
  const double* freq;
  int32_t rot_dim;  // 0: nothing turns
  int32_t pairs;    // pair j is (2 j, 2 j + 1), else (j, j + rot_dim / 2)
  float scale;
};

struct RotateArgs {
  Rope rope;
  Rows x, y;
  const int32_t* pos;
  int64_t pos_ld;
  int32_t batch, n_heads;
  int64_t n_tok;
  int32_t bf16, backward;
};

// Where the tokens of a call's sequences lie.
struct Pages {
  const int32_t* table;
  int64_t table_ld, page_ld;
  int32_t n_pages;
  int32_t shift;  // a page holds 2^shift tokens
  uint16_t* k;
  uint16_t* v;
  uint16_t* kc;
};

struct PagedAppendArgs {
  Pages pg;
  Rope rope;
  Rows k_new, v_new, q, q_out, f, f_out;  // data null: absent
  const int32_t* n_new;                   // null: n_max
  const int32_t* t_ctx;
  int32_t* t_new;
  int32_t batch, n_kv_heads, group_size, n_max;
  int64_t t_cap;
  WinGrid grid;
};

struct PagedSelectArgs {
  Pages pg;
  const uint16_t* f;
  const int32_t* t_ctx;
  int64_t t_max;
  int16_t* sel;
  int16_t* cnt;
  float* ws;           // block scores: row stride ws_stride, the first candidate at slot 0
  int64_t ws_stride;
  int32_t batch, n_kv_heads, n_init, n_local, k_total;
  WinGrid grid;
};

struct PagedAttnArgs {
  Pages pg;
  const uint16_t* q;
  const int32_t* t_ctx;
  int64_t t_max;
  const int16_t* sel;  // null: whole contexts
  const int16_t* cnt;
  uint16_t* o;
  float* ws;
  int32_t batch, n_kv_heads, group_size, k_total;
  float scale_log2;
};

inline int64_t paged_select_stride(int64_t t_max, int32_t n_init, int32_t n_local) {
  const int64_t c = (t_max - 1) / 64 - n_local - n_init + 1;
  return c > 0 ? (c + 3) & ~(int64_t)3 : 0;
}
inline size_t paged_select_ws(int64_t rows, int64_t t_max, int32_t n_init, int32_t n_local) {
  return (size_t)rows * (size_t)paged_select_stride(t_max, n_init, n_local) * sizeof(float);
}

// How an attention call is cut.  The work of a row (a sequence's KV head) is counted in units of 32 tokens.  Either every
// row has n_splits workgroups, which divide it evenly; or (n_splits -1) every row has a wavefront; or (0) the rows lie one
// behind the other on a line, which is cut into equal pieces whatever the lengths are, at the price of a scan over the lengths
// and a second launch (about 7 us).
//
// The host knows the longest context only.  A workgroup alone reads about 50 GB/s, 0.33 us per unit: up to 64 units of the
// longest row per workgroup, workgroups per row cost at most 20 us where all other rows are short, and are faster where
// they are not (us, contexts between half of t and t; line and workgroups per row): 32 rows of t = 500 12.1 and 8.1; 256
// rows of 1000 24 and 19; 512 rows of 1000 with 4 heads 42 and 35, with 16 heads 55 and 37; 1600 rows of 1000 113 and 101;
// but 320 rows of 2000 46 and 49, the second round being short.  The rows of one sequence are of the same length and need no
// line.  Nor do lists while most contexts are longer than they are, which the host does not know: up to 128 units per
// workgroup they take none while they fill at most one round of workgroups (256 rows of k blocks; all contexts longer, every
// second one, one: k = 48 69 and 63, 43 and 40, 20 and 33; k = 64 87 and 84, 53 and 52, 21 and 42; beyond, the line costs
// little and saves much: k = 96 130 and 129, 77 and 75, 22 and 60; k = 256 337 and 332, 180 and 186, 28 and 146; k = 1000
// 1270 and 1273, 617 and 701, 58 and 547).
//
// Many short rows have a wavefront each, the more units the more rows there are, up to 16 units (a wavefront alone needs 35
// us for them).  Workgroups per row and a wavefront (us, contexts up to t): 320 rows of t = 60 7.9 and 7.1, of 100 8.3 and
// 10.4; 800 rows of 100 15.8 and 12.7, of 300 24.7 and 27.4; 1600 rows of 100 26 and 14.6, of 300 43 and 34, of 500 61 and
// 54; 3200 rows of 100 40 and 27, of 500 113 and 107.
constexpr int kPagedWaves = 8;    // wavefronts of a workgroup
constexpr int kPagedMaxWgs = 256; // one workgroup per CU
// Units of a row of t tokens, of which a list of k_total blocks (0: no list) may name a part.
__host__ __device__ inline uint32_t paged_units(int64_t t, int32_t k_total) {
  if (t <= 0) return 0;
  if (k_total <= 0) return (uint32_t)((t + 31) >> 5);
  const int64_t blocks = (t + 63) >> 6;
  return 2 * (uint32_t)(blocks < k_total ? blocks : k_total);
}
struct PagedPlan {
  int32_t n_wgs, n_splits;  // n_splits 0: the line, -1: a wavefront per row
  bool joined;  // there may be partial results
};
inline PagedPlan paged_attn_plan(int32_t batch, int32_t n_kv_heads, int64_t t_max, int32_t k_total) {
  const int64_t rows = (int64_t)batch * n_kv_heads, units = paged_units(t_max, k_total);
  int64_t s = rows <= kPagedMaxWgs && units > 16 ? kPagedMaxWgs / rows : 1;
  const int64_t most = (units + kPagedWaves - 1) / kPagedWaves;
  s = s < most ? s : most;
  const bool one_round = rows <= kPagedMaxWgs;
  const int64_t rounds = (rows + kPagedMaxWgs - 1) / kPagedMaxWgs;
  if (units <= (rounds >= 6 ? 16 : rounds >= 4 ? 6 : rounds >= 2 ? 2 : 0))
    return {(int32_t)((rows + kPagedWaves - 1) / kPagedWaves), -1, false};
  if ((one_round && batch == 1) || units <= (one_round && k_total > 0 ? 128 : 64) * s)
    return {(int32_t)(rows * s), (int32_t)s, s > 1};
  const int64_t wgs = (rows * units + kPagedWaves - 1) / kPagedWaves;
  return {(int32_t)(wgs < kPagedMaxWgs ? wgs : kPagedMaxWgs), 0, true};
}
// Wavefronts that join a (row, head) pair's results, eight at a time each.  With workgroups per row it has n_splits of them;
// on the line up to n_wgs / n_kv_heads + 1, since the sequence's other KV heads are as long.  Most rows of a line have few,
// and a call has `pairs` pairs: wavefronts without results cost more than the rounds that a long row saves (us, one, four and
// sixteen wavefronts; 64 sequences with a KV head each, one of them of 131072 tokens, the others of 200: 1 head per group 41,
// 25 and 22, 4 heads 43, 27 and 22, 16 heads 48, 32 and 30; 64 sequences with 4 KV heads of 4 heads 61, 55 and 58; 8 ragged
// sequences with 8 KV heads 129, 131 and 131; 300 with 8 KV heads of 4 heads, 9600 pairs, 79, 86 and 119; 16000 pairs of
// one KV head 59, 53 and 107, 64000 60, 107 and 310).
inline int paged_join_waves(const PagedPlan& p, int32_t n_kv_heads, int64_t pairs) {
  const int results = p.n_splits > 0 ? p.n_splits : p.n_wgs / n_kv_heads;
  if (results > 64 && pairs <= 1024) return 16;
  return results > (p.n_splits > 0 ? 8 : 32) && pairs <= 16384 ? 4 : 1;
}
// Two partial results per wavefront, each per head: 128 sums, the maximum and the denominator (4 floats apart).
constexpr int kPartFloats = 132;
// Before them a flag per workgroup and the starts of the sequences: 4 bytes each.
__host__ __device__ inline int64_t paged_parts_at(int64_t batch) { return (kPagedMaxWgs + batch + 1 + 63) & ~(int64_t)63; }
inline size_t paged_attn_ws(int64_t batch, int32_t group_size) {
  return ((size_t)paged_parts_at(batch) + (size_t)kPagedMaxWgs * kPagedWaves * 2 * (size_t)group_size * kPartFloats) * sizeof(float);
}

hipError_t launch_rotate(const RotateArgs& a, hipStream_t stream);
hipError_t launch_paged_append(const PagedAppendArgs& a, hipStream_t stream);
hipError_t launch_paged_select(const PagedSelectArgs& a, hipStream_t stream);
hipError_t launch_paged_attn(const PagedAttnArgs& a, hipStream_t stream);

// ---- device helpers ------------------------------------------------------------------------------

// The page that holds token `tok` of the sequence whose table row is `row`; -1: none.
__device__ __forceinline__ int32_t page_of(const Pages& pg, const int32_t* row, int64_t tok) {
  const int32_t p = row[tok >> pg.shift];
  return (uint32_t)p < (uint32_t)pg.n_pages ? p : -1;
}
// First element of token `tok` of KV head h in page p, of k and of v.
__device__ __forceinline__ int64_t token_at(const Pages& pg, int32_t p, int h, int64_t tok) {
  return p * pg.page_ld + (((int64_t)h << pg.shift) + (tok & (((int64_t)1 << pg.shift) - 1))) * 128;
}
// First element of the compressed key of the window that begins at token `tok`.
__device__ __forceinline__ int64_t key_at(const Pages& pg, int32_t p, int n_kv_heads, int h, int64_t tok, int stride_log2) {
  const int64_t slot = (tok & (((int64_t)1 << pg.shift) - 1)) >> stride_log2;
  return ((((int64_t)p * n_kv_heads + h) << (pg.shift - stride_log2)) + slot) * 128;
}

}  // namespace sparda
