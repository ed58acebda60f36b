// paged_append.hip -- new tokens into the pages of a layer (paper Alg. 2's append), their keys turned to their positions
// on the way, the compressed keys of the windows that they complete (Sec. 3, Eq. 2), and the tokens' queries and Forecast
// rows turned to the same positions.
//
// The first workgroups take a (sequence, block of 64 positions, KV head) each: eight lanes per row turn the block's new
// keys, store them, and keep them in LDS where a window ends in the block, together with the window's older keys.
// Up to 16 rows before the block belong to its windows on the (32, 16) grid: cached ones are read, new ones turned
// again, so no workgroup waits for another.  The others turn q and f, eight lanes per row.
//
// A window's mean has the bits of compress_kernel (compress.hip): the float64 sums run in its order, rows r + 16 x
// first, then over r.
//
// What bounds it: for a token per sequence the chain length -> page -> rows -> stores (5.6 us for one sequence, 6.0 for
// 32); for prompts the memory's rate (13289 tokens of 56 heads, 381 MB: 71 us, 5.4 TB/s).  Of those the angles, which every
// KV head forms again, are 4 us, the windows 5.
#include "rotary.hpp"

namespace sparda {

namespace {

constexpr int kRowsBefore = 16;  // of a block that its windows reach back

__device__ __forceinline__ int new_tokens(const PagedAppendArgs& a, int b, int64_t t0) {
  if (t0 < 0) return 0;
  int64_t n = a.n_new ? a.n_new[b] : a.n_max;
  n = n < 0 ? 0 : n > a.n_max ? a.n_max : n;
  const int64_t room = a.t_cap - t0;
  return (int)(n < room ? n : room > 0 ? room : 0);
}

__device__ __forceinline__ const uint16_t* row_of(const Rows& r, int64_t b, int64_t h, int64_t t) {
  return static_cast<const uint16_t*>(r.data) + b * r.ld_batch + h * r.ld_head + t * r.ld_token;
}

template <int L>  // tokens of a window; its stride is 64 with L = 64, else 16
__device__ void append_block(const PagedAppendArgs& a, char* lds, int64_t unit, int slices) {
  constexpr int S = L == 64 ? 64 : 16, kBefore = L - S;
  const int tid = threadIdx.x, c = tid & 7, g = tid >> 3;
  Slot<8> slot(a.rope, c);
  const int h = (int)(unit % a.n_kv_heads);
  const int64_t rest = unit / a.n_kv_heads;
  const int b = (int)(rest / slices);
  const int64_t t0 = a.t_ctx[b];
  const int n = new_tokens(a, b, t0);
  const int64_t t1 = t0 + n;
  if (rest % slices == 0 && h == 0 && tid == 0) a.t_new[b] = (int32_t)t1;
  const int64_t base = (t0 / 64 + rest % slices) * 64;  // the block's first position
  if (n == 0 || base >= t1) return;
  const int64_t end = base + 64 < t1 ? base + 64 : t1;
  const int64_t from = base > t0 ? base : t0;
  const int32_t* table = a.pg.table + b * a.pg.table_ld;
  // windows that end in (from, end]: ends first_end, first_end + S, ..
  int64_t first_end = (from / S + 1) * S;
  if (first_end < L) first_end = L;
  const bool windows = a.pg.kc && first_end <= end;
  const int64_t low = windows ? first_end - L : from;  // the first key that a window needs
  // the rows of a thread, their loads under way together
  constexpr int kRows = (64 + kBefore + 31) / 32;
  uint4 ka[kRows], kb[kRows], va[kRows], vb[kRows];
  int32_t page[kRows];
  bool used[kRows];
#pragma unroll
  for (int x = 0; x < kRows; ++x) {
    const int64_t tok = base - kBefore + g + 32 * x;
    used[x] = g + 32 * x < 64 + kBefore && tok >= low && tok < end;
    page[x] = used[x] ? page_of(a.pg, table, tok) : -1;
    ka[x] = kb[x] = va[x] = vb[x] = make_uint4(0u, 0u, 0u, 0u);
    if (used[x] && tok >= t0) {
      const uint16_t* src = row_of(a.k_new, b, h, tok - t0);
      ka[x] = ld16_nt(src + 8 * slot.a);
      kb[x] = ld16_nt(src + 8 * slot.b);
      if (tok >= base) {
        const uint16_t* vs = row_of(a.v_new, b, h, tok - t0);
        va[x] = ld16_nt(vs + 8 * c);
        vb[x] = ld16_nt(vs + 8 * c + 64);
      }
    }
  }
#pragma unroll
  for (int x = 0; x < kRows; ++x) {
    const int rr = g + 32 * x;
    const int64_t tok = base - kBefore + rr;
    if (!used[x]) continue;
    if (tok >= t0) {
      slot.angles(a.rope, tok, 1.f);
      turn_pieces(a.rope, slot, ka[x], kb[x]);
      if (tok >= base && page[x] >= 0) {
        const int64_t at = token_at(a.pg, page[x], h, tok);
        *reinterpret_cast<uint4*>(a.pg.k + at + 8 * slot.a) = ka[x];
        *reinterpret_cast<uint4*>(a.pg.k + at + 8 * slot.b) = kb[x];
        *reinterpret_cast<uint4*>(a.pg.v + at + 8 * c) = va[x];
        *reinterpret_cast<uint4*>(a.pg.v + at + 8 * c + 64) = vb[x];
      }
    } else if (page[x] >= 0) {
      const uint16_t* src = a.pg.k + token_at(a.pg, page[x], h, tok);
      ka[x] = ld16(src + 8 * slot.a);
      kb[x] = ld16(src + 8 * slot.b);
    }
    *reinterpret_cast<uint4*>(lds + rr * 256 + 16 * slot.a) = ka[x];
    *reinterpret_cast<uint4*>(lds + rr * 256 + 16 * slot.b) = kb[x];
  }
  if (!windows) return;
  __syncthreads();
  // a wavefront per window (at most four end in a block), two elements per lane
  const int n_win = (int)((end - first_end) / S) + 1, w = tid >> 6, d = 2 * (tid & 63);
  if (w >= n_win) return;
  const int64_t w_begin = first_end + w * S - L;
  const int32_t at = page_of(a.pg, table, w_begin);
  if (at < 0 || (L == 32 && page_of(a.pg, table, w_begin + 16) < 0)) return;
  const char* rows = lds + (w_begin - (base - kBefore)) * 256 + 2 * d;
  double s0 = 0.0, s1 = 0.0;
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    double p0 = 0.0, p1 = 0.0;
#pragma unroll
    for (int x = 0; x < L / 16; ++x) {
      const uint32_t y = *reinterpret_cast<const uint32_t*>(rows + (r + 16 * x) * 256);
      p0 += bf16lo(y);
      p1 += bf16hi(y);
    }
    s0 += p0;
    s1 += p1;
  }
  *reinterpret_cast<uint32_t*>(a.pg.kc + key_at(a.pg, at, a.n_kv_heads, h, w_begin, L == 64 ? 6 : 4) + d) =
      f64_to_bf16(s0 * (1.0 / L)) | (uint32_t)f64_to_bf16(s1 * (1.0 / L)) << 16;
}

// Rows of q (heads [0, Hq)) and f (the Hkv heads behind them) of one token, eight lanes each.
__device__ void append_turn(const PagedAppendArgs& a, int64_t grp, int64_t n_groups, int heads) {
  if (grp >= n_groups) return;
  const int c = threadIdx.x & 7;
  Slot<8> slot(a.rope, c);
  const int hq = a.q.data ? a.n_kv_heads * a.group_size : 0, hf = a.f.data ? a.n_kv_heads : 0;
  const int64_t tokens = (int64_t)a.batch * a.n_max;
  const int64_t tok = grp % tokens;
  const int h0 = (int)(grp / tokens) * heads, h1 = min(h0 + heads, hq + hf);
  const int b = (int)(tok / a.n_max), j = (int)(tok % a.n_max);
  const int64_t t0 = a.t_ctx[b];
  if (j >= new_tokens(a, b, t0)) return;
  slot.angles(a.rope, t0 + j, 1.f);
  // the loads of four heads under way
  for (int h = h0; h < h1; h += 4) {
    uint4 wa[4], wb[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (h + e >= h1) break;
      const uint16_t* x = h + e < hq ? row_of(a.q, b, h + e, j) : row_of(a.f, b, h + e - hq, j);
      wa[e] = ld16_nt(x + 8 * slot.a);
      wb[e] = ld16_nt(x + 8 * slot.b);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (h + e >= h1) break;
      uint16_t* y = const_cast<uint16_t*>(h + e < hq ? row_of(a.q_out, b, h + e, j) : row_of(a.f_out, b, h + e - hq, j));
      turn_pieces(a.rope, slot, wa[e], wb[e]);
      *reinterpret_cast<uint4*>(y + 8 * slot.a) = wa[e];
      *reinterpret_cast<uint4*>(y + 8 * slot.b) = wb[e];
    }
  }
}

template <int L>
__global__ __launch_bounds__(256) void paged_append_kernel(PagedAppendArgs a, int64_t kv_units, int slices, int64_t n_groups,
                                                           int heads) {
  __shared__ __align__(16) char lds[(64 + (L == 64 ? 0 : kRowsBefore)) * 256];
  if ((int64_t)blockIdx.x < kv_units)
    append_block<L>(a, lds, blockIdx.x, slices);
  else
    append_turn(a, ((int64_t)blockIdx.x - kv_units) * 32 + (threadIdx.x >> 3), n_groups, heads);
}

}  // namespace

hipError_t launch_paged_append(const PagedAppendArgs& a, hipStream_t stream) {
  const int slices = (int)(((int64_t)a.n_max + 62) / 64) + 1;  // blocks that n_max tokens touch at most
  const int64_t kv_units = (int64_t)a.batch * a.n_kv_heads * slices;
  const int n_heads = (a.q.data ? a.n_kv_heads * a.group_size : 0) + (a.f.data ? a.n_kv_heads : 0);
  const int64_t tokens = (int64_t)a.batch * a.n_max;
  const int64_t heads = n_heads ? rotary_heads(tokens * n_heads, n_heads) : 1;
  const int64_t groups = n_heads ? tokens * ((n_heads + heads - 1) / heads) : 0;
  const dim3 grid((unsigned)(kv_units + (groups + 31) / 32)), block(256);
  if (a.grid.l == 64)
    hipLaunchKernelGGL(paged_append_kernel<64>, grid, block, 0, stream, a, kv_units, slices, groups, (int)heads);
  else
    hipLaunchKernelGGL(paged_append_kernel<32>, grid, block, 0, stream, a, kv_units, slices, groups, (int)heads);
  return hipGetLastError();
}

}  // namespace sparda
