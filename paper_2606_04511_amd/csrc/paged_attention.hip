// paged_attention.hip -- attention of every sequence's newest token over the tokens of its listed blocks, or over its whole
// context, for sequences of different lengths whose K and V lie in pages (paper Sec. 4.1, Eq. 5).
//
// The work is a line of units of 32 tokens, row after row (a row is a sequence's KV head with its G query heads), cut into
// equal pieces, one per wavefront, whatever the lengths are.  A wavefront goes over its piece once with a running maximum
// and sum per head; a piece that holds a whole row writes its output, any other leaves a partial result per row, which the
// eight wavefronts of a workgroup join in LDS where one row fills the workgroup, and paged_join_kernel joins the rest.
//
// A unit is two slices of 16 tokens, the smallest page.  S^T = K Q^T on the matrix cores with 16 tokens as rows and the
// heads as columns: K goes through 8 KiB of the wavefront's LDS (whole rows in, fragments of 16 bytes out, swizzled).
// A lane then holds 8 tokens' scores of one head, which is the B operand of O^T += V^T P^T when the lane's sixteen
// loads those 8 tokens of V, 16 bytes (8 elements) of each; the 8 x 8 corner is turned in registers and element j of every
// lane's eight is the j-th A operand, 16 rows of it: lane (g, c) ends with elements 32 g .. 32 g + 31 of head c.
#include <type_traits>

#include "device_util.hpp"
#include "launch.hpp"
#include "paged.hpp"

namespace sparda {

namespace {

constexpr int kThreads = kPagedWaves * 64;

struct Line {        // a workgroup's view of the line of units
  int64_t total;     // units
  int64_t piece;     // units of a wavefront
};

// A row's place on the line.
struct RowAt {
  int b, h;
  int64_t t;         // tokens of the sequence
  int64_t u0, units; // its first unit on the line, its units
};

__device__ __forceinline__ int64_t attn_context(const PagedAttnArgs& a, int b) {
  const int64_t t = a.t_ctx[b];
  return t > a.t_max ? a.t_max : t;
}
__device__ __forceinline__ int64_t dense_units(int64_t t) { return t > 0 ? (t + 31) >> 5 : 0; }

// Units per KV head of the sequences before each thread's, and of all (a thread has `per` consecutive sequences); the
// starts go to pre[0 .. kThreads).  Every thread of the workgroup must call it.
template <int kT>
__device__ __forceinline__ int64_t scan_lengths(const PagedAttnArgs& a, int per, int64_t* pre, int64_t* sums) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int64_t mine = 0;
  for (int i = 0; i < per; ++i) {
    const int b = tid * per + i;
    if (b < a.batch) mine += dense_units(attn_context(a, b));
  }
  int64_t incl = mine;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t y = __shfl_up((long long)incl, d, 64);
    if (lane >= d) incl += y;
  }
  if (lane == 63) sums[wave] = incl;
  __syncthreads();
  int64_t before = 0, total = 0;
  for (int w = 0; w < kT / 64; ++w) {
    if (w < wave) before += sums[w];
    total += sums[w];
  }
  pre[tid] = before + incl - mine;
  __syncthreads();
  return total;
}

// The row that holds unit u (u < total) of a dense call's line.
template <int kT>
__device__ __forceinline__ RowAt dense_row(const PagedAttnArgs& a, int per, const int64_t* pre, int64_t u) {
  const int lane = threadIdx.x & 63;
  int n = 0;  // starts at or before u: the last of them holds it
#pragma unroll
  for (int i = 0; i < kT / 64; ++i) n += (int)__popcll(__ballot(pre[64 * i + lane] * a.n_kv_heads <= u));
  int b = (n - 1) * per;
  int64_t at = pre[n - 1] * a.n_kv_heads;
  for (;; ++b) {
    const int64_t t = attn_context(a, b), units = dense_units(t);
    if (u < at + units * a.n_kv_heads || b + 1 >= a.batch) {
      const int h = units > 0 ? (int)((u - at) / units) : 0;
      return {b, h, t, at + h * units, units};
    }
    at += units * a.n_kv_heads;
  }
}
// The next row that has units.
__device__ __forceinline__ void next_dense_row(const PagedAttnArgs& a, RowAt* r) {
  r->u0 += r->units;
  if (++r->h < a.n_kv_heads) return;
  r->h = 0;
  while (++r->b < a.batch) {
    r->t = attn_context(a, r->b);
    r->units = dense_units(r->t);
    if (r->units > 0) return;
  }
  r->units = (int64_t)1 << 60;  // past the line
}

__device__ __forceinline__ RowAt sparse_row(const PagedAttnArgs& a, int64_t row_units, int64_t u) {
  const int64_t row = u / row_units;
  const int b = (int)(row / a.n_kv_heads), h = (int)(row % a.n_kv_heads);
  return {b, h, attn_context(a, b), row * row_units, row_units};
}

// Does the piece of workgroup [w0, w1) lie in one row?  Then its wavefronts join in LDS.
__device__ __forceinline__ bool shares_row(const RowAt& r, int64_t w0, int64_t w1) {
  return r.u0 <= w0 && w1 <= r.u0 + r.units;
}

// Partial result `slot` of head i.
__device__ __forceinline__ float* partial(const PagedAttnArgs& a, int64_t slot, int head) {
  return a.ws + (slot * a.group_size + head) * kPartFloats;
}

// A wavefront's running softmax: lane (g, c) holds elements 32 g + 8 r + j of head c in acc[j][r], the denominators of its
// own tokens in l (summed over g at the end), the reference m of head c.
struct Running {
  f32x4 acc[8];
  float m, l;
};

// The wavefront's units [u0, u1) of row r (counted within the row).
template <bool kSparse>
__device__ __forceinline__ void attend(const PagedAttnArgs& a, const RowAt& r, int64_t u0, int64_t u1, char* kbuf, Running* run) {
  const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
#pragma unroll
  for (int j = 0; j < 8; ++j) run->acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
  run->m = -INFINITY;
  run->l = 0.f;
  if (r.t <= 0) return;
  const int64_t row = (int64_t)r.b * a.n_kv_heads + r.h;
  const int32_t* table = a.pg.table + r.b * a.pg.table_ld;
  bf16x8 qf[4];
  {
    const uint16_t* q = a.q + (row * a.group_size + (c < a.group_size ? c : 0)) * kHeadDim + 8 * g;
#pragma unroll
    for (int s = 0; s < 4; ++s) qf[s] = as_bf16x8(c < a.group_size ? ld16(q + 32 * s) : make_uint4(0u, 0u, 0u, 0u));
  }
  int cnt = 0;
  bool ascending = true;
  const int16_t* sel = nullptr;
  if constexpr (kSparse) {
    sel = a.sel + row * a.k_total;
    cnt = a.cnt[row];
    cnt = cnt < 0 ? 0 : cnt > a.k_total ? a.k_total : cnt;
    // a list that ascends strictly names no block twice
    const int last = (int)min((int64_t)cnt, (u1 + 1) >> 1);
    for (int i0 = 0; i0 < last; i0 += 64) {
      const int i = i0 + lane;
      if (__ballot(i > 0 && i < last && sel[min(i, last - 1)] <= sel[max(min(i, last - 1) - 1, 0)]) != 0ull) ascending = false;
    }
  }
  for (int64_t hb = u0; hb < u1; hb += 32) {
    // lane i: slice i of the next 32 units; lim: its tokens
    int64_t tok = 0, off = 0;
    int lim = 0;
    const int64_t u = hb + (lane >> 1);
    if constexpr (kSparse) {
      const int64_t e = u >> 1;
      if (u < u1 && e < cnt) {
        const int blk = sel[e];
        tok = (int64_t)blk * 64 + ((int)u & 1) * 32 + (lane & 1) * 16;
        if (blk >= 0 && tok < r.t) {
          lim = (int)min(r.t - tok, (int64_t)16);
          if (!ascending)
            for (int64_t x = 0; x < e; ++x)
              if (sel[x] == blk) lim = 0;
        }
      }
    } else {
      tok = u * 32 + (lane & 1) * 16;
      if (u < u1 && tok < r.t) lim = (int)min(r.t - tok, (int64_t)16);
    }
    if (lim > 0) {
      const int32_t page = page_of(a.pg, table, tok);
      if (page >= 0)
        off = token_at(a.pg, page, r.h, tok);
      else
        lim = 0;
    }
    // an empty slice of a unit that has tokens reads the other's (it counts for nothing)
    {
      const int64_t other = __shfl_xor((long long)off, 1, 64);
      if (lim == 0) off = other;
    }
    const uint64_t slices = __ballot(lim > 0);
    uint64_t todo = (slices | slices >> 1) & 0x5555555555555555ull;
    if (todo == 0ull) continue;
    const int off_lo = (int)(uint32_t)off, off_hi = (int)(off >> 32);
    auto slice_at = [&](int i) {
      return (int64_t)(((uint64_t)(uint32_t)readlane_i(off_hi, i) << 32) | (uint32_t)readlane_i(off_lo, i));
    };
    uint4 kr[8], vr[8];
    auto load_k = [&](int i) {
      const uint16_t *s0 = a.pg.k + slice_at(i), *s1 = a.pg.k + slice_at(i + 1);
#pragma unroll
      for (int x = 0; x < 4; ++x) kr[x] = ld16_nt(s0 + 8 * lane + 512 * x);
#pragma unroll
      for (int x = 0; x < 4; ++x) kr[4 + x] = ld16_nt(s1 + 8 * lane + 512 * x);
    };
    auto load_v = [&](int i) {
      const uint16_t *s0 = a.pg.v + slice_at(i), *s1 = a.pg.v + slice_at(i + 1);
#pragma unroll
      for (int x = 0; x < 4; ++x) vr[x] = ld16_nt(s0 + 512 * g + 8 * c + 128 * x);
#pragma unroll
      for (int x = 0; x < 4; ++x) vr[4 + x] = ld16_nt(s1 + 512 * g + 8 * c + 128 * x);
    };
    // slices i and i + 1; kMore: the unit at slice `next` follows
    auto unit = [&](int i, int next, auto more) {
      constexpr bool kMore = decltype(more)::value;
      // ---- K through LDS: row 4 x + g (+ 16) holds its piece c at c ^ row
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        const int z = 4 * x + g;
        *reinterpret_cast<uint4*>(kbuf + z * 256 + 16 * (c ^ (z & 15))) = kr[x];
      }
      if constexpr (kMore) load_k(next);
      __builtin_amdgcn_sched_barrier(0);
      f32x4 s[2];
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        s[x] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          const uint4 kw = *reinterpret_cast<const uint4*>(kbuf + (16 * x + c) * 256 + 16 * ((4 * y + g) ^ c));
          s[x] = mfma16x16x32(as_bf16x8(kw), qf[y], s[x]);
        }
      }
      // ---- scores in the exp2 domain; tokens past the limits are replaced, and their V rows too
      const int lim0 = readlane_i(lim, i), lim1 = readlane_i(lim, i + 1);
      float z[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) z[e] = s[e >> 2][e & 3] * a.scale_log2;
      if (lim0 < 16 || lim1 < 16) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const bool in = 4 * g + (e & 3) < (e < 4 ? lim0 : lim1);
          z[e] = in ? z[e] : -INFINITY;
          vr[e].x = in ? vr[e].x : 0u;
          vr[e].y = in ? vr[e].y : 0u;
          vr[e].z = in ? vr[e].z : 0u;
          vr[e].w = in ? vr[e].w : 0u;
        }
      }
      float mx = fmaxf(fmaxf(fmaxf(z[0], z[1]), fmaxf(z[2], z[3])), fmaxf(fmaxf(z[4], z[5]), fmaxf(z[6], z[7])));
      mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
      mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
      // the reference follows the maximum within 2^8
      if (__ballot(mx > run->m + 8.f) != 0ull) {
        const float m = fmaxf(run->m, mx);
        const float f = m == run->m ? 1.f : __builtin_amdgcn_exp2f(run->m - m);
        run->m = m;
        run->l *= f;
#pragma unroll
        for (int j = 0; j < 8; ++j) run->acc[j] *= f;
      }
      const float m = run->m == -INFINITY ? 0.f : run->m;
      uint32_t hi[4], lo[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float p0 = __builtin_amdgcn_exp2f(z[2 * e] - m), p1 = __builtin_amdgcn_exp2f(z[2 * e + 1] - m);
        run->l += p0 + p1;
        hi[e] = pack_bf16(p0, p1);
        lo[e] = pack_bf16(p0 - bf16lo(hi[e]), p1 - bf16hi(hi[e]));
      }
      const bf16x8 ph = as_bf16x8(make_uint4(hi[0], hi[1], hi[2], hi[3]));
      const bf16x8 pl = as_bf16x8(make_uint4(lo[0], lo[1], lo[2], lo[3]));
      // ---- the lane's 8 x 8 corner of V: element j of the eight tokens
      uint4 vt[8];
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        auto part = [&](int e) { return d == 0 ? vr[e].x : d == 1 ? vr[e].y : d == 2 ? vr[e].z : vr[e].w; };
        vt[2 * d] = make_uint4(__builtin_amdgcn_perm(part(1), part(0), 0x05040100u), __builtin_amdgcn_perm(part(3), part(2), 0x05040100u),
                               __builtin_amdgcn_perm(part(5), part(4), 0x05040100u), __builtin_amdgcn_perm(part(7), part(6), 0x05040100u));
        vt[2 * d + 1] = make_uint4(__builtin_amdgcn_perm(part(1), part(0), 0x07060302u), __builtin_amdgcn_perm(part(3), part(2), 0x07060302u),
                                   __builtin_amdgcn_perm(part(5), part(4), 0x07060302u), __builtin_amdgcn_perm(part(7), part(6), 0x07060302u));
      }
      if constexpr (kMore) load_v(next);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        run->acc[j] = mfma16x16x32(as_bf16x8(vt[j]), ph, run->acc[j]);
        run->acc[j] = mfma16x16x32(as_bf16x8(vt[j]), pl, run->acc[j]);
      }
    };
    int i = (int)__builtin_ctzll(todo);
    todo &= todo - 1;
    load_k(i);
    load_v(i);
    while (todo != 0ull) {
      const int next = (int)__builtin_ctzll(todo);
      todo &= todo - 1;
      unit(i, next, std::true_type{});
      i = next;
    }
    unit(i, 0, std::false_type{});
  }
  run->l += __shfl_xor(run->l, 16, 64);
  run->l += __shfl_xor(run->l, 32, 64);
}

// Elements 32 g .. 32 g + 31 of head c, divided by the denominator.
__device__ __forceinline__ void write_row(const PagedAttnArgs& a, const RowAt& r, const Running& run) {
  const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
  if (c >= a.group_size) return;
  uint16_t* o = a.o + (((int64_t)r.b * a.n_kv_heads + r.h) * a.group_size + c) * kHeadDim + 32 * g;
  const float inv = run.l == 0.f ? 0.f : 1.f / run.l;
#pragma unroll
  for (int x = 0; x < 4; ++x) {
    uint4 w;
    w.x = pack_bf16(run.acc[0][x] * inv, run.acc[1][x] * inv);
    w.y = pack_bf16(run.acc[2][x] * inv, run.acc[3][x] * inv);
    w.z = pack_bf16(run.acc[4][x] * inv, run.acc[5][x] * inv);
    w.w = pack_bf16(run.acc[6][x] * inv, run.acc[7][x] * inv);
    *reinterpret_cast<uint4*>(o + 8 * x) = w;
  }
}

// Head c's 128 sums to dst, its maximum and denominator behind them.
__device__ __forceinline__ void write_partial(float* dst, const Running& run) {
  const int g = (threadIdx.x & 63) >> 4;
#pragma unroll
  for (int x = 0; x < 4; ++x) {
    *reinterpret_cast<f32x4*>(dst + 32 * g + 8 * x) = f32x4{run.acc[0][x], run.acc[1][x], run.acc[2][x], run.acc[3][x]};
    *reinterpret_cast<f32x4*>(dst + 32 * g + 8 * x + 4) = f32x4{run.acc[4][x], run.acc[5][x], run.acc[6][x], run.acc[7][x]};
  }
  if (g == 0) {
    dst[128] = run.m;
    dst[129] = run.l;
  }
}

// Weight of a part whose reference is m in a sum whose reference is the parts' largest.
__device__ __forceinline__ float join_weight(float m, float top) {
  return m == top ? 1.f : __builtin_amdgcn_exp2f(m - top);  // (both -inf: the part is empty, its sums are zero)
}

template <bool kSparse>
__global__ __launch_bounds__(kThreads, 2) void paged_attn_kernel(PagedAttnArgs a, int64_t row_units, int per) {
  __shared__ __align__(16) char kbuf[kPagedWaves][32 * 256];
  __shared__ int64_t pre[kSparse ? 1 : kThreads], sums[kPagedWaves];
  __shared__ float stat[kPagedWaves][16][2];
  const int tid = threadIdx.x, lane = tid & 63, c = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  Line line;
  if constexpr (kSparse) {
    line.total = (int64_t)a.batch * a.n_kv_heads * row_units;
  } else {
    line.total = scan_lengths<kThreads>(a, per, pre, sums) * a.n_kv_heads;
    // rows without tokens are on no piece
    for (int64_t b = blockIdx.x; b < a.batch; b += gridDim.x)
      if (attn_context(a, (int)b) <= 0) {
        uint4* o = reinterpret_cast<uint4*>(a.o + b * a.n_kv_heads * a.group_size * kHeadDim);
        for (int i = tid; i < a.n_kv_heads * a.group_size * (kHeadDim / 8); i += kThreads) o[i] = make_uint4(0u, 0u, 0u, 0u);
      }
  }
  const int64_t pieces = (int64_t)gridDim.x * kPagedWaves;
  line.piece = (line.total + pieces - 1) / pieces;
  const int64_t w0 = (int64_t)blockIdx.x * kPagedWaves * line.piece;
  if (w0 >= line.total) return;
  const int64_t w1 = min(w0 + kPagedWaves * line.piece, line.total);
  const int64_t p0 = w0 + wave * line.piece, p1 = min(p0 + line.piece, line.total);
  Running run;
  RowAt r = kSparse ? sparse_row(a, row_units, w0) : dense_row<kThreads>(a, per, pre, w0);
  if (shares_row(r, w0, w1)) {
    const int64_t u0 = min(p0, w1), u1 = max(p1, u0);  // the last piece may be short, or empty
    attend<kSparse>(a, r, u0 - r.u0, u1 - r.u0, kbuf[wave], &run);
    // ---- the wavefronts' results joined: a head's 128 sums of a wavefront in its K buffer
    float* mine = reinterpret_cast<float*>(kbuf[wave]);
    __builtin_amdgcn_wave_barrier();
    const int g = lane >> 4;
#pragma unroll
    for (int x = 0; x < 4; ++x)
#pragma unroll
      for (int j = 0; j < 8; ++j) mine[c * 128 + 32 * g + 8 * x + j] = run.acc[j][x];
    if (g == 0) {
      stat[wave][c][0] = run.m;
      stat[wave][c][1] = run.l;
    }
    __syncthreads();
    const bool whole = r.u0 == w0 && r.units == w1 - w0;
    for (int i = tid; i < a.group_size * 128; i += kThreads) {
      const int head = i >> 7, d = i & 127;
      float top = -INFINITY;
#pragma unroll
      for (int w = 0; w < kPagedWaves; ++w) top = fmaxf(top, stat[w][head][0]);
      float sum = 0.f, l = 0.f;
#pragma unroll
      for (int w = 0; w < kPagedWaves; ++w) {
        const float f = join_weight(stat[w][head][0], top);
        sum = fmaf(f, reinterpret_cast<const float*>(kbuf[w])[i], sum);
        l = fmaf(f, stat[w][head][1], l);
      }
      if (whole) {
        a.o[(((int64_t)r.b * a.n_kv_heads + r.h) * a.group_size + head) * kHeadDim + d] =
            f32_to_bf16(l == 0.f ? 0.f : sum / l);
      } else {
        float* dst = partial(a, (int64_t)blockIdx.x * kPagedWaves * 2, head);
        dst[d] = sum;
        if (d == 0) {
          dst[128] = top;
          dst[129] = l;
        }
      }
    }
    return;
  }
  if (p0 >= p1) return;
  if constexpr (kSparse)
    r = sparse_row(a, row_units, p0);
  else
    r = dense_row<kThreads>(a, per, pre, p0);
  for (int64_t u = p0; u < p1;) {
    const int64_t end = min(r.u0 + r.units, p1);
    attend<kSparse>(a, r, u - r.u0, end - r.u0, kbuf[wave], &run);
    if (u == r.u0 && end == r.u0 + r.units)
      write_row(a, r, run);
    else if (c < a.group_size)
      write_partial(partial(a, ((int64_t)blockIdx.x * kPagedWaves + wave) * 2 + (u == p0 ? 0 : 1), c), run);
    u = end;
    if (u >= p1) break;
    if constexpr (kSparse)
      r = sparse_row(a, row_units, u);
    else
      next_dense_row(a, &r);
  }
}

// Joins the partial results of a row's head, in the order of the line.  One workgroup per (row, head): its wavefronts
// take the parts in turn, two elements per lane.
template <bool kSparse>
__global__ __launch_bounds__(256) void paged_join_kernel(PagedAttnArgs a, int64_t row_units, int per, int n_wgs) {
  __shared__ int64_t pre[256], sums[4];
  __shared__ float acc[4][128], stat[4][2];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t row = blockIdx.x / a.group_size;
  const int head = (int)(blockIdx.x % a.group_size);
  RowAt r;
  r.b = (int)(row / a.n_kv_heads);
  r.h = (int)(row % a.n_kv_heads);
  int64_t total;
  if constexpr (kSparse) {
    r.u0 = row * row_units;
    r.units = row_units;
    total = (int64_t)a.batch * a.n_kv_heads * row_units;
  } else {
    total = scan_lengths<256>(a, per, pre, sums) * a.n_kv_heads;
    int64_t before = pre[r.b / per];
    for (int b = r.b / per * per; b < r.b; ++b) before += dense_units(attn_context(a, b));
    r.units = dense_units(attn_context(a, r.b));
    r.u0 = before * a.n_kv_heads + r.h * r.units;
    if (r.units == 0) return;
  }
  const int64_t pieces = (int64_t)n_wgs * kPagedWaves, piece = (total + pieces - 1) / pieces, wg = piece * kPagedWaves;
  const int64_t first = r.u0 / piece, last = (r.u0 + r.units - 1) / piece;  // wavefronts that hold a part
  const int64_t g0 = first / kPagedWaves, g1 = last / kPagedWaves;
  auto joined = [&](int64_t x) { return shares_row(r, x * wg, min((x + 1) * wg, total)); };
  if (first == last && !joined(g0)) return;  // written by its wavefront
  if (g0 == g1 && joined(g0) && r.u0 == g0 * wg && r.units == min((g0 + 1) * wg, total) - g0 * wg) return;  // by its workgroup
  float m = -INFINITY, l = 0.f, s0 = 0.f, s1 = 0.f;
  auto take = [&](int64_t slot) {
    const float* src = partial(a, slot, head);
    const float pm = src[128], pl = src[129], x0 = src[2 * lane], x1 = src[2 * lane + 1];
    const float top = fmaxf(m, pm), f = join_weight(m, top), pf = join_weight(pm, top);
    s0 = s0 * f + x0 * pf;
    s1 = s1 * f + x1 * pf;
    l = l * f + pl * pf;
    m = top;
  };
  for (int64_t x = g0 + wave; x <= g1; x += 4) {
    if (joined(x)) {
      take(x * kPagedWaves * 2);
    } else {
      for (int64_t w = max(first, x * kPagedWaves); w <= min(last, x * kPagedWaves + kPagedWaves - 1); ++w)
        take(2 * w + (w * piece >= r.u0 ? 0 : 1));  // slot 0: the part at the piece's beginning
    }
  }
  acc[wave][2 * lane] = s0;
  acc[wave][2 * lane + 1] = s1;
  if (lane == 0) {
    stat[wave][0] = m;
    stat[wave][1] = l;
  }
  __syncthreads();
  if (tid < 128) {
    float top = -INFINITY, sum = 0.f, den = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) top = fmaxf(top, stat[w][0]);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float f = join_weight(stat[w][0], top);
      sum = fmaf(f, acc[w][tid], sum);
      den = fmaf(f, stat[w][1], den);
    }
    a.o[(row * a.group_size + head) * kHeadDim + tid] = f32_to_bf16(den == 0.f ? 0.f : sum / den);
  }
}

}  // namespace

hipError_t launch_paged_attn(const PagedAttnArgs& a, hipStream_t stream) {
  const int64_t rows = (int64_t)a.batch * a.n_kv_heads;
  const bool sparse = a.sel != nullptr;
  const PagedPlan p = paged_attn_plan(rows, a.t_max, a.k_total, sparse);
  const int per = (a.batch + kThreads - 1) / kThreads, join_per = (a.batch + 255) / 256;
  const dim3 grid((unsigned)p.n_wgs), block(kThreads);
  if (sparse)
    hipLaunchKernelGGL(paged_attn_kernel<true>, grid, block, 0, stream, a, p.row_units, per);
  else
    hipLaunchKernelGGL(paged_attn_kernel<false>, grid, block, 0, stream, a, p.row_units, per);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !p.joined) return e;
  const dim3 join_grid((unsigned)(rows * a.group_size));
  if (sparse)
    hipLaunchKernelGGL(paged_join_kernel<true>, join_grid, dim3(256), 0, stream, a, p.row_units, join_per, p.n_wgs);
  else
    hipLaunchKernelGGL(paged_join_kernel<false>, join_grid, dim3(256), 0, stream, a, p.row_units, join_per, p.n_wgs);
  return hipGetLastError();
}

}  // namespace sparda
