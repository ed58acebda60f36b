// paged_attention.hip -- attention of every sequence's newest token over the tokens of its listed blocks, or over its whole
// context, for sequences of different lengths whose K and V lie in pages (paper Sec. 4.1, Eq. 5).
//
// A row is a sequence's KV head with its G query heads; its work is counted in units of 32 tokens.  Where the rows are few
// and about as long, or none is long (paged_attn_plan), a row has its own workgroups, which divide it evenly; where they are
// many and short, a wavefront.  Otherwise the rows lie one behind the other on a line, which is cut into equal pieces, one per
// wavefront, whatever the lengths are; where a workgroup's piece holds long rows, its wavefronts divide each of them instead.
// A wavefront goes over its units once with a running maximum and sum per head; those of a workgroup that share a row join
// their results in LDS.  A row that ends up whole is written; the results of the others go to the workspace and
// paged_join_kernel joins them.
//
// A unit is two slices of 16 tokens, the smallest page.  S^T = K Q^T on the matrix cores with 16 tokens as rows and the
// heads as columns: K goes through 8 KiB of the wavefront's LDS (whole rows in, fragments of 16 bytes out, swizzled).
// A lane then holds 8 tokens' scores of one head, which is the B operand of O^T += V^T P^T when the lane's sixteen
// loads those 8 tokens of V, 16 bytes (8 elements) of each; the 8 x 8 corner is turned in registers and element j of every
// lane's eight is the j-th A operand, 16 rows of it: lane (g, c) ends with elements 32 g .. 32 g + 31 of head c.  The weights
// enter the product as two bf16 numbers, which costs matrix time that is free here (they are busy for less than a tenth).
// The next unit's K and V are under way in registers during a unit's products: 16 KiB per wavefront, 128 KiB per CU.
//
// What bounds it: the memory's rate of block reads.  8 sequences of 18K to 33K tokens, 8 KV heads (839 MB): 128 us, 6.6 TB/s,
// and 5 for the join; 256 rows of 64 blocks (537 MB): 81 us, 6.6 TB/s.  Small calls are chains: length -> page -> K -> V ->
// join in LDS -> second launch, 8.9 us for 8 rows of 4K; a row of a few tokens 4.7.
#include <type_traits>

#include "device_util.hpp"
#include "launch.hpp"
#include "paged.hpp"

namespace sparda {

namespace {

constexpr int kThreads = kPagedWaves * 64;

// A row's place on the line.  A call has fewer than 2^32 units (65535 rows of 65536).
struct RowAt {
  int b, h;
  int64_t t;          // tokens of the sequence
  uint32_t u0, units; // its first unit on the line, its units
  __device__ uint32_t end() const { return u0 + units; }
};

__device__ __forceinline__ int64_t attn_context(const PagedAttnArgs& a, int b) {
  const int64_t t = a.t_ctx[b];
  return t > a.t_max ? a.t_max : t;
}
__device__ __forceinline__ uint32_t units_of(const PagedAttnArgs& a, int64_t t) { return paged_units(t, a.k_total); }

// Where the sequences begin on the line, in units per KV head.  Up to 64 sequences: lane i holds the start
// of sequence i, formed by each wavefront on its own.  More: thread i has `per` consecutive sequences and its start is
// pre[i] in LDS.  Every thread of the workgroup must call it.
struct Starts {
  uint32_t mine;   // per KV head
  uint32_t total;
};
__device__ __forceinline__ Starts scan_lengths(const PagedAttnArgs& a, int per, uint32_t* pre, uint32_t* sums) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  uint32_t mine = 0;
  if (per == 0) {
    mine = lane < a.batch ? units_of(a, attn_context(a, lane)) : 0u;
    const uint32_t incl = (uint32_t)wave_incl_scan_dpp((int)mine);
    return {incl - mine, (uint32_t)readlane_i((int)incl, 63)};
  }
  for (int i = 0; i < per; ++i) {
    const int b = tid * per + i;
    if (b < a.batch) mine += units_of(a, attn_context(a, b));
  }
  const uint32_t incl = (uint32_t)wave_incl_scan_dpp((int)mine);
  if (lane == 63) sums[wave] = incl;
  __syncthreads();
  uint32_t before = 0, total = 0;
#pragma unroll
  for (int w = 0; w < kPagedWaves; ++w) {
    if (w < wave) before += sums[w];
    total += sums[w];
  }
  pre[tid] = before + incl - mine;
  __syncthreads();
  return {before + incl - mine, total};
}

// The row that holds unit u of the line.
__device__ __forceinline__ RowAt line_row(const PagedAttnArgs& a, int per, const Starts& st, const uint32_t* pre, uint32_t u) {
  const int lane = threadIdx.x & 63;
  const uint32_t H = (uint32_t)a.n_kv_heads;
  int b;
  uint32_t at;
  if (per == 0) {  // starts at or before u: the last of them holds it
    b = (int)__popcll(__ballot(lane < a.batch && st.mine * H <= u)) - 1;
    at = (uint32_t)readlane_i((int)st.mine, b) * H;
  } else {
    int n = 0;
#pragma unroll
    for (int i = 0; i < kPagedWaves; ++i) n += (int)__popcll(__ballot(pre[64 * i + lane] * H <= u));
    b = (n - 1) * per;
    at = pre[n - 1] * H;
  }
  for (;; ++b) {
    const int64_t t = attn_context(a, b);
    const uint32_t units = units_of(a, t);
    if (u < at + units * H || b + 1 >= a.batch) {
      const uint32_t h = units > 0 ? (u - at) / units : 0u;
      return {b, (int)h, t, at + h * units, units};
    }
    at += units * H;
  }
}
// The row behind r that has units.
__device__ __forceinline__ RowAt next_row(const PagedAttnArgs& a, RowAt r) {
  r.u0 += r.units;
  if (++r.h < a.n_kv_heads) return r;
  r.h = 0;
  while (++r.b < a.batch) {
    r.t = attn_context(a, r.b);
    r.units = units_of(a, r.t);
    if (r.units > 0) return r;
  }
  r.units = 0;  // past the line
  return r;
}
// The workspace: whether the wavefronts of workgroup i share their rows; where sequence b begins on the line;
// the partial results, two per wavefront.
__device__ __forceinline__ int32_t* shared_flags(const PagedAttnArgs& a) { return reinterpret_cast<int32_t*>(a.ws); }
__device__ __forceinline__ uint32_t* line_starts(const PagedAttnArgs& a) {
  return reinterpret_cast<uint32_t*>(a.ws) + kPagedMaxWgs;
}
__device__ __forceinline__ float* partial(const PagedAttnArgs& a, int64_t slot, int head) {
  return a.ws + paged_parts_at(a.batch) + (slot * a.group_size + head) * kPartFloats;
}

// Units of a wavefront's piece.
__device__ __forceinline__ uint32_t line_piece(uint32_t total, uint32_t n_wgs) {
  return (total + n_wgs * kPagedWaves - 1) / (n_wgs * kPagedWaves);
}

// A wavefront's running softmax: lane (g, c) holds elements 32 g + 8 r + j of head c in acc[j][r], the denominators of its
// own tokens in l (summed over g at the end), the reference m of head c.
struct Running {
  f32x4 acc[8];
  float m, l;
};

// The beginning of a row's list: its length and, in lane i, entry i.  The two loads do not wait for each other (entries
// past the length, which k_total bounds, are not used).
struct Listed {
  int cnt, entry;
};
template <bool kSparse>
__device__ __forceinline__ Listed list_of(const PagedAttnArgs& a, int64_t row) {
  if constexpr (!kSparse) return {0, -1};
  const int lane = threadIdx.x & 63;
  return {a.cnt[row], a.sel[row * a.k_total + min(lane, a.k_total - 1)]};
}

// The wavefront's units [u0, u1) of row r (counted within the row; those of a list are the blocks that it names, in its
// order, each once).  list: 64 block indices of the wavefront's own LDS.
template <bool kSparse>
__device__ __forceinline__ void attend(const PagedAttnArgs& a, const RowAt& r, const Listed& listed, int u0, int u1, char* kbuf,
                                       int16_t* list, Running* run) {
  const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
#pragma unroll
  for (int j = 0; j < 8; ++j) run->acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
  run->m = -INFINITY;
  run->l = 0.f;
  if (u0 >= u1) return;
  const int64_t row = (int64_t)r.b * a.n_kv_heads + r.h;
  const int32_t* table = a.pg.table + r.b * a.pg.table_ld;
  bf16x8 qf[4];
  {
    const uint16_t* q = a.q + (row * a.group_size + (c < a.group_size ? c : 0)) * kHeadDim + 8 * g;
#pragma unroll
    for (int s = 0; s < 4; ++s) qf[s] = as_bf16x8(c < a.group_size ? ld16(q + 32 * s) : make_uint4(0u, 0u, 0u, 0u));
  }
  // Up to 32 units: lane i has slice i of them, from token tok on, lim tokens of it (0: none).
  auto chunk = [&](int64_t tok, int lim) {
    int64_t off = 0;
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
    if (todo == 0ull) return;
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
      wave_lds_order();  // other lanes' pieces are read
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
      wave_lds_order();  // before the next unit's stores
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
  };
  if constexpr (!kSparse) {
    for (int hb = u0; hb < u1; hb += 32) {
      const int u = hb + (lane >> 1);
      const int64_t tok = (int64_t)u * 32 + (lane & 1) * 16, left = r.t - tok;
      chunk(tok, u < u1 && left > 0 ? (int)(left < 16 ? left : 16) : 0);
    }
  } else {
    const int16_t* sel = a.sel + row * a.k_total;
    const int cnt = min(listed.cnt, a.k_total);
    bool ascending = true;  // so far: a list that ascends strictly names no block twice
    int before = 0;         // blocks that the entries before i0 name
    int entry = listed.entry, last_entry = -1;
    for (int i0 = 0; i0 < cnt && 2 * before < u1; i0 += 64) {
      const int i = i0 + lane;
      if (i0 > 0) entry = sel[min(i, cnt - 1)];
      const int blk = i < cnt ? entry : -1;
      bool in = blk >= 0 && (int64_t)blk * 64 < r.t;
      int prev = __shfl_up(entry, 1, 64);
      if (lane == 0) prev = last_entry;
      last_entry = __shfl(entry, 63, 64);
      if (__ballot(i > 0 && i < cnt && prev >= blk) != 0ull) ascending = false;
      // elsewhere every entry is compared with those before it, 64 at a time through LDS (a row of 64 blocks in descending
      // order 11.0 us, ascending 9.7; 1024 blocks 218 and 17)
      if (!ascending) {
        for (int x0 = 0; x0 <= i0; x0 += 64) {
          list[lane] = (int16_t)(x0 < i0 ? sel[x0 + lane] : blk);
          wave_lds_sync();
          const int n = min(i - x0, 64);
#pragma unroll 1
          for (int x = 0; x < 64; x += 8) {
            const uint4 w = *reinterpret_cast<const uint4*>(list + x);
            const uint32_t y[4] = {w.x, w.y, w.z, w.w};
            uint32_t same = 0;  // bit e: entry x0 + x + e is the block
#pragma unroll
            for (int e = 0; e < 8; ++e) same |= (int)(int16_t)(y[e >> 1] >> 16 * (e & 1)) == blk ? 1u << e : 0u;
            if (x < n && (same & ((n - x < 8 ? 1u << (n - x) : 256u) - 1u)) != 0u) in = false;
          }
          wave_lds_sync();
        }
      }
      const uint64_t named = __ballot(in);
      const int n = (int)__popcll(named);
      if (2 * (before + n) > u0) {
        if (in) list[mbcnt64(named)] = (int16_t)blk;
        wave_lds_sync();
        const int first = max((u0 >> 1) - before, 0), last = min(((u1 + 1) >> 1) - before, n);
        for (int c0 = first; c0 < last; c0 += 16) {
          const int e = c0 + (lane >> 2), u = 2 * (before + e) + ((lane >> 1) & 1);
          int64_t tok = 0, left = 0;
          if (e < last && u >= u0 && u < u1) {
            tok = (int64_t)list[e] * 64 + (lane & 3) * 16;
            left = r.t - tok;
          }
          chunk(tok, left > 0 ? (int)(left < 16 ? left : 16) : 0);
        }
        wave_lds_sync();
      }
      before += n;
    }
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

// The wavefronts' results of a workgroup that share row r, joined (a head's 128 sums of a wavefront in its K buffer, 16
// bytes at a time; piece x of head c lies at x ^ 2 c, free of bank conflicts): to the output, or to partial result `slot`.
// Every thread of the workgroup must call it.
__device__ __forceinline__ void join_waves(const PagedAttnArgs& a, const RowAt& r, const Running& run, char (*kbuf)[32 * 256],
                                           float (*stat)[16][2], bool whole, int64_t slot) {
  const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  char* mine = kbuf[wave] + c * 512;
  wave_lds_order();
#pragma unroll
  for (int x = 0; x < 4; ++x) {
    *reinterpret_cast<f32x4*>(mine + 16 * ((8 * g + 2 * x) ^ (2 * c))) = f32x4{run.acc[0][x], run.acc[1][x], run.acc[2][x], run.acc[3][x]};
    *reinterpret_cast<f32x4*>(mine + 16 * ((8 * g + 2 * x + 1) ^ (2 * c))) = f32x4{run.acc[4][x], run.acc[5][x], run.acc[6][x], run.acc[7][x]};
  }
  if (g == 0) {
    stat[wave][c][0] = run.m;
    stat[wave][c][1] = run.l;
  }
  __syncthreads();
  for (int i = tid; i < a.group_size * 32; i += kThreads) {
    const int head = i >> 5, x = i & 31;
    float top = -INFINITY, l = 0.f;
#pragma unroll
    for (int w = 0; w < kPagedWaves; ++w) top = fmaxf(top, stat[w][head][0]);
    f32x4 sum = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kPagedWaves; ++w) {
      const float f = join_weight(stat[w][head][0], top);
      l = fmaf(f, stat[w][head][1], l);
      const f32x4 y = *reinterpret_cast<const f32x4*>(kbuf[w] + head * 512 + 16 * (x ^ (2 * head)));
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[e] = fmaf(f, y[e], sum[e]);
    }
    if (whole) {
      const float inv = l == 0.f ? 0.f : 1.f / l;
      uint16_t* o = a.o + (((int64_t)r.b * a.n_kv_heads + r.h) * a.group_size + head) * kHeadDim + 4 * x;
      *reinterpret_cast<uint2*>(o) = make_uint2(pack_bf16(sum[0] * inv, sum[1] * inv), pack_bf16(sum[2] * inv, sum[3] * inv));
    } else {
      float* dst = partial(a, slot, head);
      *reinterpret_cast<f32x4*>(dst + 4 * x) = sum;
      if (x == 0) *reinterpret_cast<float2*>(dst + 128) = make_float2(top, l);
    }
  }
}

// Wavefront w's share of n units.
__device__ __forceinline__ void share_of(uint32_t n, int w, int parts, uint32_t* v0, uint32_t* v1) {
  const uint32_t each = (n + parts - 1) / parts;
  *v0 = w * each < n ? w * each : n;
  *v1 = *v0 + each < n ? *v0 + each : n;
}

// n_splits > 0: n_splits workgroups per row; -1: a wavefront per row; 0: the line.
template <bool kSparse>
__global__ __launch_bounds__(kThreads, 2) void paged_attn_kernel(PagedAttnArgs a, int n_splits, int per) {
  __shared__ __align__(16) char kbuf[kPagedWaves][32 * 256];
  __shared__ uint32_t pre[kThreads], sums[kPagedWaves];
  __shared__ float stat[kPagedWaves][16][2];
  __shared__ __align__(16) int16_t lists[kPagedWaves][kSparse ? 64 : 1];
  const int tid = threadIdx.x, lane = tid & 63, c = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  Running run;
  RowAt r;
  uint32_t w0, w1, piece = 0;
  Starts st = {0u, 0u};
  Listed listed = {0, -1};
  if (n_splits < 0) {
    const int64_t row = (int64_t)blockIdx.x * kPagedWaves + wave;
    if (row >= (int64_t)a.batch * a.n_kv_heads) return;
    listed = list_of<kSparse>(a, row);
    r.b = (int)(row / a.n_kv_heads);
    r.h = (int)(row % a.n_kv_heads);
    r.t = attn_context(a, r.b);
    attend<kSparse>(a, r, listed, 0, (int)units_of(a, r.t), kbuf[wave], lists[wave], &run);
    write_row(a, r, run);
    return;
  }
  if (n_splits > 0) {
    const uint32_t row = blockIdx.x / (uint32_t)n_splits, split = blockIdx.x % (uint32_t)n_splits;
    r.b = (int)(row / (uint32_t)a.n_kv_heads);
    r.h = (int)(row % (uint32_t)a.n_kv_heads);
    listed = list_of<kSparse>(a, row);  // (requested beside the length)
    r.t = attn_context(a, r.b);
    r.u0 = 0;
    r.units = units_of(a, r.t);
    // the row's shares are those of its n_splits * 8 wavefronts
    const uint32_t each = (r.units + n_splits * kPagedWaves - 1) / (n_splits * kPagedWaves) * kPagedWaves;
    w0 = split * each < r.units ? split * each : r.units;
    w1 = w0 + each < r.units ? w0 + each : r.units;
  } else {
    st = scan_lengths(a, per, pre, sums);
    const uint32_t total = st.total * (uint32_t)a.n_kv_heads;
    if (blockIdx.x == 0) {  // for the join
      uint32_t* starts = line_starts(a);
      const int n = per == 0 ? 1 : per;
      uint32_t at = st.mine;
      for (int i = 0; i < n; ++i) {
        const int b = tid * n + i;
        if (b >= a.batch || (per == 0 && wave > 0)) break;
        starts[b] = at;
        at += units_of(a, attn_context(a, b));
      }
      if (tid == 0) starts[a.batch] = st.total;
    }
    // rows without tokens are on no piece
    for (int b = blockIdx.x; b < a.batch; b += gridDim.x)
      if (attn_context(a, b) <= 0) {
        uint4* o = reinterpret_cast<uint4*>(a.o + (int64_t)b * a.n_kv_heads * a.group_size * kHeadDim);
        for (int i = tid; i < a.n_kv_heads * a.group_size * (kHeadDim / 8); i += kThreads) o[i] = make_uint4(0u, 0u, 0u, 0u);
      }
    piece = line_piece(total, gridDim.x);
    w0 = blockIdx.x * kPagedWaves * piece;
    if (w0 >= total) return;
    w1 = total - w0 < kPagedWaves * piece ? total : w0 + kPagedWaves * piece;
    r = line_row(a, per, st, pre, w0);
    const RowAt last = r.end() < w1 ? line_row(a, per, st, pre, w1 - 1) : r;
    const uint32_t n_rows = (uint32_t)(last.b - r.b) * (uint32_t)a.n_kv_heads + (uint32_t)(last.h - r.h) + 1;
    const bool share = n_rows <= 2 || (w1 - w0) / 16 >= n_rows;
    if (tid == 0) shared_flags(a)[blockIdx.x] = share ? 1 : 0;
    if (!share) {  // several short rows
      const uint32_t p0 = w0 + wave * piece, p1 = p0 + piece < w1 ? p0 + piece : w1;
      if (p0 >= p1) return;
      r = line_row(a, per, st, pre, p0);
      for (uint32_t u = p0;;) {
        const uint32_t end = r.end() < p1 ? r.end() : p1;
        attend<kSparse>(a, r, list_of<kSparse>(a, (int64_t)r.b * a.n_kv_heads + r.h), (int)(u - r.u0), (int)(end - r.u0), kbuf[wave], lists[wave], &run);
        if (u == r.u0 && end == r.end())
          write_row(a, r, run);
        else if (c < a.group_size)
          write_partial(partial(a, ((int64_t)blockIdx.x * kPagedWaves + wave) * 2 + (u == p0 ? 0 : 1), c), run);
        u = end;
        if (u >= p1) return;
        r = next_row(a, r);
      }
    }
    listed = list_of<kSparse>(a, (int64_t)r.b * a.n_kv_heads + r.h);
  }
  // every row divided by the wavefronts
  for (uint32_t u = w0;;) {
    const uint32_t end = r.end() < w1 ? r.end() : w1;
    uint32_t v0, v1;
    share_of(end - u, wave, kPagedWaves, &v0, &v1);
    attend<kSparse>(a, r, listed, (int)(u - r.u0 + v0), (int)(u - r.u0 + v1), kbuf[wave], lists[wave], &run);
    const bool whole = n_splits > 0 ? n_splits == 1 : u == r.u0 && end == r.end();
    join_waves(a, r, run, kbuf, stat, whole, (int64_t)blockIdx.x * kPagedWaves * 2 + (u == w0 ? 0 : 1));
    u = end;
    if (u >= w1) return;
    r = next_row(a, r);
    listed = list_of<kSparse>(a, (int64_t)r.b * a.n_kv_heads + r.h);
    __syncthreads();  // the results have been read
  }
}

// Joins the partial results of a row's head, in their order: kWaves wavefronts per (row, head), two elements per lane, eight
// results requested at once.
template <int kWaves>
__global__ __launch_bounds__(kWaves == 16 ? 1024 : 256) void paged_join_kernel(PagedAttnArgs a, int n_splits, int n_wgs, int n_pairs) {
  constexpr int kPerWg = kWaves == 1 ? 4 : 1;  // (row, head) pairs of a workgroup
  __shared__ float acc[kWaves][128], stat[kWaves][2];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), part = wave % kWaves;
  const int pair = (int)blockIdx.x * kPerWg + (kWaves == 1 ? wave : 0);
  if (pair >= n_pairs) return;
  const int row = pair / a.group_size, head = pair % a.group_size;
  float m = -INFINITY, l = 0.f, s0 = 0.f, s1 = 0.f;
  auto take8 = [&](auto slot_of, uint32_t valid) {  // results e whose bit is set
    float pm[8], pl[8], x0[8], x1[8], top = m;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (valid >> e & 1u) {
        const float* src = partial(a, slot_of(e), head);
        const float2 x = *reinterpret_cast<const float2*>(src + 2 * lane), y = *reinterpret_cast<const float2*>(src + 128);
        x0[e] = x.x;
        x1[e] = x.y;
        pm[e] = y.x;
        pl[e] = y.y;
      } else {
        x0[e] = x1[e] = pl[e] = 0.f;
        pm[e] = -INFINITY;
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) top = fmaxf(top, pm[e]);
    const float f = join_weight(m, top);
    s0 *= f;
    s1 *= f;
    l *= f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float pf = join_weight(pm[e], top);
      s0 = fmaf(pf, x0[e], s0);
      s1 = fmaf(pf, x1[e], s1);
      l = fmaf(pf, pl[e], l);
    }
    m = top;
  };
  if (n_splits > 0) {
    for (int x = 8 * part; x < n_splits; x += 8 * kWaves)
      take8([&](int e) { return ((int64_t)row * n_splits + x + e) * (kPagedWaves * 2); },
            n_splits - x >= 8 ? 0xffu : (1u << (n_splits - x)) - 1u);
  } else {
    const int b = row / a.n_kv_heads;
    const uint32_t* starts = line_starts(a);
    const uint32_t at = starts[b], units = starts[b + 1] - at, total = starts[a.batch] * (uint32_t)a.n_kv_heads;
    if (units == 0) return;
    const uint32_t u0 = at * (uint32_t)a.n_kv_heads + (uint32_t)(row % a.n_kv_heads) * units, end = u0 + units;
    const uint32_t piece = line_piece(total, n_wgs), wg = piece * kPagedWaves;
    const int g0 = (int)(u0 / wg), g1 = (int)((end - 1) / wg);
    const int32_t* flags = shared_flags(a);
    if (g0 == g1) {  // written by its workgroup, or by one wavefront?
      if (flags[g0] != 0 || u0 / piece == (end - 1) / piece) return;
    }
    for (int x0 = g0 + 8 * part; x0 <= g1; x0 += 8 * kWaves) {
      const int flag = lane < 8 && x0 + lane <= g1 ? flags[x0 + lane] : -1;
      const uint32_t joined = (uint32_t)__ballot(flag == 1), apart = (uint32_t)__ballot(flag == 0);
      // slot 0 holds the result that begins where the piece does
      if (joined)
        take8([&](int e) { return (int64_t)(x0 + e) * (kPagedWaves * 2) + ((uint32_t)(x0 + e) * wg >= u0 ? 0 : 1); }, joined);
      for (uint32_t todo = apart; todo != 0u; todo &= todo - 1u) {
        const int x = x0 + __builtin_ctz(todo);
        uint32_t in = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const uint32_t p0 = (uint32_t)x * wg + e * piece;
          if (p0 < end && p0 + piece > u0) in |= 1u << e;
        }
        take8([&](int e) { return ((int64_t)x * kPagedWaves + e) * 2 + ((uint32_t)x * wg + e * piece >= u0 ? 0 : 1); }, in);
      }
    }
  }
  uint32_t* out = reinterpret_cast<uint32_t*>(a.o + ((int64_t)row * a.group_size + head) * kHeadDim);
  if constexpr (kWaves == 1) {
    const float inv = l == 0.f ? 0.f : 1.f / l;
    out[lane] = pack_bf16(s0 * inv, s1 * inv);
  } else {
    *reinterpret_cast<float2*>(&acc[wave][2 * lane]) = make_float2(s0, s1);
    if (lane == 0) {
      stat[wave][0] = m;
      stat[wave][1] = l;
    }
    __syncthreads();
    if (wave != 0) return;
    float top = -INFINITY, y0 = 0.f, y1 = 0.f, den = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) top = fmaxf(top, stat[w][0]);
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float f = join_weight(stat[w][0], top);
      const float2 x = *reinterpret_cast<const float2*>(&acc[w][2 * lane]);
      y0 = fmaf(f, x.x, y0);
      y1 = fmaf(f, x.y, y1);
      den = fmaf(f, stat[w][1], den);
    }
    const float inv = den == 0.f ? 0.f : 1.f / den;
    out[lane] = pack_bf16(y0 * inv, y1 * inv);
  }
}

}  // namespace

hipError_t launch_paged_attn(const PagedAttnArgs& args, hipStream_t stream) {
  PagedAttnArgs a = args;
  if (!a.sel) a.k_total = 0;
  const PagedPlan p = paged_attn_plan(a.batch, a.n_kv_heads, a.t_max, a.k_total);
  const int per = a.batch <= 64 ? 0 : (a.batch + kThreads - 1) / kThreads;
  const dim3 grid((unsigned)p.n_wgs), block(kThreads);
  if (a.sel)
    hipLaunchKernelGGL(paged_attn_kernel<true>, grid, block, 0, stream, a, p.n_splits, per);
  else
    hipLaunchKernelGGL(paged_attn_kernel<false>, grid, block, 0, stream, a, p.n_splits, per);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !p.joined) return e;
  const int pairs = a.batch * a.n_kv_heads * a.group_size, waves = paged_join_waves(p, a.n_kv_heads, pairs);
  if (waves == 16)
    hipLaunchKernelGGL(paged_join_kernel<16>, dim3((unsigned)pairs), dim3(1024), 0, stream, a, p.n_splits, p.n_wgs, pairs);
  else if (waves == 4)
    hipLaunchKernelGGL(paged_join_kernel<4>, dim3((unsigned)pairs), dim3(256), 0, stream, a, p.n_splits, p.n_wgs, pairs);
  else
    hipLaunchKernelGGL(paged_join_kernel<1>, dim3((unsigned)((pairs + 3) / 4)), dim3(256), 0, stream, a, p.n_splits, p.n_wgs, pairs);
  return hipGetLastError();
}

}  // namespace sparda
