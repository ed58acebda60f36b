// paged_abi.cpp -- the extern "C" entry points of rotary positions and paged caches (include/sparda.h).
//
// As in sparda_abi.cpp every argument is checked on the host before any HIP call.  What lives in device memory
// (lengths, tables, positions, block lists) is bounded by the kernels.
#include "sparda.h"

#include <hip/hip_runtime.h>

#include <cmath>
#include <utility>

#include "abi_checks.hpp"
#include "paged.hpp"

using namespace sparda::abi;

namespace {

constexpr int64_t kMaxStride = (int64_t)1 << 40;
constexpr int kDim = 128;

int check_rope(const sparda_rope* r, sparda::Rope* out) {
  *out = {nullptr, 0, 0, 1.f};
  if (!r) return SPARDA_OK;
  if (r->struct_size != sizeof(sparda_rope))
    return fail(SPARDA_ERR_INVALID_ARG, "rope.struct_size is %u, expected %zu", r->struct_size, sizeof(sparda_rope));
  if (r->rot_dim < 0 || r->rot_dim > kDim || r->rot_dim % 2 != 0)
    return fail(SPARDA_ERR_INVALID_ARG, "rot_dim %d is not an even number in [0, 128]", r->rot_dim);
  if (r->rot_dim % 16 != 0) return fail(SPARDA_ERR_UNSUPPORTED, "rot_dim %d is not a multiple of 16", r->rot_dim);
  if (r->layout != SPARDA_ROPE_HALF && r->layout != SPARDA_ROPE_PAIRS)
    return fail(SPARDA_ERR_INVALID_ARG, "rope layout %d", r->layout);
  if (!std::isfinite(r->scale)) return fail(SPARDA_ERR_INVALID_ARG, "rope scale is not finite");
  if (r->rot_dim > 0) {
    const int rc = check_dev(r->freq, "freq", 8);
    if (rc) return rc;
  }
  *out = {r->freq, r->rot_dim, r->layout == SPARDA_ROPE_PAIRS, r->scale};
  return SPARDA_OK;
}

// Rows [nb][nh][nt] of elements of `size` bytes.
int check_rows_of(const sparda_rows* r, const char* name, int64_t nb, int64_t nh, int64_t nt, int size, bool output,
                  sparda::Rows* out) {
  if (!r) return fail(SPARDA_ERR_INVALID_ARG, "%s is null", name);
  const int rc = check_dev(r->data, name, 16);
  if (rc) return rc;
  int64_t ld[3] = {nb > 1 ? r->ld_batch : 0, nh > 1 ? r->ld_head : 0, nt > 1 ? r->ld_token : 0};
  *out = {r->data, ld[0], ld[1], ld[2]};
  int64_t n[3] = {nb, nh, nt};
  for (int i = 0; i < 3; ++i) {
    if (ld[i] < 0 || ld[i] >= kMaxStride) return fail(SPARDA_ERR_INVALID_ARG, "%s: stride %lld", name, (long long)ld[i]);
    if (ld[i] * size % 16 != 0)
      return fail(SPARDA_ERR_INVALID_ARG, "%s: stride %lld is not a multiple of 16 bytes", name, (long long)ld[i]);
  }
  if (!output) return SPARDA_OK;
  // sorted by stride, each clears what the smaller ones span
  for (int i = 0; i < 2; ++i)
    for (int j = 0; j < 2 - i; ++j)
      if (ld[j] > ld[j + 1]) {
        std::swap(ld[j], ld[j + 1]);
        std::swap(n[j], n[j + 1]);
      }
  int64_t span = kDim;
  for (int i = 0; i < 3; ++i) {
    if (n[i] <= 1) continue;
    if (ld[i] < span) return fail(SPARDA_ERR_INVALID_ARG, "%s: its rows overlap", name);
    if (ld[i] > (((int64_t)1 << 62) - span) / n[i]) return fail(SPARDA_ERR_INVALID_ARG, "%s: stride too large", name);
    span += ld[i] * (n[i] - 1);
  }
  return SPARDA_OK;
}

int check_pages(const sparda_shape* s, const sparda_pages* p, bool kv, bool cmp, sparda::Pages* out) {
  if (!p) return fail(SPARDA_ERR_INVALID_ARG, "pages is null");
  if (p->struct_size != sizeof(sparda_pages))
    return fail(SPARDA_ERR_INVALID_ARG, "pages.struct_size is %u, expected %zu", p->struct_size, sizeof(sparda_pages));
  const int32_t P = p->page_size;
  if (P < 1) return fail(SPARDA_ERR_INVALID_ARG, "page_size %d < 1", P);
  if (P < 16 || P > 65536 || (P & (P - 1)) != 0)
    return fail(SPARDA_ERR_UNSUPPORTED, "page_size %d (a power of two in [16, 65536])", P);
  if (p->n_pages < 1 || p->n_pages > 0x7fffffff)
    return fail(SPARDA_ERR_INVALID_ARG, "n_pages %lld", (long long)p->n_pages);
  int rc = check_dev(p->table, "table", 4);
  if (rc) return rc;
  if (p->table_ld < (s->t_cap + P - 1) / P || p->table_ld >= kMaxStride)
    return fail(SPARDA_ERR_INVALID_ARG, "table_ld %lld: a sequence has up to %lld pages", (long long)p->table_ld,
                (long long)((s->t_cap + P - 1) / P));
  if (kv) {
    if ((rc = check_dev(p->k, "pages.k", 16)) || (rc = check_dev(p->v, "pages.v", 16))) return rc;
    if (p->page_ld < (int64_t)s->n_kv_heads * P * kDim || p->page_ld >= kMaxStride || p->page_ld % 8 != 0)
      return fail(SPARDA_ERR_INVALID_ARG, "page_ld %lld: a page is %lld elements, and the stride a multiple of 8",
                  (long long)p->page_ld, (long long)s->n_kv_heads * P * kDim);
  }
  if (cmp) {
    if ((rc = check_dev(p->k_cmp, "pages.k_cmp", 16))) return rc;
    if (P % s->cmp_stride != 0)
      return fail(SPARDA_ERR_UNSUPPORTED, "page_size %d is not a multiple of the window stride %d", P, s->cmp_stride);
  }
  int shift = 0;
  while ((1 << shift) < P) ++shift;
  *out = {p->table, p->table_ld, p->page_ld, (int32_t)p->n_pages, shift, static_cast<uint16_t*>(p->k),
          static_cast<uint16_t*>(p->v), static_cast<uint16_t*>(p->k_cmp)};
  return SPARDA_OK;
}

int check_t_max(const sparda_shape* s, int64_t t_max) {
  if (t_max < 1 || t_max > s->t_cap)
    return fail(SPARDA_ERR_INVALID_ARG, "t_max %lld outside [1, t_cap %lld]", (long long)t_max, (long long)s->t_cap);
  return SPARDA_OK;
}

int check_ws(const void* ws, size_t ws_bytes, size_t need) {
  if (need == 0) return SPARDA_OK;
  if (!ws || !aligned(ws, 16)) return fail(SPARDA_ERR_WORKSPACE, "workspace of %zu bytes required", need);
  if (ws_bytes < need) return fail(SPARDA_ERR_WORKSPACE, "workspace %zu < %zu bytes", ws_bytes, need);
  return SPARDA_OK;
}

}  // namespace

extern "C" {

int sparda_rope_freqs(int32_t rot_dim, double base, int32_t scaling, double factor, double t_train, double low,
                      double high, const double* factors, double* freq, float* scale) {
  if (rot_dim < 2 || rot_dim > kDim || rot_dim % 2 != 0)
    return fail(SPARDA_ERR_INVALID_ARG, "rot_dim %d is not an even number in [2, 128]", rot_dim);
  if (rot_dim % 16 != 0) return fail(SPARDA_ERR_UNSUPPORTED, "rot_dim %d is not a multiple of 16", rot_dim);
  if (!std::isfinite(base) || base <= 1.0) return fail(SPARDA_ERR_INVALID_ARG, "base %g", base);
  if (scaling < SPARDA_ROPE_PLAIN || scaling > SPARDA_ROPE_FACTORS)
    return fail(SPARDA_ERR_INVALID_ARG, "rope scaling %d", scaling);
  if (!freq || !scale) return fail(SPARDA_ERR_INVALID_ARG, "freq or scale is null");
  const bool bands = scaling == SPARDA_ROPE_BANDS, listed = scaling == SPARDA_ROPE_FACTORS;
  if (scaling != SPARDA_ROPE_PLAIN && !(std::isfinite(factor) && factor >= 1.0))
    return fail(SPARDA_ERR_INVALID_ARG, "factor %g", factor);
  if ((bands || listed) && !(std::isfinite(t_train) && t_train > 1.0))
    return fail(SPARDA_ERR_INVALID_ARG, "t_train %g", t_train);
  if (bands && !(low >= 0.0 && low < high && std::isfinite(high)))
    return fail(SPARDA_ERR_INVALID_ARG, "band [%g, %g]", low, high);
  const int n = rot_dim / 2;
  if (listed) {
    if (!factors) return fail(SPARDA_ERR_INVALID_ARG, "factors is null");
    for (int j = 0; j < n; ++j)
      if (!(std::isfinite(factors[j]) && factors[j] > 0.0))
        return fail(SPARDA_ERR_INVALID_ARG, "factors[%d] is %g", j, factors[j]);
  }
  if (scaling == SPARDA_ROPE_BASE) base *= std::pow(factor, rot_dim / (rot_dim - 2.0));
  for (int j = 0; j < n; ++j) {
    const double f = std::pow(base, -2.0 * j / rot_dim);
    double out = f;
    if (scaling == SPARDA_ROPE_LINEAR) out = f / factor;
    if (bands) {
      const double turns = t_train * f / 6.28318530717958647693;
      double keep = (turns - low) / (high - low);
      keep = keep < 0.0 ? 0.0 : keep > 1.0 ? 1.0 : keep;
      out = f * (keep + (1.0 - keep) / factor);
    }
    if (listed) out = f / factors[j];
    freq[j] = out;
  }
  *scale = bands    ? (float)(1.0 + 0.1 * std::log(factor))
           : listed ? (float)std::sqrt(1.0 + std::log(factor) / std::log(t_train))
                    : 1.f;
  return ok();
}

int sparda_rotate(const sparda_rope* rope, int32_t type, int32_t batch, int32_t n_heads, int64_t n_tok,
                  const sparda_rows* x, const int32_t* pos, int64_t pos_ld, const sparda_rows* y, int32_t backward,
                  hipStream_t stream) {
  sparda::RotateArgs a;
  if (!rope) return fail(SPARDA_ERR_INVALID_ARG, "rope is null");
  int rc = check_rope(rope, &a.rope);
  if (rc) return rc;
  if (type != SPARDA_F32 && type != SPARDA_BF16) return fail(SPARDA_ERR_INVALID_ARG, "type %d", type);
  if (backward != 0 && backward != 1) return fail(SPARDA_ERR_INVALID_ARG, "backward %d", backward);
  if (batch < 0 || n_heads < 0 || n_tok < 0) return fail(SPARDA_ERR_INVALID_ARG, "a negative number of rows");
  if (batch == 0 || n_heads == 0 || n_tok == 0) return ok();
  if (n_tok > ((int64_t)1 << 28) / batch) return fail(SPARDA_ERR_UNSUPPORTED, "more than 2^28 tokens");
  const int size = type == SPARDA_F32 ? 4 : 2;
  if ((rc = check_rows_of(x, "x", batch, n_heads, n_tok, size, false, &a.x)) ||
      (rc = check_rows_of(y, "y", batch, n_heads, n_tok, size, true, &a.y)) || (rc = check_dev(pos, "pos", 4)))
    return rc;
  if (pos_ld != 0 && (pos_ld < n_tok || pos_ld >= kMaxStride))
    return fail(SPARDA_ERR_INVALID_ARG, "pos_ld %lld", (long long)pos_ld);
  if (a.x.data == a.y.data &&
      (a.x.ld_batch != a.y.ld_batch || a.x.ld_head != a.y.ld_head || a.x.ld_token != a.y.ld_token))
    return fail(SPARDA_ERR_INVALID_ARG, "in place with other strides");
  a.pos = pos;
  a.pos_ld = pos_ld;
  a.batch = batch;
  a.n_heads = n_heads;
  a.n_tok = n_tok;
  a.bf16 = type == SPARDA_BF16;
  a.backward = backward;
  return hip_status(sparda::launch_rotate(a, stream), "rotation launch");
}

int sparda_paged_append(const sparda_shape* shape, const sparda_pages* pages, const sparda_rope* rope, int32_t n_max,
                        const int32_t* n_new, const int32_t* t_ctx, const sparda_rows* k_new, const sparda_rows* v_new,
                        const sparda_rows* q, const sparda_rows* q_out, const sparda_rows* f, const sparda_rows* f_out,
                        int32_t* t_new, hipStream_t stream) {
  sparda::PagedAppendArgs a = {};
  int rc = check_shape(shape);
  if (rc) return rc;
  if ((rc = check_pages(shape, pages, true, pages && pages->k_cmp, &a.pg)) || (rc = check_rope(rope, &a.rope))) return rc;
  if (n_max < 1) return fail(SPARDA_ERR_INVALID_ARG, "n_max %d < 1", n_max);
  if ((rc = check_rows(shape, n_max, 0))) return rc;
  if ((int64_t)shape->batch * shape->n_kv_heads * n_max > (int64_t)1 << 27)
    return fail(SPARDA_ERR_UNSUPPORTED, "more than 2^27 new rows");
  if ((n_new && (rc = check_dev(n_new, "n_new", 4))) || (rc = check_dev(t_ctx, "t_ctx", 4)) ||
      (rc = check_dev(t_new, "t_new", 4)))
    return rc;
  if (t_new == t_ctx || t_new == n_new)
    return fail(SPARDA_ERR_INVALID_ARG, "t_new is t_ctx or n_new: other workgroups still read it");
  const int B = shape->batch, H = shape->n_kv_heads, Hq = H * shape->group_size;
  if ((q == nullptr) != (q_out == nullptr)) return fail(SPARDA_ERR_INVALID_ARG, "q and q_out: both or neither");
  if ((f == nullptr) != (f_out == nullptr)) return fail(SPARDA_ERR_INVALID_ARG, "f and f_out: both or neither");
  if ((rc = check_rows_of(k_new, "k_new", B, H, n_max, 2, false, &a.k_new)) ||
      (rc = check_rows_of(v_new, "v_new", B, H, n_max, 2, false, &a.v_new)))
    return rc;
  if (q && ((rc = check_rows_of(q, "q", B, Hq, n_max, 2, false, &a.q)) ||
            (rc = check_rows_of(q_out, "q_out", B, Hq, n_max, 2, true, &a.q_out))))
    return rc;
  if (f && ((rc = check_rows_of(f, "f", B, H, n_max, 2, false, &a.f)) ||
            (rc = check_rows_of(f_out, "f_out", B, H, n_max, 2, true, &a.f_out))))
    return rc;
  for (const auto* io : {&a.q, &a.f}) {
    const sparda::Rows& o = io == &a.q ? a.q_out : a.f_out;
    if (io->data && io->data == o.data &&
        (io->ld_batch != o.ld_batch || io->ld_head != o.ld_head || io->ld_token != o.ld_token))
      return fail(SPARDA_ERR_INVALID_ARG, "in place with other strides");
  }
  a.n_new = n_new;
  a.t_ctx = t_ctx;
  a.t_new = t_new;
  a.batch = B;
  a.n_kv_heads = H;
  a.group_size = shape->group_size;
  a.n_max = n_max;
  a.t_cap = shape->t_cap;
  a.grid = grid_of(shape);
  return hip_status(sparda::launch_paged_append(a, stream), "paged append launch");
}

int sparda_paged_select(const sparda_shape* shape, const sparda_pages* pages, const void* f, const int32_t* t_ctx,
                        int64_t t_max, int16_t* sel, int16_t* cnt, void* ws, size_t ws_bytes, hipStream_t stream) {
  sparda::PagedSelectArgs a;
  int rc = check_shape(shape);
  if (rc) return rc;
  if ((rc = check_pages(shape, pages, false, true, &a.pg)) || (rc = check_dev(f, "f", 16)) ||
      (rc = check_dev(t_ctx, "t_ctx", 4)) || (rc = check_dev(sel, "sel", 2)) || (rc = check_dev(cnt, "cnt", 2)) ||
      (rc = check_t_max(shape, t_max)))
    return rc;
  const int64_t rows = (int64_t)shape->batch * shape->n_kv_heads;
  if ((rc = check_ws(ws, ws_bytes, sparda::paged_select_ws(rows, t_max, shape->n_init, shape->n_local)))) return rc;
  a.f = static_cast<const uint16_t*>(f);
  a.t_ctx = t_ctx;
  a.t_max = t_max;
  a.sel = sel;
  a.cnt = cnt;
  a.ws = static_cast<float*>(ws);
  a.ws_stride = sparda::paged_select_stride(t_max, shape->n_init, shape->n_local);
  a.batch = shape->batch;
  a.n_kv_heads = shape->n_kv_heads;
  a.n_init = shape->n_init;
  a.n_local = shape->n_local;
  a.k_total = shape->k_total;
  a.grid = grid_of(shape);
  return hip_status(sparda::launch_paged_select(a, stream), "paged select launch");
}

int sparda_paged_attn(const sparda_shape* shape, const sparda_pages* pages, const void* q, const int32_t* t_ctx,
                      int64_t t_max, const int16_t* sel, const int16_t* cnt, float sm_scale, void* o, void* ws,
                      size_t ws_bytes, hipStream_t stream) {
  sparda::PagedAttnArgs a;
  int rc = check_shape(shape);
  if (rc) return rc;
  if ((rc = check_pages(shape, pages, true, false, &a.pg)) || (rc = check_dev(q, "q", 16)) ||
      (rc = check_dev(t_ctx, "t_ctx", 4)) || (rc = check_dev(o, "o", 16)) || (rc = check_t_max(shape, t_max)))
    return rc;
  if ((sel == nullptr) != (cnt == nullptr)) return fail(SPARDA_ERR_INVALID_ARG, "sel and cnt: both or neither");
  if (sel && ((rc = check_dev(sel, "sel", 2)) || (rc = check_dev(cnt, "cnt", 2)))) return rc;
  if (!std::isfinite(sm_scale * 1.44269504088896340736f)) return fail(SPARDA_ERR_INVALID_ARG, "sm_scale is not finite");
  if ((rc = check_ws(ws, ws_bytes, sparda::paged_attn_ws(shape->batch, shape->group_size)))) return rc;
  a.q = static_cast<const uint16_t*>(q);
  a.t_ctx = t_ctx;
  a.t_max = t_max;
  a.sel = sel;
  a.cnt = cnt;
  a.o = static_cast<uint16_t*>(o);
  a.ws = static_cast<float*>(ws);
  a.batch = shape->batch;
  a.n_kv_heads = shape->n_kv_heads;
  a.group_size = shape->group_size;
  a.k_total = shape->k_total;
  a.scale_log2 = sm_scale * 1.44269504088896340736f;
  return hip_status(sparda::launch_paged_attn(a, stream), "paged attention launch");
}

}  // extern "C"
