// tree_abi.cpp -- the extern "C" entry points over trees of drafted tokens (include/sparda.h).
//
// As in sparda_abi.cpp every argument is checked on the host before any HIP call.  What lives in
// device memory (lengths, parents, paths, block lists) is bounded by the kernels.
#include "sparda.h"

#include <hip/hip_runtime.h>

#include <cmath>

#include "abi_checks.hpp"
#include "tree.hpp"

using namespace sparda::abi;

namespace {

// n_nodes and, where the call has one, the longest context.
int check_tree(const sparda_shape* s, int32_t n_nodes, int64_t t_max) {
  if (n_nodes < 1) return fail(SPARDA_ERR_INVALID_ARG, "n_nodes %d < 1", n_nodes);
  if (n_nodes > sparda::kTreeMaxNodes)
    return fail(SPARDA_ERR_UNSUPPORTED, "n_nodes %d > %d", n_nodes, sparda::kTreeMaxNodes);
  return check_rows(s, n_nodes, t_max);
}

}  // namespace

extern "C" {

int sparda_tree_select(const sparda_shape* shape, const void* f, int32_t n_nodes, const int32_t* t_ctx, int64_t t_max,
                       const int32_t* parent, const void* k_cmp, int16_t* sel, int16_t* cnt, void* ws,
                       size_t ws_bytes, hipStream_t stream) {
  int rc = check_shape(shape);
  if (rc) return rc;
  if ((rc = check_dev(f, "f", 16)) || (rc = check_dev(t_ctx, "t_ctx", 4)) || (rc = check_dev(parent, "parent", 4)) ||
      (rc = check_dev(k_cmp, "k_cmp", 16)) || (rc = check_dev(sel, "sel", 2)) || (rc = check_dev(cnt, "cnt", 2)))
    return rc;
  if ((rc = check_tree(shape, n_nodes, t_max))) return rc;
  if (shape->n_local < 2)
    return fail(SPARDA_ERR_UNSUPPORTED, "n_local %d < 2: the block that drafted tokens complete has no compressed key",
                shape->n_local);
  const int32_t last = sparda::tree_last_key(grid_of(shape), t_max, n_nodes, shape->n_init, shape->n_local, shape->k_total);
  if (last >= shape->nc_cap)
    return fail(SPARDA_ERR_INVALID_ARG, "compressed key %d beyond nc_cap %lld", last, (long long)shape->nc_cap);
  const int64_t groups = (int64_t)shape->batch * shape->n_kv_heads;
  const size_t need = sparda::tree_select_ws(groups, t_max, n_nodes, shape->n_init, shape->n_local);
  if (need > 0) {
    if (!ws || !aligned(ws, 16)) return fail(SPARDA_ERR_WORKSPACE, "workspace of %zu bytes required", need);
    if (ws_bytes < need) return fail(SPARDA_ERR_WORKSPACE, "workspace %zu < %zu bytes", ws_bytes, need);
  }
  sparda::TreeSelectArgs a;
  a.tb = {t_ctx, parent, shape->batch, n_nodes, t_max};
  a.f = static_cast<const uint16_t*>(f);
  a.kc = static_cast<const uint16_t*>(k_cmp);
  a.sel = sel;
  a.cnt = cnt;
  a.ws = static_cast<float*>(ws);
  a.ws_stride = sparda::tree_select_stride(t_max, n_nodes, shape->n_init, shape->n_local);
  a.n_kv_heads = shape->n_kv_heads;
  a.nc_cap = shape->nc_cap;
  a.n_init = shape->n_init;
  a.n_local = shape->n_local;
  a.k_total = shape->k_total;
  a.grid = grid_of(shape);
  return hip_status(sparda::launch_tree_select(a, stream), "tree select launch");
}

int sparda_tree_attn(const sparda_shape* shape, const void* q, int32_t n_nodes, const int32_t* t_ctx, int64_t t_max,
                     const int32_t* parent, const void* k, const void* v, const void* k_tree, const void* v_tree,
                     int32_t n_sel, const int16_t* sel, const int16_t* cnt, float sm_scale, void* o, void* ws,
                     size_t ws_bytes, hipStream_t stream) {
  int rc = check_shape(shape);
  if (rc) return rc;
  if ((rc = check_dev(q, "q", 16)) || (rc = check_dev(t_ctx, "t_ctx", 4)) || (rc = check_dev(parent, "parent", 4)) ||
      (rc = check_dev(k, "k", 16)) || (rc = check_dev(v, "v", 16)) || (rc = check_dev(k_tree, "k_tree", 16)) ||
      (rc = check_dev(v_tree, "v_tree", 16)) || (rc = check_dev(sel, "sel", 2)) || (rc = check_dev(cnt, "cnt", 2)) ||
      (rc = check_dev(o, "o", 16)))
    return rc;
  if ((rc = check_tree(shape, n_nodes, t_max))) return rc;
  if (n_sel != 1 && n_sel != n_nodes)
    return fail(SPARDA_ERR_INVALID_ARG, "n_sel %d is neither 1 nor n_nodes %d", n_sel, n_nodes);
  if (!std::isfinite(sm_scale)) return fail(SPARDA_ERR_INVALID_ARG, "sm_scale is not finite");
  const sparda::TreeAttnPlan plan = sparda::tree_attn_plan((int64_t)shape->batch * shape->n_kv_heads, n_nodes,
                                                           shape->group_size, shape->k_total, t_max, n_sel == 1);
  const size_t need = sparda::tree_attn_ws((int64_t)shape->batch * shape->n_kv_heads, n_nodes, shape->group_size,
                                           shape->k_total, t_max);
  if (need > 0) {
    if (!ws || !aligned(ws, 16)) return fail(SPARDA_ERR_WORKSPACE, "workspace of %zu bytes required", need);
    if (ws_bytes < need) return fail(SPARDA_ERR_WORKSPACE, "workspace %zu < %zu bytes", ws_bytes, need);
  }
  sparda::TreeAttnArgs a;
  a.tb = {t_ctx, parent, shape->batch, n_nodes, t_max};
  a.q = static_cast<const uint16_t*>(q);
  a.k = static_cast<const uint16_t*>(k);
  a.v = static_cast<const uint16_t*>(v);
  a.kt = static_cast<const uint16_t*>(k_tree);
  a.vt = static_cast<const uint16_t*>(v_tree);
  a.sel = sel;
  a.cnt = cnt;
  a.o = static_cast<uint16_t*>(o);
  a.ws = static_cast<float*>(ws);
  a.n_kv_heads = shape->n_kv_heads;
  a.group_size = shape->group_size;
  a.n_sel = n_sel;
  a.k_total = shape->k_total;
  a.t_cap = shape->t_cap;
  a.sm_scale = sm_scale;
  a.width = plan.width;
  a.n_splits = plan.n_splits;
  a.k_recip = (((uint64_t)1 << 36) + shape->k_total - 1) / shape->k_total;
  a.groups_recip = (((uint64_t)1 << 36) + (uint64_t)shape->batch * shape->n_kv_heads - 1) /
                   ((uint64_t)shape->batch * shape->n_kv_heads);
  a.ns_recip = ((1u << 20) + plan.n_splits - 1) / plan.n_splits;
  a.g_recip = ((1u << 16) + shape->group_size - 1) / shape->group_size;
  return hip_status(sparda::launch_tree_attn(a, stream), "tree attention launch");
}

int sparda_tree_verify_workspace_size(const sparda_shape* shape, int32_t n_nodes, int32_t vocab, size_t* bytes) {
  int rc = check_shape(shape);
  if (rc) return rc;
  if (!bytes) return fail(SPARDA_ERR_INVALID_ARG, "bytes is null");
  if ((rc = check_tree(shape, n_nodes, 0))) return rc;
  if (vocab < 1) return fail(SPARDA_ERR_INVALID_ARG, "vocab %d < 1", vocab);
  *bytes = sparda::tree_verify_ws(shape->batch, vocab);
  return ok();
}

int sparda_tree_verify(const sparda_shape* shape, int32_t n_nodes, int32_t vocab, int64_t ld, int32_t prob_type,
                       const void* p, const void* q, const int32_t* tokens, const int32_t* parent, const float* u,
                       int32_t* path, int32_t* n_path, int32_t* next_token, void* ws, size_t ws_bytes,
                       hipStream_t stream) {
  int rc = check_shape(shape);
  if (rc) return rc;
  if ((rc = check_dev(p, "p", 16)) || (q && (rc = check_dev(q, "q", 16))) || (rc = check_dev(tokens, "tokens", 4)) ||
      (rc = check_dev(parent, "parent", 4)) || (rc = check_dev(u, "u", 4)) || (rc = check_dev(path, "path", 4)) ||
      (rc = check_dev(n_path, "n_path", 4)) || (rc = check_dev(next_token, "next_token", 4)))
    return rc;
  if ((rc = check_tree(shape, n_nodes, 0))) return rc;
  if (vocab < 1) return fail(SPARDA_ERR_INVALID_ARG, "vocab %d < 1", vocab);
  if (ld < vocab) return fail(SPARDA_ERR_INVALID_ARG, "ld %lld < vocab %d", (long long)ld, vocab);
  if (prob_type != SPARDA_PROB_F32 && prob_type != SPARDA_PROB_BF16)
    return fail(SPARDA_ERR_INVALID_ARG, "prob_type %d", prob_type);
  const size_t need = sparda::tree_verify_ws(shape->batch, vocab);
  if (!ws || !aligned(ws, 16)) return fail(SPARDA_ERR_WORKSPACE, "workspace of %zu bytes required", need);
  if (ws_bytes < need) return fail(SPARDA_ERR_WORKSPACE, "workspace %zu < %zu bytes", ws_bytes, need);
  sparda::TreeVerifyArgs a;
  a.p = p;
  a.q = q;
  a.tokens = tokens;
  a.parent = parent;
  a.u = u;
  a.path = path;
  a.n_path = n_path;
  a.next_token = next_token;
  a.ws = ws;
  a.ld = ld;
  a.batch = shape->batch;
  a.n = n_nodes;
  a.vocab = vocab;
  a.bf16 = prob_type == SPARDA_PROB_BF16;
  return hip_status(sparda::launch_tree_verify(a, stream), "tree verify launch");
}

int sparda_tree_commit(const sparda_shape* shape, int32_t n_nodes, const int32_t* t_ctx, const int32_t* path,
                       const int32_t* n_path, int32_t n_layers, const void* const* k_tree, const void* const* v_tree,
                       void* const* k_cache, void* const* v_cache, void* const* k_cmp, int32_t* t_new,
                       hipStream_t stream) {
  int rc = check_shape(shape);
  if (rc) return rc;
  if ((rc = check_dev(t_ctx, "t_ctx", 4)) || (rc = check_dev(path, "path", 4)) ||
      (rc = check_dev(n_path, "n_path", 4)) || (rc = check_dev(t_new, "t_new", 4)))
    return rc;
  if ((rc = check_tree(shape, n_nodes, 0))) return rc;
  if (t_new == t_ctx) return fail(SPARDA_ERR_INVALID_ARG, "t_new is t_ctx: other workgroups still read it");
  if (n_layers < 1) return fail(SPARDA_ERR_INVALID_ARG, "n_layers %d < 1", n_layers);
  if (!k_tree || !v_tree || !k_cache || !v_cache)
    return fail(SPARDA_ERR_INVALID_ARG, "a table of the layers' pointers is null");
  for (int32_t l = 0; l < n_layers; ++l) {
    if ((rc = check_dev(k_tree[l], "k_tree", 16)) || (rc = check_dev(v_tree[l], "v_tree", 16)) ||
        (rc = check_dev(k_cache[l], "k_cache", 16)) || (rc = check_dev(v_cache[l], "v_cache", 16)) ||
        (k_cmp && (rc = check_dev(k_cmp[l], "k_cmp", 16))))
      return rc;
  }
  for (int32_t l0 = 0; l0 < n_layers; l0 += sparda::kCommitLayers) {
    sparda::TreeCommitArgs a = {};
    a.n_layers = n_layers - l0 < sparda::kCommitLayers ? n_layers - l0 : sparda::kCommitLayers;
    for (int32_t i = 0; i < a.n_layers; ++i) {
      a.kt[i] = static_cast<const uint16_t*>(k_tree[l0 + i]);
      a.vt[i] = static_cast<const uint16_t*>(v_tree[l0 + i]);
      a.k[i] = static_cast<uint16_t*>(k_cache[l0 + i]);
      a.v[i] = static_cast<uint16_t*>(v_cache[l0 + i]);
      a.kc[i] = k_cmp ? static_cast<uint16_t*>(k_cmp[l0 + i]) : nullptr;
    }
    a.t_ctx = t_ctx;
    a.path = path;
    a.n_path = n_path;
    a.t_new = l0 == 0 ? t_new : nullptr;
    a.batch = shape->batch;
    a.n_kv_heads = shape->n_kv_heads;
    a.n = n_nodes;
    a.t_cap = shape->t_cap;
    a.nc_cap = shape->nc_cap;
    a.grid = grid_of(shape);
    if ((rc = hip_status(sparda::launch_tree_commit(a, stream), "tree commit launch"))) return rc;
  }
  return ok();
}

}  // extern "C"
