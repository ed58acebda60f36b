// abi_checks.hpp -- what the extern "C" entry points share: the thread's error text, the checks of a
// shape, a pointer and a row range, and the status of a launch (private to the library).
#pragma once

#include "sparda.h"

#include <hip/hip_runtime.h>

#include <cstdarg>
#include <cstdio>
#include <string>

#include "launch.hpp"

namespace sparda {
namespace abi {

inline thread_local std::string g_detail;

inline int fail(int status, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  std::vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  g_detail = buf;
  return status;
}

inline int ok() {
  g_detail.clear();
  return SPARDA_OK;
}

inline bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

constexpr int64_t kMaxBlocks = 32768;  // block indices are int16

inline int check_shape(const sparda_shape* s) {
  if (!s) return fail(SPARDA_ERR_INVALID_ARG, "shape is null");
  if (s->struct_size != sizeof(sparda_shape))
    return fail(SPARDA_ERR_INVALID_ARG, "shape.struct_size is %u, expected %zu", s->struct_size, sizeof(sparda_shape));
  if (s->batch < 1 || s->n_kv_heads < 1 || s->group_size < 1)
    return fail(SPARDA_ERR_INVALID_ARG, "batch, n_kv_heads and group_size must be >= 1");
  if (s->group_size > 16) return fail(SPARDA_ERR_UNSUPPORTED, "group_size %d > 16", s->group_size);
  if (s->head_dim != 128) return fail(SPARDA_ERR_UNSUPPORTED, "head_dim %d (only 128)", s->head_dim);
  if (s->block_size != 64) return fail(SPARDA_ERR_UNSUPPORTED, "block_size %d (only 64)", s->block_size);
  if (!((s->cmp_kernel == 64 && s->cmp_stride == 64) || (s->cmp_kernel == 32 && s->cmp_stride == 16)))
    return fail(SPARDA_ERR_UNSUPPORTED, "compression window (%d, %d) (only (64, 64) and (32, 16))", s->cmp_kernel,
                s->cmp_stride);
  if (s->n_init < 0 || s->n_local < 1) return fail(SPARDA_ERR_INVALID_ARG, "n_init >= 0 and n_local >= 1 required");
  if ((int64_t)s->k_total < (int64_t)s->n_init + s->n_local)
    return fail(SPARDA_ERR_INVALID_ARG, "k_total %d < n_init + n_local", s->k_total);
  if (s->k_total >= kMaxBlocks) return fail(SPARDA_ERR_UNSUPPORTED, "k_total %d too large", s->k_total);
  if (s->t_cap < 64 || s->t_cap % 64 != 0)
    return fail(SPARDA_ERR_INVALID_ARG, "t_cap %lld must be a positive multiple of 64", (long long)s->t_cap);
  if (s->t_cap / 64 > kMaxBlocks)
    return fail(SPARDA_ERR_UNSUPPORTED, "t_cap %lld exceeds 32768 blocks", (long long)s->t_cap);
  if (s->nc_cap < 0 || s->nc_cap > kMaxBlocks * (64 / s->cmp_stride))
    return fail(SPARDA_ERR_INVALID_ARG, "nc_cap out of range");
  if ((int64_t)s->batch * s->n_kv_heads > 65535)
    return fail(SPARDA_ERR_UNSUPPORTED, "batch * n_kv_heads > 65535");
  return SPARDA_OK;
}

inline int check_dev(const void* p, const char* name, uintptr_t align) {
  if (!p) return fail(SPARDA_ERR_INVALID_ARG, "%s is null", name);
  if (!aligned(p, align)) return fail(SPARDA_ERR_INVALID_ARG, "%s is not %zu-byte aligned", name, (size_t)align);
  return SPARDA_OK;
}

inline int check_rows(const sparda_shape* s, int32_t n_q, int64_t q_pos0) {
  if (n_q < 1) return fail(SPARDA_ERR_INVALID_ARG, "n_q %d < 1", n_q);
  if (q_pos0 < 0 || q_pos0 > s->t_cap - n_q)  // (q_pos0 + n_q can pass 64 bits)
    return fail(SPARDA_ERR_INVALID_ARG, "%d positions from %lld on outside t_cap %lld", n_q, (long long)q_pos0,
                (long long)s->t_cap);
  const int64_t rows = (int64_t)s->batch * s->n_kv_heads * n_q;
  if (rows > (int64_t)1 << 30) return fail(SPARDA_ERR_UNSUPPORTED, "too many query rows");
  return SPARDA_OK;
}

inline WinGrid grid_of(const sparda_shape* s) { return WinGrid{s->cmp_kernel, s->cmp_stride}; }

inline int hip_status(hipError_t e, const char* what) {
  if (e != hipSuccess) return fail(SPARDA_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
  return ok();
}

}  // namespace abi
}  // namespace sparda
