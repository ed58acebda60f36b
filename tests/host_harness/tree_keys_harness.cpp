// tree_keys_harness.cpp -- which rows of K~ the selection over trees reads, on the host: for many shapes it finds the
// smallest nc_cap that sparda_tree_select accepts and walks through every key that the scoring launch requests then.
// The launch itself is replaced by that walk, with the launch's own bounds (tree.hpp).
#include <algorithm>
#include <cstdint>
#include <cstdio>
#include <vector>

#include "sparda.h"
#include "tree.hpp"

namespace {
long g_rows = 0, g_outside = 0;
std::vector<int64_t> g_contexts;  // of the next call's sequences
}  // namespace

extern "C" const char* hipGetErrorString(hipError_t) { return "no runtime"; }

namespace sparda {

hipError_t launch_tree_attn(const TreeAttnArgs&, hipStream_t) { return hipSuccess; }
hipError_t launch_tree_verify(const TreeVerifyArgs&, hipStream_t) { return hipSuccess; }
hipError_t launch_tree_commit(const TreeCommitArgs&, hipStream_t) { return hipSuccess; }

// A step takes 64 consecutive keys from its first candidate's first window on; the windows of 32 tokens begin with the
// window before the first candidate's.
hipError_t launch_tree_select(const TreeSelectArgs& a, hipStream_t) {
  const bool blocks = grid_is_blocks(a.grid);
  auto read = [&](int32_t row) {
    ++g_rows;
    if (row < 0 || row >= a.nc_cap) ++g_outside;
  };
  for (const int64_t t : g_contexts) {
    const RowGeom g = row_geom(t + a.tb.n - 1, a.n_init, a.n_local, a.k_total);
    if (g.n_take >= g.n_cand) continue;
    const int32_t last = tree_last_key(a.grid, t, a.tb.n, a.n_init, a.n_local, a.k_total);
    for (int x = 0; x < g.n_cand; x += blocks ? 64 : 16) {
      const int32_t w0 = blocks ? g.cand_lo + x : 4 * (g.cand_lo + x);
      if (!blocks) read(tree_key_row(w0 - 1, last));
      for (int z = 0; z < 64; ++z) read(tree_key_row(w0 + z, last));
    }
    // every window that a score takes is among them
    const int32_t first = std::max(grid_win_lo(a.grid, g.cand_lo), 0);
    const int32_t hi = grid_win_hi(a.grid, g.cand_lo + g.n_cand - 1), vis = grid_win_vis(a.grid, t - 1);
    for (int32_t w = first; w <= std::min(hi, vis); ++w)
      if (tree_key_row(w, last) != w) ++g_outside;
  }
  return hipSuccess;
}

}  // namespace sparda

int main() {
  long calls = 0, refused = 0;
  void* const at = reinterpret_cast<void*>((uintptr_t)1 << 44);
  for (int grid : {64, 32})
    for (int n_local : {2, 3, 32})
      for (int n_init : {0, 1, 4})
        for (int n : {1, 7, 64})
          for (int64_t t_max : {0, 64, 127, 300, 2047, 4096, 4111, 9000, 33000}) {
            sparda_shape s{(uint32_t)sizeof(sparda_shape), 2, 3, 4, 128, 64, grid, grid == 64 ? 64 : 16, n_init, n_local,
                           n_init + n_local + 2, (t_max + n + 63) / 64 * 64, 0};
            g_contexts.clear();
            for (int64_t back = 0; back <= std::min<int64_t>(t_max, 200); ++back) g_contexts.push_back(t_max - back);
            int16_t* const out = static_cast<int16_t*>(at);
            int32_t* const in = static_cast<int32_t*>(at);
            for (;; ++s.nc_cap) {
              const int rc = sparda_tree_select(&s, at, n, in, t_max, in, at, out, out, at, (size_t)1 << 40, nullptr);
              ++calls;
              if (rc == SPARDA_OK) break;
              ++refused;
              if (rc != SPARDA_ERR_INVALID_ARG) return 2;
            }
          }
  std::printf("%ld calls, %ld refused, %ld rows requested, %ld outside the cache\n", calls, refused, g_rows, g_outside);
  return g_outside == 0 && g_rows > 100000 ? 0 : 1;
}
