// tree_harness.cpp -- drives the entry points over trees of drafted tokens through their host code, built like
// abi_harness.cpp against the stub runtime of hip_stub.cpp: the planning of every size from one token to the largest
// shapes the limits allow, exact workspaces, and a refusal for each documented error.  Device pointers are never
// dereferenced on the host; the layer tables are host arrays of exactly n_layers entries.
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <vector>

#include "sparda.h"

extern "C" {
long stub_launches(void);
long stub_bad_launches(void);
}

namespace {

int g_failures = 0;
void expect(int got, int want, const char* what, int line) {
  if (got == want) return;
  std::fprintf(stderr, "line %d: %s returned %d, expected %d: %s\n", line, what, got, want, sparda_last_error_detail());
  ++g_failures;
}
#define EXPECT(call, want) expect((call), (want), #call, __LINE__)

void* dev() {
  static uintptr_t next = (uintptr_t)1 << 44;
  next += 4096;
  return reinterpret_cast<void*>(next);
}
int16_t* i16() { return static_cast<int16_t*>(dev()); }
int32_t* i32() { return static_cast<int32_t*>(dev()); }

sparda_shape shape(int batch, int heads, int group, int k, int64_t t_cap, int64_t nc, int l, int s) {
  return sparda_shape{(uint32_t)sizeof(sparda_shape), batch, heads, group, 128, 64, l, s, 1, 2, k, t_cap, nc};
}

void step(const sparda_shape& s, int n, int64_t t_max, int vocab, int layers) {
  size_t ws = 0;
  EXPECT(sparda_workspace_size(&s, SPARDA_OP_TREE_SELECT, n, t_max, &ws), SPARDA_OK);
  EXPECT(sparda_tree_select(&s, dev(), n, i32(), t_max, i32(), dev(), i16(), i16(), ws ? dev() : nullptr, ws, nullptr), SPARDA_OK);
  if (ws) EXPECT(sparda_tree_select(&s, dev(), n, i32(), t_max, i32(), dev(), i16(), i16(), dev(), ws - 1, nullptr), SPARDA_ERR_WORKSPACE);
  EXPECT(sparda_workspace_size(&s, SPARDA_OP_TREE_ATTN, n, t_max, &ws), SPARDA_OK);
  for (int n_sel : {1, n})
    EXPECT(sparda_tree_attn(&s, dev(), n, i32(), t_max, i32(), dev(), dev(), dev(), dev(), n_sel, i16(), i16(), 0.088f, dev(), ws ? dev() : nullptr, ws, nullptr), SPARDA_OK);
  if (ws) EXPECT(sparda_tree_attn(&s, dev(), n, i32(), t_max, i32(), dev(), dev(), dev(), dev(), n, i16(), i16(), 0.088f, dev(), dev(), ws - 1, nullptr), SPARDA_ERR_WORKSPACE);
  EXPECT(sparda_tree_verify_workspace_size(&s, n, vocab, &ws), SPARDA_OK);
  for (int type : {SPARDA_PROB_F32, SPARDA_PROB_BF16}) {
    EXPECT(sparda_tree_verify(&s, n, vocab, vocab, type, dev(), nullptr, i32(), i32(), (float*)dev(), i32(), i32(), i32(), dev(), ws, nullptr), SPARDA_OK);
    EXPECT(sparda_tree_verify(&s, n, vocab, vocab, type, dev(), dev(), i32(), i32(), (float*)dev(), i32(), i32(), i32(), dev(), ws, nullptr), SPARDA_OK);
  }
  std::vector<void*> tab(layers);
  for (auto& p : tab) p = dev();
  EXPECT(sparda_tree_commit(&s, n, i32(), i32(), i32(), layers, tab.data(), tab.data(), tab.data(), tab.data(), tab.data(), i32(), nullptr), SPARDA_OK);
  EXPECT(sparda_tree_commit(&s, n, i32(), i32(), i32(), layers, tab.data(), tab.data(), tab.data(), tab.data(), nullptr, i32(), nullptr), SPARDA_OK);
}

}  // namespace

int main() {
  for (int n : {1, 2, 5, 16, 33, 64})
    for (int g : {1, 3, 4, 7, 16}) {
      step(shape(1, 1, g, 3, 128, 2, 64, 64), n, 0, 1, 1);
      step(shape(1, 8, g, 16, 4160, 65, 64, 64), n, 4096, 32000, 1);
      step(shape(8, 8, g, 64, 32832, 2051, 32, 16), n, 32700, 50021, 32);
      step(shape(32, 8, g, 64, 131072, 2048, 64, 64), n, 131000, 131072, 33);
      step(shape(2, 2, g, 96, 2097152, 131071, 32, 16), n, 2097000, 1 << 20, 70);
    }
  step(shape(65535, 1, 16, 32767, 2097152, 32768, 64, 64), 64, 2097088, 2147483647, 1);
  step(shape(4095, 16, 1, 3, 64, 1, 64, 64), 1, 63, 7, 1000);
  sparda_shape s = shape(2, 2, 4, 16, 4096, 64, 64, 64);
  size_t ws = 0;
  EXPECT(sparda_workspace_size(&s, SPARDA_OP_TREE_ATTN, 65, 0, &ws), SPARDA_ERR_UNSUPPORTED);
  EXPECT(sparda_workspace_size(&s, SPARDA_OP_TREE_SELECT, 8, 4089, &ws), SPARDA_ERR_INVALID_ARG);
  EXPECT(sparda_tree_verify_workspace_size(&s, 8, 0, &ws), SPARDA_ERR_INVALID_ARG);
  EXPECT(sparda_tree_verify_workspace_size(&s, 8, 10, nullptr), SPARDA_ERR_INVALID_ARG);
  EXPECT(sparda_tree_verify_workspace_size(nullptr, 8, 10, &ws), SPARDA_ERR_INVALID_ARG);
  s.n_local = 1;
  EXPECT(sparda_tree_select(&s, dev(), 8, i32(), 100, i32(), dev(), i16(), i16(), dev(), 1 << 20, nullptr), SPARDA_ERR_UNSUPPORTED);
  std::printf("tree harness: %ld launches checked, %ld with an invalid configuration, %d failed expectations\n",
              stub_launches(), stub_bad_launches(), g_failures);
  return g_failures == 0 && stub_bad_launches() == 0 ? 0 : 1;
}
