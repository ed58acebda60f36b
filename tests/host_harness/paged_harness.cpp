// paged_harness.cpp -- drives the entry points of rotary positions and paged caches through their host code, built like
// abi_harness.cpp against the stub runtime of hip_stub.cpp: the planning of every size from one token to the largest
// shapes the limits allow, exact workspaces, frequency tables in buffers of exactly their size, and refusals.  Device
// pointers are never dereferenced on the host.
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

sparda_shape shape(int batch, int heads, int group, int k, int64_t t_cap, int l, int s) {
  return sparda_shape{(uint32_t)sizeof(sparda_shape), batch, heads, group, 128, 64, l, s, 1, 2, k, t_cap, 0};
}
sparda_pages pages(const sparda_shape& s, int page, int64_t n_pages, bool cmp) {
  return sparda_pages{(uint32_t)sizeof(sparda_pages), page, n_pages, (s.t_cap + page - 1) / page,
                      (int64_t)s.n_kv_heads * page * 128, i32(), dev(), dev(), cmp ? dev() : nullptr};
}
sparda_rows rows(int64_t heads, int64_t tokens) { return sparda_rows{dev(), heads * tokens * 128, tokens * 128, 128}; }

void step(const sparda_shape& s, int page, int64_t t_max, int n_max) {
  const bool cmp = page % s.cmp_stride == 0;
  const sparda_pages p = pages(s, page, 1000, cmp);
  const sparda_rope rope{(uint32_t)sizeof(sparda_rope), 96, SPARDA_ROPE_PAIRS, 1.25f, static_cast<double*>(dev())};
  size_t ws = 0;
  if (cmp) {
    EXPECT(sparda_workspace_size(&s, SPARDA_OP_PAGED_SELECT, 1, t_max - 1, &ws), SPARDA_OK);
    EXPECT(sparda_paged_select(&s, &p, dev(), i32(), t_max, i16(), i16(), ws ? dev() : nullptr, ws, nullptr), SPARDA_OK);
    if (ws) EXPECT(sparda_paged_select(&s, &p, dev(), i32(), t_max, i16(), i16(), dev(), ws - 1, nullptr), SPARDA_ERR_WORKSPACE);
  }
  EXPECT(sparda_workspace_size(&s, SPARDA_OP_PAGED_ATTN, 1, t_max - 1, &ws), SPARDA_OK);
  EXPECT(sparda_paged_attn(&s, &p, dev(), i32(), t_max, nullptr, nullptr, 0.088f, dev(), dev(), ws, nullptr), SPARDA_OK);
  EXPECT(sparda_paged_attn(&s, &p, dev(), i32(), t_max, i16(), i16(), 0.088f, dev(), dev(), ws, nullptr), SPARDA_OK);
  EXPECT(sparda_paged_attn(&s, &p, dev(), i32(), t_max, i16(), i16(), 0.088f, dev(), dev(), ws - 1, nullptr), SPARDA_ERR_WORKSPACE);
  const int H = s.n_kv_heads, Hq = H * s.group_size;
  const sparda_rows k = rows(H, n_max), v = rows(H, n_max), q = rows(Hq, n_max), qo = rows(Hq, n_max), f = rows(H, n_max);
  const bool fits = (int64_t)s.batch * H * n_max <= (int64_t)1 << 27;
  EXPECT(sparda_paged_append(&s, &p, &rope, n_max, i32(), i32(), &k, &v, &q, &qo, &f, &f, i32(), nullptr), fits ? SPARDA_OK : SPARDA_ERR_UNSUPPORTED);
  EXPECT(sparda_paged_append(&s, &p, nullptr, n_max, nullptr, i32(), &k, &v, nullptr, nullptr, nullptr, nullptr, i32(), nullptr), fits ? SPARDA_OK : SPARDA_ERR_UNSUPPORTED);
  for (int type : {SPARDA_F32, SPARDA_BF16})
    EXPECT(sparda_rotate(&rope, type, s.batch, Hq, n_max, &q, i32(), 0, &qo, 1, nullptr),
           (int64_t)s.batch * n_max <= (int64_t)1 << 28 ? SPARDA_OK : SPARDA_ERR_UNSUPPORTED);
}

}  // namespace

int main() {
  for (int page : {16, 64, 4096})
    for (int g : {1, 4, 16}) {
      step(shape(1, 1, g, 3, 64, 64, 64), page, 1, 1);
      step(shape(1, 8, g, 16, 4096, 32, 16), page, 4096, 17);
      step(shape(8, 8, g, 64, 32768, 32, 16), page, 32700, 4096);
      step(shape(32, 8, g, 64, 131072, 64, 64), page, 131000, 1);
      step(shape(200, 8, g, 70, 2048, 64, 64), page, 250, 64);
      step(shape(700, 3, g, 5, 8192, 32, 16), page, 8192, 1);
      step(shape(2, 2, g, 2000, 2097152, 32, 16), page, 2097152, 1000);
    }
  step(shape(65535, 1, 16, 32767, 2097152, 64, 64), 65536, 2097152, 2048);
  step(shape(4095, 16, 1, 3, 2097152, 32, 16), 16, 2097152, 2097152);
  for (int rot = 16; rot <= 128; rot += 16)
    for (int kind = SPARDA_ROPE_PLAIN; kind <= SPARDA_ROPE_FACTORS; ++kind) {
      std::vector<double> freq(rot / 2, NAN), factors(rot / 2, 2.0);
      float scale = NAN;
      EXPECT(sparda_rope_freqs(rot, 10000.0, kind, 4.0, 8192.0, 1.0, 32.0, factors.data(), freq.data(), &scale), SPARDA_OK);
      for (double x : freq)
        if (!(x > 0.0 && x <= 1.0)) ++g_failures;
      if (!(scale >= 1.f)) ++g_failures;
    }
  EXPECT(sparda_rope_freqs(128, 10000.0, SPARDA_ROPE_FACTORS, 4.0, 8192.0, 1.0, 32.0, nullptr, nullptr, nullptr), SPARDA_ERR_INVALID_ARG);
  const sparda_rope none{(uint32_t)sizeof(sparda_rope), 0, SPARDA_ROPE_HALF, 1.f, nullptr};
  const sparda_rows r = rows(4, 1 << 26);
  EXPECT(sparda_rotate(&none, SPARDA_BF16, 4, 4, (int64_t)1 << 26, &r, i32(), (int64_t)1 << 26, &r, 0, nullptr), SPARDA_OK);
  EXPECT(sparda_rotate(&none, SPARDA_BF16, 5, 4, (int64_t)1 << 26, &r, i32(), (int64_t)1 << 26, &r, 0, nullptr), SPARDA_ERR_UNSUPPORTED);
  EXPECT(sparda_rotate(&none, SPARDA_BF16, 0, 4, 7, nullptr, nullptr, 0, nullptr, 0, nullptr), SPARDA_OK);
  EXPECT(sparda_rotate(nullptr, SPARDA_BF16, 1, 4, 7, &r, i32(), 7, &r, 0, nullptr), SPARDA_ERR_INVALID_ARG);
  std::printf("paged harness: %ld launches checked, %ld with an invalid configuration, %d failed expectations\n",
              stub_launches(), stub_bad_launches(), g_failures);
  return g_failures == 0 && stub_bad_launches() == 0 ? 0 : 1;
}
