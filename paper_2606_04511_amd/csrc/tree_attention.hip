// tree_attention.hip -- attention of the nodes of drafted-token trees over their blocks of the cache
// and their ancestors (paper Sec. 4.1, Eq. 5 over the set of Eq. 1):
//   o_i = softmax(sm_scale q_i K^T) V over {t' < t in the blocks of node i} U A(i).
#include <math.h>

#include "device_util.hpp"
#include "launch.hpp"
#include "tree.hpp"

namespace sparda {

namespace {

constexpr float kLog2eT = 1.4426950408889634f;

// One wavefront per (node, query head).  64 tokens at a time: lane = token for the scores, lane = two
// head dims for P V, an online softmax in between.
__global__ __launch_bounds__(64) void tree_attn_kernel(TreeAttnArgs a) {
  __shared__ float qs[kHeadDim];
  const int lane = threadIdx.x;
  const int n = a.tb.n, G = a.group_size;
  const int i = (int)(blockIdx.x % n);
  const int64_t bh = blockIdx.x / n;  // (b, query head)
  const int64_t bm = bh / G;
  const int b = (int)(bm / a.n_kv_heads);
  const int64_t t = tree_context(a.tb, b);
  const uint64_t anc = tree_ancestors(a.tb.parent + (int64_t)b * n, n, lane);
  const uint64_t mine = ((uint64_t)(uint32_t)readlane_i((int)(anc >> 32), i) << 32) | (uint32_t)readlane_i((int)(uint32_t)anc, i);
  const int64_t qrow = (bh * n + i) * kHeadDim;
  uint32_t* out = reinterpret_cast<uint32_t*>(a.o + qrow);
  if (t < 0 || mine == 0) {
    out[lane] = 0u;
    return;
  }
  const uint32_t qw = reinterpret_cast<const uint32_t*>(a.q + qrow)[lane];
  qs[2 * lane] = bf16lo(qw) * (a.sm_scale * kLog2eT);
  qs[2 * lane + 1] = bf16hi(qw) * (a.sm_scale * kLog2eT);
  __syncthreads();
  float m = -INFINITY, l = 0.f, o0 = 0.f, o1 = 0.f;
  // 64 tokens at kp, vp; lane's token is attended if `on`
  auto tokens = [&](const uint16_t* kp, const uint16_t* vp, bool on) {
    float z = -INFINITY;
    if (on) {
      z = 0.f;
      for (int d = 0; d < kHeadDim; d += 8) {
        const uint4 w = ld16(kp + lane * kHeadDim + d);
        z += bf16lo(w.x) * qs[d] + bf16hi(w.x) * qs[d + 1] + bf16lo(w.y) * qs[d + 2] + bf16hi(w.y) * qs[d + 3] +
             bf16lo(w.z) * qs[d + 4] + bf16hi(w.z) * qs[d + 5] + bf16lo(w.w) * qs[d + 6] + bf16hi(w.w) * qs[d + 7];
      }
    }
    float top = z;
    for (int x = 1; x < 64; x <<= 1) top = fmaxf(top, __shfl_xor(top, x, 64));
    const float m2 = fmaxf(m, top);
    const float ref = m2 > -INFINITY ? m2 : 0.f;
    const float keep = exp2f(m - ref), p = exp2f(z - ref);
    l = l * keep + p;
    o0 *= keep;
    o1 *= keep;
    m = m2;
    for (uint64_t rest = __ballot(on); rest; rest &= rest - 1) {
      const int x = (int)__builtin_ctzll(rest);
      const uint32_t w = reinterpret_cast<const uint32_t*>(vp + x * kHeadDim)[lane];
      const float px = readlane_f(p, x);
      o0 = fmaf(px, bf16lo(w), o0);
      o1 = fmaf(px, bf16hi(w), o1);
    }
  };
  const int64_t srow = a.n_sel == 1 ? bm : bm * n + i;
  const int16_t* sel = a.sel + srow * a.k_total;
  const int listed = min((int)a.cnt[srow], a.k_total);
  for (int e = 0; e < listed; ++e) {
    const int64_t j = sel[e];
    if (j < 0 || j * kBlock >= t) continue;
    bool dup = false;
    for (int x = lane; x < e; x += 64) dup |= sel[x] == j;
    if (__ballot(dup)) continue;
    const int64_t at = (bm * a.t_cap + j * kBlock) * kHeadDim;
    tokens(a.k + at, a.v + at, j * kBlock + lane < t);
  }
  tokens(a.kt + bm * n * kHeadDim, a.vt + bm * n * kHeadDim, ((mine >> lane) & 1ull) != 0ull);
  for (int x = 1; x < 64; x <<= 1) l += __shfl_xor(l, x, 64);
  const float inv = l > 0.f ? 1.f / l : 0.f;
  out[lane] = (uint32_t)f32_to_bf16(o0 * inv) | ((uint32_t)f32_to_bf16(o1 * inv) << 16);
}

}  // namespace

hipError_t launch_tree_attn(const TreeAttnArgs& a, hipStream_t stream) {
  const int64_t rows = (int64_t)a.tb.batch * a.n_kv_heads * a.group_size * a.tb.n;
  hipLaunchKernelGGL(tree_attn_kernel, dim3((unsigned)rows), dim3(64), 0, stream, a);
  return hipGetLastError();
}

}  // namespace sparda
