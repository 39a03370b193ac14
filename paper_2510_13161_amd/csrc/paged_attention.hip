// Paged attention: dispatch, and the kernel that joins a sequence's chunks.
#include "paged_plan.h"

namespace msd {

void launch_paged_bf16_64(const PagedAttnArgs& a, const Topo& topo, dim3 grid, hipStream_t s);
void launch_paged_bf16_128(const PagedAttnArgs& a, const Topo& topo, dim3 grid, hipStream_t s);
void launch_paged_fp8_64(const PagedAttnArgs& a, const Topo& topo, dim3 grid, hipStream_t s);
void launch_paged_fp8_128(const PagedAttnArgs& a, const Topo& topo, dim3 grid, hipStream_t s);

namespace {

// A workgroup a (sequence, kv head, query tile), a thread 8 dims of a query (half
// of the threads idle at head dim 64). 4 us for 4 chunks or fewer (a launch and two
// dependent loads), 5 for 8, 8.5 for 24.
template <int HD>
__global__ __launch_bounds__(256) void paged_merge_kernel(PagedAttnArgs a) {
  const int tid = threadIdx.x;
  int id = blockIdx.x;
  const int kvh = id % a.kv.heads;
  id /= a.kv.heads;
  const int tile = id % (a.groups * a.q_per_wg);
  const int b = id / (a.groups * a.q_per_wg);
  const int G = a.n_heads / a.kv.heads, Qn = G * a.n_slots;
  if (tile * 16 >= Qn) return;
  const int u0 = a.plan[b], nch = a.plan[b + 1] - u0;
  if (nch <= 1) return;  // none, or written by its workgroup
  const int qloc = tid / (HD / 8), c8 = tid % (HD / 8);
  const int qg = tile * 16 + qloc;
  if (qloc >= 16 || qg >= Qn) return;
  int gq, slot;
  query_of(a, qg, gq, slot);
  if (slot >= row_count(a, b)) return;
  const int qgi = tile / a.q_per_wg, t = tile % a.q_per_wg;
  float M = -INFINITY, S = 0.0f;
  floatx4 o0 = {0.f, 0.f, 0.f, 0.f}, o1 = o0;
  constexpr int MB = 4;  // chunks whose loads are in flight together
  for (int c0 = 0; c0 < nch; c0 += MB) {
    float2 ml[MB];
    floatx4 v0[MB], v1[MB];
#pragma unroll
    for (int u = 0; u < MB; ++u) {
      const int c = min(c0 + u, nch - 1);
      const size_t row = ((((size_t)(u0 + c) * a.kv.heads + kvh) * a.groups + qgi) * a.q_per_wg + t) * 16 + qloc;
      ml[u] = *reinterpret_cast<const float2*>(a.part_ml + 2 * row);
      v0[u] = *reinterpret_cast<const floatx4*>(a.part_o + row * HD + 8 * c8);
      v1[u] = *reinterpret_cast<const floatx4*>(a.part_o + row * HD + 8 * c8 + 4);
    }
#pragma unroll
    for (int u = 0; u < MB; ++u) {
      if (c0 + u >= nch || ml[u].x == -INFINITY) continue;
      const float Mn = fmaxf(M, ml[u].x);
      const float fa = M == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(M - Mn);
      const float fb = __builtin_amdgcn_exp2f(ml[u].x - Mn);
      S = S * fa + ml[u].y * fb;
      o0 = o0 * fa + v0[u] * fb;
      o1 = o1 * fa + v1[u] * fb;
      M = Mn;
    }
  }
  const float inv = S != 0.0f ? 1.0f / S : 0.0f;
  const float y[8] = {o0[0] * inv, o0[1] * inv, o0[2] * inv, o0[3] * inv, o1[0] * inv, o1[1] * inv, o1[2] * inv, o1[3] * inv};
  write_output(a, b, kvh * G + gq, slot, 8 * c8, y);
}

}  // namespace

hipError_t launch_paged_attention(bool fp8, const PagedAttnArgs& a, const Topo& topo, hipStream_t s) {
  const int64_t wgs = (int64_t)(a.wgs > 0 ? a.wgs : a.batch) * a.kv.heads * a.groups;
  if (wgs > 0x7FFFFFFF / 512 || a.q_per_wg < 1 || a.q_per_wg > paged_max_tiles(fp8, a.kv.head_dim) || (a.wgs > 0 && a.batch > kPagedPlanBatch))
    return hipErrorInvalidValue;
  const dim3 grid((uint32_t)wgs);
  if (a.kv.head_dim == 128) {
    if (fp8) launch_paged_fp8_128(a, topo, grid, s);
    else launch_paged_bf16_128(a, topo, grid, s);
  } else {
    if (fp8) launch_paged_fp8_64(a, topo, grid, s);
    else launch_paged_bf16_64(a, topo, grid, s);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.wgs == 0) return e;
  const dim3 merge((uint32_t)((int64_t)a.batch * a.kv.heads * a.groups * a.q_per_wg));
  if (a.kv.head_dim == 128) hipLaunchKernelGGL(paged_merge_kernel<128>, merge, dim3(256), 0, s, a);
  else hipLaunchKernelGGL(paged_merge_kernel<64>, merge, dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace msd
