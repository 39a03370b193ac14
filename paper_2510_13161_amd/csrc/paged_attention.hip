// Attention of a block's rows over the paged cache.
//
// A wave owns one (sequence, query head, slot). It walks the visible keys 64 at
// a time: each lane takes the dot product of its key with the rotated query,
// the wave keeps a running maximum m and sum s of exp(score - m) (the output
// rescaled when m rises), and the lanes then gather the values of the tile's
// visible keys, each its dims.
#include "paged.h"

namespace msd {
namespace {

template <int HD, bool FP8>
__global__ __launch_bounds__(64) void paged_attn_kernel(PagedAttnArgs a) {
  __shared__ float qs[HD];
  __shared__ float ps[64];
  const int lane = threadIdx.x;
  const int slot = blockIdx.x % a.n_slots, h = blockIdx.x / a.n_slots, b = blockIdx.y;
  const int kvh = h / (a.n_heads / a.kv.heads);
  const int cnt = a.count ? min(max(a.count[b], 0), a.n_slots) : a.n_slots;
  const int64_t L = a.kv.len[b];
  if (L < 0 || L + a.n_slots > a.kv.capacity) {
    if (blockIdx.x == 0 && lane == 0) atomicOr(a.kv.status, 1u);
    return;
  }
  if (slot >= cnt) return;
  const int64_t P = L + a.topo.depth[slot];
  if (lane < HD / 8) {
    float v[8];
    load_rotated8(a.q + b * a.q_seq + slot * a.q_row + h * a.q_head, lane, a.rope, P, v);
    for (int i = 0; i < 8; ++i) qs[8 * lane + i] = v[i];
  }
  __syncthreads();
  const int page_size = 1 << a.kv.page_shift;
  const int64_t cached = a.k_new ? L : P + 1;
  const int64_t total = cached + (a.k_new ? slot + 1 : 0);
  float m = -INFINITY, sum = 0.0f, o[HD / 64];
  for (int i = 0; i < HD / 64; ++i) o[i] = 0.0f;
  const size_t heads0 = (size_t)a.layer * a.kv.n_pages;
  auto page_of = [&](int64_t pos) {
    const int pg = a.kv.page_table[(size_t)b * a.kv.max_pages + (size_t)(pos >> a.kv.page_shift)];
    return pg >= 0 && pg < a.kv.n_pages ? pg : -1;
  };
  for (int64_t t0 = 0; t0 < total; t0 += 64) {
    const int64_t t = t0 + lane;
    bool vis = false;
    float sc = -INFINITY;
    if (t < cached) {
      vis = a.window <= 0 || P - t < a.window || t < a.sinks;
      if (vis) {
        const int pg = page_of(t);
        if (pg < 0) {
          atomicOr(a.kv.status, 8u);
          vis = false;
        } else {
          const size_t plane = (heads0 + pg) * a.kv.heads + kvh;
          const int off = (int)(t & (page_size - 1));
          const size_t at = (plane * page_size + off) * HD;
          float acc = 0.0f, f = a.scale;
          for (int c = 0; c < HD / 8; ++c) {
            float k[8];
            if constexpr (FP8) {
              const u32x2 w = *reinterpret_cast<const u32x2*>(static_cast<const uint8_t*>(a.kv.k) + at + 8 * c);
              float k0[4], k1[4];
              decode4(w[0], k0);
              decode4(w[1], k1);
              for (int i = 0; i < 4; ++i) k[i] = k0[i], k[4 + i] = k1[i];
            } else {
              load8(static_cast<const uint16_t*>(a.kv.k) + at + 8 * c, k);
            }
            for (int i = 0; i < 8; ++i) acc += qs[8 * c + i] * k[i];
          }
          if constexpr (FP8) f *= scale_value(a.kv.k_scale[plane * (page_size / kScaleTokens) + off / kScaleTokens]);
          sc = acc * f;
        }
      }
    } else if (t < total) {
      const int j = (int)(t - cached);
      const int64_t pj = L + a.topo.depth[j];
      vis = ((a.topo.anc[slot] >> j) & 1ull) && (a.window <= 0 || P - pj < a.window || pj < a.sinks);
      if (vis) {
        float acc = 0.0f;
        for (int c = 0; c < HD / 8; ++c) {
          float k[8];
          load_rotated8(a.k_new + b * a.new_seq + j * a.new_row + kvh * a.new_head, c, a.rope, pj, k);
          for (int i = 0; i < 8; ++i) acc += qs[8 * c + i] * k[i];
        }
        sc = acc * a.scale;
      }
    }
    const unsigned long long any = __ballot(vis);
    if (!any) continue;
    const float mt = wave_max(vis ? sc : -INFINITY);
    const float mn = fmaxf(m, mt);
    const float alpha = m == -INFINITY ? 0.0f : __expf(m - mn);
    const float ref = mn == -INFINITY ? 0.0f : mn;  // every score -inf
    const float p = vis ? expf(sc - ref) : 0.0f;
    sum = sum * alpha + wave_sum(p);
    m = mn;
    for (int i = 0; i < HD / 64; ++i) o[i] *= alpha;
    __syncthreads();
    ps[lane] = p;
    __syncthreads();
    for (int k = 0; k < 64; ++k) {
      if (!((any >> k) & 1ull)) continue;
      const int64_t tk = t0 + k;
      float f = ps[k];
      if (tk < cached) {
        const size_t plane = (heads0 + page_of(tk)) * a.kv.heads + kvh;
        const int off = (int)(tk & (page_size - 1));
        const size_t at = (plane * page_size + off) * HD;
        if constexpr (FP8) f *= scale_value(a.kv.v_scale[plane * (page_size / kScaleTokens) + off / kScaleTokens]);
        for (int i = 0; i < HD / 64; ++i) {
          float v;
          if constexpr (FP8) {
            const int code = static_cast<const uint8_t*>(a.kv.v)[at + lane + 64 * i];
            v = __builtin_amdgcn_cvt_pk_f32_fp8(code, false)[0];
          } else {
            v = bf2f(static_cast<const uint16_t*>(a.kv.v)[at + lane + 64 * i]);
          }
          o[i] += f * v;
        }
      } else {
        const uint16_t* row = a.v_new + b * a.new_seq + (tk - cached) * a.new_row + kvh * a.new_head;
        for (int i = 0; i < HD / 64; ++i) o[i] += f * bf2f(row[lane + 64 * i]);
      }
    }
  }
  uint16_t* dst = a.out + b * a.out_seq + slot * a.out_row + h * a.out_head;
  const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
  for (int i = 0; i < HD / 64; ++i) dst[lane + 64 * i] = f2bf(o[i] * inv);
}

}  // namespace

hipError_t launch_paged_attention(bool fp8, const PagedAttnArgs& a, hipStream_t s) {
  const dim3 grid(a.n_heads * a.n_slots, a.batch), block(64);
  if (a.kv.head_dim == 128) {
    if (fp8) hipLaunchKernelGGL((paged_attn_kernel<128, true>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((paged_attn_kernel<128, false>), grid, block, 0, s, a);
  } else {
    if (fp8) hipLaunchKernelGGL((paged_attn_kernel<64, true>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((paged_attn_kernel<64, false>), grid, block, 0, s, a);
  }
  return hipGetLastError();
}

}  // namespace msd
