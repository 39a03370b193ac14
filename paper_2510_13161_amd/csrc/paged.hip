// Paged cache: append and commit.
//
// A wave owns one block of 16 tokens of one (layer, sequence, kv head) of k
// or v: at most 16 rows of head_dim. Rows of keys are rotated in fp32 (a c -
// b s, b c + a s); bf16 pages take them rounded once. 8-bit pages: the block's
// scale is 2^e, e the smallest with amax <= 448 2^e over the new rows and, where
// the block already holds committed rows, never below the scale they have;
// where it grows, their codes are decoded, multiplied by the ratio (a power of
// two: exact but for codes that fall below 2^-6) and coded again. Everything
// that a block needs sits in one wave's registers, so no wave waits for another.
#include "paged.h"

namespace msd {
namespace {

// rows of sequence b that this call stores; 0 where it must leave the sequence
// alone (bad_capacity: it would pass the page table)
__device__ __forceinline__ int append_count(const AppendArgs& a, int b, int64_t L, bool* bad_capacity) {
  int n = a.n_rows;
  if (a.acc_len) {
    const int A = a.acc_len[b];
    n = A < 0 || A >= a.n_rows ? 0 : A + 1;
  } else if (a.count) {
    n = min(max(a.count[b], 0), a.n_rows);
  }
  *bad_capacity = L < 0 || L + n > a.kv.capacity;
  return *bad_capacity ? 0 : n;
}

template <int HD, bool FP8>
__global__ __launch_bounds__(256) void append_kernel(AppendArgs a, int n_blocks) {
  constexpr int C8 = HD / 8;        // 8-dim groups of a row
  constexpr int RPI = 64 / C8;      // rows of an iteration
  constexpr int IT = 16 / RPI;      // iterations of a block
  const int lane = threadIdx.x & 63;
  int64_t item = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int which = (int)(item & 1);  // 0 keys, 1 values
  item >>= 1;
  const int h = (int)(item % a.kv.heads);
  item /= a.kv.heads;
  const int j = (int)(item % n_blocks);
  item /= n_blocks;
  const int b = (int)(item % a.batch);
  const int l = (int)(item / a.batch);
  if (l >= a.n_layers) return;
  const int64_t L = a.kv.len[b];
  bool bad;
  const int n = append_count(a, b, L, &bad);
  if (bad && j == 0 && h == 0 && which == 0 && l == 0 && lane == 0) atomicOr(a.kv.status, 1u);
  if (n == 0) return;
  const int64_t t0 = (L / kScaleTokens + j) * kScaleTokens;  // first position of the block
  if (t0 >= L + n) return;
  const int page = a.kv.page_table[(size_t)b * a.kv.max_pages + (size_t)(t0 >> a.kv.page_shift)];
  if (page < 0 || page >= a.kv.n_pages) {
    if (h == 0 && which == 0 && l == 0 && lane == 0) atomicOr(a.kv.status, 8u);
    return;
  }
  const int page_size = 1 << a.kv.page_shift;
  const int off = (int)(t0 & (page_size - 1));
  const size_t plane = ((size_t)(a.layer + l) * a.kv.n_pages + page) * a.kv.heads + h;
  const size_t row0 = (plane * page_size + off) * HD;  // first element of the block
  const uint16_t* src = (which ? a.v : a.k) + l * a.layer_stride + b * a.seq_stride + h * a.head_stride;
  const RopeView rp = which ? RopeView{nullptr, 0, 0} : a.rope;
  const int c = lane % C8;

  // new rows of this lane, fp32
  float x[IT][8];
  bool now[IT];
#pragma unroll
  for (int it = 0; it < IT; ++it) {
    const int64_t pos = t0 + it * RPI + lane / C8;
    now[it] = pos >= L && pos < L + n;
#pragma unroll
    for (int i = 0; i < 8; ++i) x[it][i] = 0.0f;
    if (now[it]) {
      int r = (int)(pos - L);
      if (a.path) r = min(max(a.path[(size_t)b * a.n_rows + r], 0), a.n_rows - 1);
      load_rotated8(src + r * a.row_stride, c, rp, pos, x[it]);
    }
  }
  if constexpr (!FP8) {
    uint16_t* dst = static_cast<uint16_t*>(which ? a.kv.v : a.kv.k) + row0;
#pragma unroll
    for (int it = 0; it < IT; ++it)
      if (now[it])
        *reinterpret_cast<bf16x8*>(dst + (it * RPI + lane / C8) * HD + 8 * c) = round_vals(x[it]);
  } else {
    uint8_t* dst = static_cast<uint8_t*>(which ? a.kv.v : a.kv.k) + row0;
    uint8_t* sc = (which ? a.kv.v_scale : a.kv.k_scale) + plane * (page_size / kScaleTokens) + off / kScaleTokens;
    float amax = 0.0f;
#pragma unroll
    for (int it = 0; it < IT; ++it)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float m = fabsf(x[it][i]);
        amax = m <= 3.402823466e38f ? fmaxf(amax, m) : amax;  // infinities and NaN left out
      }
    amax = wave_max(amax);
    const uint32_t was = *sc;
    const bool held = t0 < L;  // committed rows in the block
    uint32_t e = scale_exponent(amax);
    if (held) e = max(e, was);
    const float inv = __uint_as_float(e < 254u ? (254u - e) << 23 : 0x00400000u);  // 2^(127 - e)
#pragma unroll
    for (int it = 0; it < IT; ++it) {
      u32x2* at = reinterpret_cast<u32x2*>(dst + (it * RPI + lane / C8) * HD + 8 * c);
      if (now[it]) {
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = clamp_code(x[it][i] * inv);
        *at = u32x2{encode4(y[0], y[1], y[2], y[3]), encode4(y[4], y[5], y[6], y[7])};
      } else if (held && e > was && t0 + it * RPI + lane / C8 < L) {
        const float f = exp2_int((int)was - (int)e);
        u32x2 w = *at;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float y[4];
          decode4(w[i], y);
          w[i] = encode4(y[0] * f, y[1] * f, y[2] * f, y[3] * f);
        }
        *at = w;
      }
    }
    if (lane == 0) *sc = (uint8_t)e;
  }
}

__global__ void advance_kernel(AppendArgs a) {
  const int b = blockIdx.x * blockDim.x + threadIdx.x;
  if (b >= a.batch) return;
  bool bad;
  a.kv.len[b] += append_count(a, b, a.kv.len[b], &bad);
}

}  // namespace

hipError_t launch_paged_append(bool fp8, const AppendArgs& a, hipStream_t s) {
  const int n_blocks = (a.n_rows + 14) / 16 + 1;  // n rows touch that many 16-token blocks at most
  const int64_t waves = (int64_t)a.n_layers * a.batch * n_blocks * a.kv.heads * 2;
  const int64_t wgs = (waves + 3) / 4;
  if (wgs > 0x7FFFFFFF / 256) return hipErrorInvalidValue;
  const dim3 grid((uint32_t)wgs), block(256);
  if (a.kv.head_dim == 128) {
    if (fp8) hipLaunchKernelGGL((append_kernel<128, true>), grid, block, 0, s, a, n_blocks);
    else hipLaunchKernelGGL((append_kernel<128, false>), grid, block, 0, s, a, n_blocks);
  } else {
    if (fp8) hipLaunchKernelGGL((append_kernel<64, true>), grid, block, 0, s, a, n_blocks);
    else hipLaunchKernelGGL((append_kernel<64, false>), grid, block, 0, s, a, n_blocks);
  }
  return hipGetLastError();
}

hipError_t launch_paged_advance(const AppendArgs& a, hipStream_t s) {
  hipLaunchKernelGGL(advance_kernel, dim3((a.batch + 63) / 64), dim3(64), 0, s, a);
  return hipGetLastError();
}

}  // namespace msd
