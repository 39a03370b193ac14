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
//
// What bounds it: of few rows the chain length, page number, row, scale, store (16 tokens
// of one layer 3.3 us; the accepted paths of 7 trees, 48 layers, 10 MB: 11.7 us, as the
// grid covers every slot that could be accepted); of many the bytes (14K rows, 8
// heads, to 8 bits: 101 MB in 25.5 us, 4 TB/s). A workgroup a whole page, through
// LDS, would read and write no byte less.
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

// The 8 dims of a row that a lane holds, as two groups of 4: of rotated keys in the
// half layout the two halves of 4 pairs (no lane needs another's dims, and a pair's
// (cos, sin) is read once), else 8 in a row.
struct Dims {
  int d0, d1;
  bool turned;
};
__device__ __forceinline__ Dims dims_of(int c, const RopeView& rp) {
  if (rp.table && 8 * c < rp.rd) {
    if (rp.interleaved) return {8 * c, 8 * c + 4, true};
    return {4 * c, rp.rd / 2 + 4 * c, true};
  }
  return {8 * c, 8 * c + 4, false};
}
__device__ __forceinline__ void unpack4(u32x2 w, float* v) {
  v[0] = bf_lo(w[0]);
  v[1] = bf_hi(w[0]);
  v[2] = bf_lo(w[1]);
  v[3] = bf_hi(w[1]);
}
// Rotates a lane's 4 pairs by their table entries: each product and difference
// rounded by itself, as load_rotated8 does.
__device__ __forceinline__ void turn(float (&v)[8], const float2* cs, bool interleaved) {
#pragma clang fp contract(off)
  float2 f[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) f[i] = cs[i];
  if (interleaved) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float a = v[2 * i], b = v[2 * i + 1];
      v[2 * i] = a * f[i].x - b * f[i].y;
      v[2 * i + 1] = b * f[i].x + a * f[i].y;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float a = v[i], b = v[4 + i];
      v[i] = a * f[i].x - b * f[i].y;
      v[4 + i] = b * f[i].x + a * f[i].y;
    }
  }
}

template <int HD, bool FP8>
__global__ __launch_bounds__(256) void append_kernel(AppendArgs a, int n_blocks) {
  constexpr int C8 = HD / 8;        // lanes of a row
  constexpr int RPI = 64 / C8;      // rows of an iteration
  constexpr int IT = 16 / RPI;      // iterations of a block
  const int lane = threadIdx.x & 63;
  const int item = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
  const int which = item & 1;  // 0 keys, 1 values
  const int h = (item >> 1) % a.kv.heads, j = (item >> 1) / a.kv.heads;
  const int b = blockIdx.y, l = blockIdx.z;
  if (j >= n_blocks) return;
  const int64_t L = a.kv.len[b];
  bool bad;
  const int n = append_count(a, b, L, &bad);
  if (bad && item == 0 && l == 0 && lane == 0) atomicOr(a.kv.status, 1u);
  if (n == 0) return;
  const int64_t t0 = (L / kScaleTokens + j) * kScaleTokens;  // first position of the block
  if (t0 >= L + n) return;
  const int c = lane % C8, rl = lane / C8;
  const RopeView rp = which ? RopeView{nullptr, 0, 0} : a.rope;
  const Dims d = dims_of(c, rp);

  // the page's number and the rows are on their way together, then the block's scale
  const int page = a.kv.page_table[(size_t)b * a.kv.max_pages + (size_t)(t0 >> a.kv.page_shift)];
  const uint16_t* src = (which ? a.v : a.k) + l * a.layer_stride + b * a.seq_stride + h * a.head_stride;
  const int first = (int)(t0 - L);  // row of the block's first place, negative where it is held
  bool now[IT];
  float x[IT][8];
#pragma unroll
  for (int it = 0; it < IT; ++it) {
    int r = first + it * RPI + rl;
    now[it] = r >= 0 && r < n;
#pragma unroll
    for (int i = 0; i < 8; ++i) x[it][i] = 0.0f;
    if (now[it]) {
      const int64_t pos = L + r;
      if (a.path) r = min(max(a.path[(size_t)b * a.n_rows + r], 0), a.n_rows - 1);
      const uint16_t* row = src + r * a.row_stride;
      unpack4(*reinterpret_cast<const u32x2*>(row + d.d0), x[it]);
      unpack4(*reinterpret_cast<const u32x2*>(row + d.d1), x[it] + 4);
      if (d.turned) turn(x[it], rp.table + pos * (rp.rd / 2) + 4 * c, rp.interleaved != 0);
    }
  }
  const bool paged = page >= 0 && page < a.kv.n_pages;
  const size_t plane = ((size_t)(a.layer + l) * a.kv.n_pages + (paged ? page : 0)) * a.kv.heads + h;
  const size_t row0 = (plane << a.kv.page_shift) + (size_t)(t0 & ((1 << a.kv.page_shift) - 1));  // first row of the block
  const bool held = first < 0;  // committed rows in the block
  uint8_t* sc = (which ? a.kv.v_scale : a.kv.k_scale) + (row0 >> 4);
  const uint32_t was = FP8 && held ? *sc : 0;
  if (!paged) {
    if (h == 0 && which == 0 && l == 0 && lane == 0) atomicOr(a.kv.status, 8u);
    return;
  }

  if constexpr (!FP8) {
    uint16_t* dst = static_cast<uint16_t*>(which ? a.kv.v : a.kv.k) + row0 * HD;
#pragma unroll
    for (int it = 0; it < IT; ++it)
      if (now[it]) {
        uint16_t* at = dst + (it * RPI + rl) * HD;
        const u32x2 lo = {pack_bf16x2(x[it][0], x[it][1]), pack_bf16x2(x[it][2], x[it][3])};
        const u32x2 hi = {pack_bf16x2(x[it][4], x[it][5]), pack_bf16x2(x[it][6], x[it][7])};
        *reinterpret_cast<u32x2*>(at + d.d0) = lo;
        *reinterpret_cast<u32x2*>(at + d.d1) = hi;
      }
  } else {
    uint8_t* dst = static_cast<uint8_t*>(which ? a.kv.v : a.kv.k) + row0 * HD;
    float amax = 0.0f;
#pragma unroll
    for (int it = 0; it < IT; ++it)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float m = fabsf(x[it][i]);
        amax = m <= 3.402823466e38f ? fmaxf(amax, m) : amax;  // infinities and NaN left out
      }
    amax = wave_max(amax);
    const uint32_t e = max(scale_exponent(amax), was);
    const float inv = __uint_as_float(e < 254u ? (254u - e) << 23 : 0x00400000u);  // 2^(127 - e)
#pragma unroll
    for (int it = 0; it < IT; ++it) {
      uint8_t* at = dst + (it * RPI + rl) * HD;
      if (now[it]) {
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = clamp_code(x[it][i] * inv);
        *reinterpret_cast<uint32_t*>(at + d.d0) = encode4(y[0], y[1], y[2], y[3]);
        *reinterpret_cast<uint32_t*>(at + d.d1) = encode4(y[4], y[5], y[6], y[7]);
      } else if (held && e > was && first + it * RPI + rl < 0) {
        const float f = exp2_int((int)was - (int)e);
        u32x2 w = *reinterpret_cast<u32x2*>(at + 8 * c);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float y[4];
          decode4(w[i], y);
          w[i] = encode4(y[0] * f, y[1] * f, y[2] * f, y[3] * f);
        }
        *reinterpret_cast<u32x2*>(at + 8 * c) = w;
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
  const dim3 grid((uint32_t)(((int64_t)n_blocks * a.kv.heads + 1) / 2), a.batch, a.n_layers), block(256);
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
