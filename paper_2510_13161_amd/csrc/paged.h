// Device helpers of the paged cache: rotation, 8-bit block codes.
#pragma once
#include "kernels.h"

namespace msd {

typedef float floatx2 __attribute__((ext_vector_type(2)));

// Inclusive scan of a wave by lane moves inside the vector unit: rows of 16 lanes
// shifted by 1, 2, 4 and 8, then the last lane of a row given to the next row, and
// that of the lower half to the upper. Lanes without a source take 0.
__device__ __forceinline__ int wave_scan_add(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);
  return v + __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);
}
__device__ __forceinline__ int wave_max_nonneg(int v) {
  v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false));
  v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false));
  v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false));
  v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false));
  v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false));
  return __builtin_amdgcn_readlane(max(v, __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false)), 63);
}

// 2^(scale - 127), a biased scale exponent's factor (0 is 2^-127, a subnormal)
__device__ __forceinline__ float scale_value(uint32_t e) {
  return __uint_as_float(e ? e << 23 : 0x00400000u);
}

// Biased exponent of the smallest power of two 2^e, e >= -127, with
// amax <= 448 * 2^e: 448 = 1.75 * 2^8, so e = x - 8 for amax = m * 2^x with
// m <= 1.75, else x - 7. Below 2^-119 (subnormals too) that is under -127.
__device__ __forceinline__ uint32_t scale_exponent(float amax) {
  const uint32_t u = __float_as_uint(amax);
  const int e = (int)(u >> 23) - 8 + ((u & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return (uint32_t)max(e, 0);
}

// 2^d for an integer d <= 0 (0 below the subnormals)
__device__ __forceinline__ float exp2_int(int d) { return ldexpf(1.0f, d); }

__device__ __forceinline__ float clamp_code(float y) {
  return y != y ? y : fminf(fmaxf(y, -kCodeMax), kCodeMax);  // NaN stays
}
// four values (magnitudes at most 448, or NaN) as four e4m3 codes, to nearest even
__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d) {
  const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, lo, true);
}
__device__ __forceinline__ void decode4(uint32_t w, float (&v)[4]) {
  const floatx2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false);
  const floatx2 hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  v[0] = lo[0];
  v[1] = lo[1];
  v[2] = hi[0];
  v[3] = hi[1];
}

__device__ __forceinline__ void load8(const uint16_t* p, float (&v)[8]) {
  const u32x4 w = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = bf_lo(w[i]);
    v[2 * i + 1] = bf_hi(w[i]);
  }
}

// Dims 8 c .. 8 c + 7 of a bf16 row, rotated at `pos` where they lie in the
// rotated part: each product and difference rounded to fp32 by itself, so
// the values do not depend on how a kernel schedules them.
__device__ __forceinline__ void load_rotated8(const uint16_t* row, int c, const RopeView& rp, int64_t pos,
                                              float (&v)[8]) {
#pragma clang fp contract(off)
  load8(row + 8 * c, v);
  if (!rp.table || 8 * c >= rp.rd) return;
  const float2* cs = rp.table + pos * (rp.rd / 2);
  if (rp.interleaved) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = cs[4 * c + i];
      const float a = v[2 * i], b = v[2 * i + 1];
      v[2 * i] = a * f.x - b * f.y;
      v[2 * i + 1] = b * f.x + a * f.y;
    }
    return;
  }
  const int h8 = rp.rd / 16;  // 8-dim groups of a half
  const bool up = c >= h8;
  const int cl = up ? c - h8 : c;
  float w[8];
  load8(row + 8 * (up ? cl : c + h8), w);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float2 f = cs[8 * cl + i];
    v[i] = up ? v[i] * f.x + w[i] * f.y : v[i] * f.x - w[i] * f.y;
  }
}

}  // namespace msd
