// Device helpers of the sampler: a row's parameters, the value order, masses.
#pragma once
#include "kernels.h"

namespace msd {

// A logit as it is ranked: NaN as -inf, +inf as the largest fp32 ...
__device__ __forceinline__ float bounded(float z) { return z != z ? -INFINITY : fminf(z, 3.402823466e38f); }
// ... and -0 as +0 (ordered_bits would rank it below).
__device__ __forceinline__ float clean(float z) { return bounded(z) + 0.0f; }
constexpr uint32_t kDead = 0x007FFFFFu;  // ordered_bits(-inf)

// What a row asks for. A filter that is off keeps everything: k = 2^32 - 1, p = 1,
// min_p = 0.
struct Request {
  double c;          // 32 log2(e) / T
  double p, min_p, u;
  uint32_t k;
  __device__ bool filtered() const { return k != 0xFFFFFFFFu || p < 1.0 || min_p > 0.0; }
};
__device__ __forceinline__ Request request_of(const SampleArgs& a, int row) {
  Request r;
  const float T = a.temperature ? a.temperature[row] : 1.0f;
  const int k = a.top_k ? a.top_k[row] : 0;
  const float p = a.top_p ? a.top_p[row] : 1.0f;
  const float m = a.min_p ? a.min_p[row] : 0.0f;
  const float u = a.u[row];
  r.k = k > 0 ? (uint32_t)k : 0xFFFFFFFFu;
  r.c = 32 * 1.4426950408889634 / (double)T;
  if (!(T > 0.0f)) r.c = 32 * 1.4426950408889634, r.k = 1;  // greedy
  r.p = p == p ? (double)p : 1.0;
  r.min_p = m > 0.0f ? (double)m : 0.0;
  r.u = u >= 0.0f ? (double)fminf(u, 0.99999994f) : 0.0;  // below one
  return r;
}

// Distance of a logit below the largest in 32nds of an octave, <= 0.
__device__ __forceinline__ double exponent_of(float z, float top, double c) { return ((double)z - (double)top) * c; }

// 2^(j / 32), j < 32: the Taylor series of exp, whose 17th power is under 2^-57 of the sum
__device__ __forceinline__ double octave_part(int j) {
  const double x = (double)j * (0.6931471805599453 / 32);
  double p = 1.0;
#pragma unroll
  for (int k = 16; k > 0; --k) p = fma(p, x * (1.0 / k), 1.0);
  return p;
}

// 2^(t / 32 + shift), t <= 0, as p * scale: t = n + x, |x| <= 1/2; 2^(x / 32) by its series to
// the 5th power (the 6th is under 2^-48), the table's entry n mod 32 with n div 32 added to
// its exponent. n by adding 1.5 2^52, whose last bits are then its integer.
struct Exp2 {
  double p, scale;
};
__device__ __forceinline__ Exp2 exp2_of(const double* parts, double t, int shift) {
  constexpr double l = 0.6931471805599453 / 32;
  t = fmax(t, -32000.0);
  const double r = t + 0x1.8p52;
  const int n = (int)(uint32_t)__double_as_longlong(r);
  const double x = t - (r - 0x1.8p52);
  double p = l * l * l * l * l / 120.0;
  p = fma(p, x, l * l * l * l / 24.0);
  p = fma(p, x, l * l * l / 6.0);
  p = fma(p, x, l * l / 2.0);
  p = fma(p, x, l);
  p = fma(p, x, 1.0);
  const uint64_t e = (uint64_t)__double_as_longlong(parts[n & 31]) + ((uint64_t)(uint32_t)((n >> 5) + shift) << 52);
  return {p, __longlong_as_double((long long)e)};
}
__device__ __forceinline__ double exp2_64(const double* parts, double t) {
  const Exp2 e = exp2_of(parts, t, 0);
  return e.p * e.scale;
}
// Mass of a token: in units of 2^-43, to nearest (added to 2^52, the units are the mantissa).
__device__ __forceinline__ uint64_t mass_of(const double* parts, double t) {
  const Exp2 e = exp2_of(parts, t, 43);
  return __double_as_longlong(fma(e.p, e.scale, 0x1p52)) - 0x4330000000000000ull;
}

}  // namespace msd
