// Device helpers of the sampler: a row's parameters, the value order, masses.
#pragma once
#include "kernels.h"

namespace msd {

// A logit as it is ranked: NaN as -inf, +inf as the largest fp32, -0 as +0
// (ordered_bits would rank it below).
__device__ __forceinline__ float clean(float z) {
  z = z != z ? -INFINITY : z;
  return fminf(z, 3.402823466e38f) + 0.0f;
}
constexpr uint32_t kDead = 0x007FFFFFu;  // ordered_bits(-inf)

// What a row asks for. A filter that is off keeps everything: k = 2^32 - 1, p = 1,
// min_p = 0.
struct Request {
  double c;          // log2(e) / T
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
  r.c = 1.4426950408889634 / (double)T;
  if (!(T > 0.0f)) r.c = 1.4426950408889634, r.k = 1;  // greedy
  r.p = p == p ? (double)p : 1.0;
  r.min_p = m > 0.0f ? (double)m : 0.0;
  r.u = u >= 0.0f ? (double)fminf(u, 0.99999994f) : 0.0;  // below one
  return r;
}

// Distance of a logit below the largest in base-2 units, <= 0.
__device__ __forceinline__ double exponent_of(float z, float top, double c) { return ((double)z - (double)top) * c; }

// 2^(t + shift) for t <= 0: 2^f, |f| <= 1/2, by its Taylor series to the 11th
// power (the 12th is under 2^-47 of the sum), the rest in the exponent.
__device__ __forceinline__ double exp2_64(double t, int shift) {
  t = fmax(t, -1000.0);
  const double n = rint(t), x = (t - n) * 0.6931471805599453;
  double p = 1.0 / 39916800.0;
  p = fma(p, x, 1.0 / 3628800.0);
  p = fma(p, x, 1.0 / 362880.0);
  p = fma(p, x, 1.0 / 40320.0);
  p = fma(p, x, 1.0 / 5040.0);
  p = fma(p, x, 1.0 / 720.0);
  p = fma(p, x, 1.0 / 120.0);
  p = fma(p, x, 1.0 / 24.0);
  p = fma(p, x, 1.0 / 6.0);
  p = fma(p, x, 0.5);
  p = fma(p, x, 1.0);
  p = fma(p, x, 1.0);
  return ldexp(p, (int)n + shift);
}

// Mass of a token: 2^t in units of 2^-43, to nearest (added to 2^52, the units are the mantissa).
__device__ __forceinline__ uint64_t mass_of(double t) {
  return __double_as_longlong(exp2_64(t, 43) + 0x1p52) - 0x4330000000000000ull;
}

}  // namespace msd
