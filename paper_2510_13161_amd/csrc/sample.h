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

struct Params {
  double T, p, min_p, u;
  uint32_t k;
};
__device__ __forceinline__ Params params_of(const SampleArgs& a, int row) {
  Params r;
  const float T = a.temperature ? a.temperature[row] : 1.0f;
  const int k = a.top_k ? a.top_k[row] : 0;
  const float p = a.top_p ? a.top_p[row] : 1.0f;
  const float m = a.min_p ? a.min_p[row] : 0.0f;
  const float u = a.u[row];
  r.k = k > 0 ? (uint32_t)k : 0xFFFFFFFFu;
  r.T = (double)T;
  if (!(T > 0.0f)) r.T = 1.0, r.k = 1;  // greedy
  r.p = p == p ? (double)p : 1.0;
  r.min_p = m > 0.0f ? (double)m : 0.0;
  r.u = u >= 0.0f ? (double)fminf(u, 0.99999994f) : 0.0;  // below one
  return r;
}

// exp((z - max) / T) in units of 2^-43
__device__ __forceinline__ uint64_t mass_of(float z, double ref, double T) {
  return (uint64_t)(exp(((double)z - ref) / T) * 0x1p43 + 0.5);
}
__device__ __forceinline__ bool over_min(float z, double ref, double T, double min_p) {
  return exp(((double)z - ref) / T) >= min_p;
}

}  // namespace msd
