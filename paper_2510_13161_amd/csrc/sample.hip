// Sampling under temperature, top-k, top-p and min-p from given uniforms.
//
// Tokens are ranked by (logit descending, id ascending); every filter keeps a
// prefix of that order, so the kept set is the ids with (z, id) at or above one
// threshold. Masses exp((z - max) / T) are fp64 values rounded to multiples of
// 2^-43: integer sums, the same in any order, so that histograms may be
// filled with atomics and a run repeats bit for bit (2^20 tokens of mass one
// fill 2^63). A workgroup owns a row. The threshold is found digit by digit of the
// ordered fp32 bits (11, 11 and 10): a histogram of counts and masses of the
// tokens that share the digits so far, then the digit at which the running
// count reaches top_k, or the running mass top_p of the total. Equal logits at
// the threshold are cut in id order.
#include "sample.h"

namespace msd {
namespace {

constexpr int kThreads = 1024;
constexpr int kBins = 2048;

struct Shared {
  uint32_t cnt[kBins];
  uint64_t mass[kBins];
  uint64_t wave[kThreads / 64];
  uint32_t wave_max[kThreads / 64];
  uint64_t above_mass;
  uint64_t mass_sel;
  uint32_t above_cnt, cnt_sel, bin, id;
};

struct Row {
  const float* z;
  int V, tid;
  double inv_ref, T;  // largest logit, temperature
};

__device__ uint64_t block_sum(Shared& sh, uint64_t v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh.wave[threadIdx.x >> 6] = v;
  __syncthreads();
  uint64_t t = 0;
  for (int w = 0; w < kThreads / 64; ++w) t += sh.wave[w];
  return t;
}

// Tokens whose ordered bits lie at or above lo ... are kept down to a cut: by
// count (the n-th) or by mass (before < want). Finds the key of the last kept
// logit, the number of kept tokens with exactly that logit, and the count and
// mass of all tokens above it.
struct Cut {
  uint32_t key;        // ordered bits of the threshold logit
  uint32_t ties;       // kept tokens with that logit
  uint32_t above;      // tokens above it
  uint64_t above_mass;
};

template <bool BY_MASS>
__device__ Cut find_cut(Shared& sh, const Row& r, uint64_t n, double want, uint32_t floor_key) {
  uint32_t prefix = 0, above = 0;
  uint64_t above_mass = 0;
  for (int level = 0; level < 3; ++level) {
    const int shift = level == 0 ? 21 : (level == 1 ? 10 : 0);
    const int bits = level == 2 ? 10 : 11;
    for (int i = r.tid; i < kBins; i += kThreads) sh.cnt[i] = 0, sh.mass[i] = 0;
    __syncthreads();
    for (int i = r.tid; i < r.V; i += kThreads) {
      const float z = clean(r.z[i]);
      const uint32_t k = ordered_bits(z);
      if (k <= kDead || (level && (k >> (shift + bits)) != prefix) || k < floor_key) continue;
      const uint32_t d = (k >> shift) & ((1u << bits) - 1);
      atomicAdd(&sh.cnt[d], 1u);
      if (BY_MASS) atomicAdd((unsigned long long*)&sh.mass[d], (unsigned long long)mass_of(z, r.inv_ref, r.T));
    }
    __syncthreads();
    if (r.tid == 0) {
      int d = (1 << bits) - 1, last = d;
      uint32_t c = above, c_last = above;
      uint64_t m = above_mass, m_last = above_mass;
      bool any = false;
      for (; d >= 0; --d) {
        if (!sh.cnt[d]) continue;
        const bool inside = BY_MASS ? (double)m < want || c == 0 : c < n;
        if (!inside) break;
        any = true;
        last = d, c_last = c, m_last = m;
        c += sh.cnt[d];
        m += sh.mass[d];
      }
      sh.bin = any ? last : 0;
      sh.above_cnt = c_last;
      sh.above_mass = m_last;
    }
    __syncthreads();
    prefix = (prefix << bits) | sh.bin;
    above = sh.above_cnt;
    above_mass = sh.above_mass;
    __syncthreads();
  }
  Cut c{prefix, 0, above, above_mass};
  // all with the threshold's logit: the last level's bin is one key
  const uint32_t equal = sh.cnt[prefix & 1023];
  if (BY_MASS) {
    const uint64_t one = mass_of(from_ordered_bits(prefix), r.inv_ref, r.T);
    uint32_t lo = 0, hi = equal;  // smallest t >= 1 with above + t * one >= want
    while (lo + 1 < hi) {
      const uint32_t mid = (lo + hi) / 2;
      if ((double)(above_mass + mid * one) < want) lo = mid;
      else hi = mid;
    }
    c.ties = hi;
  } else {
    c.ties = (uint32_t)(n - above < equal ? n - above : equal);
  }
  __syncthreads();
  return c;
}

// mass of the tokens above key, and the id of the t-th token with that key
__device__ uint32_t tie_id(Shared& sh, const Row& r, uint32_t key, uint32_t t) {
  // contiguous chunk of ids per thread, counted, prefixed, scanned
  const int per = (r.V + kThreads - 1) / kThreads;
  const int i0 = min(r.tid * per, r.V), i1 = min(i0 + per, r.V);
  uint32_t mine = 0;
  for (int i = i0; i < i1; ++i) mine += ordered_bits(clean(r.z[i])) == key;
  __syncthreads();
  sh.cnt[r.tid] = mine;
  __syncthreads();
  if (r.tid == 0) {
    uint32_t c = 0;
    for (int i = 0; i < kThreads; ++i) {
      const uint32_t x = sh.cnt[i];
      sh.cnt[i] = c;
      c += x;
    }
    sh.id = r.V - 1;
  }
  __syncthreads();
  uint32_t c = sh.cnt[r.tid];
  if (c < t && c + mine >= t)
    for (int i = i0; i < i1; ++i)
      if (ordered_bits(clean(r.z[i])) == key && ++c == t) sh.id = i;
  __syncthreads();
  const uint32_t id = sh.id;
  __syncthreads();
  return id;
}

__global__ __launch_bounds__(kThreads) void sample_kernel(SampleArgs a) {
  __shared__ Shared sh;
  const int row = blockIdx.x;
  Row r;
  r.z = a.logits + (int64_t)row * a.row_stride;
  r.V = a.vocab;
  r.tid = threadIdx.x;
  const Params p = params_of(a, row);
  uint32_t top = 0;
  for (int i = r.tid; i < r.V; i += kThreads) top = max(top, ordered_bits(clean(r.z[i])));
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
  if ((r.tid & 63) == 0) sh.wave_max[r.tid >> 6] = top;
  __syncthreads();
  for (int w = 0; w < kThreads / 64; ++w) top = max(top, sh.wave_max[w]);
  if (top <= kDead) {
    if (r.tid == 0) {
      a.tok[row] = -1;
      if (a.logp) a.logp[row] = -INFINITY;
      if (a.kept) a.kept[row] = 0;
    }
    return;
  }
  r.T = p.T;
  r.inv_ref = (double)from_ordered_bits(top);
  // threshold: (key, id of the last kept tie)
  uint32_t key = kDead + 1, last_id = 0xFFFFFFFFu;
  uint64_t total = 0;
  if (p.k < (uint32_t)r.V) {
    const Cut c = find_cut<false>(sh, r, p.k, 0.0, 0);
    key = c.key;
    last_id = tie_id(sh, r, c.key, c.ties);
  }
  auto kept = [&](int i, float z, uint32_t k) {
    return k > key || (k == key && (uint32_t)i <= last_id);
  };
  if (p.p < 1.0) {
    uint64_t m = 0;
    for (int i = r.tid; i < r.V; i += kThreads) {
      const float z = clean(r.z[i]);
      const uint32_t k = ordered_bits(z);
      if (k > kDead && kept(i, z, k)) m += mass_of(z, r.inv_ref, r.T);
    }
    total = block_sum(sh, m);
    const Cut c = find_cut<true>(sh, r, 0, p.p * (double)total, key);
    const uint32_t id = tie_id(sh, r, c.key, c.ties);
    last_id = c.key == key ? min(id, last_id) : id;
    key = c.key;
  }
  // kept mass of each thread's contiguous ids, then the draw
  const int per = (r.V + kThreads - 1) / kThreads;
  const int i0 = min(r.tid * per, r.V), i1 = min(i0 + per, r.V);
  uint64_t m = 0;
  uint32_t n = 0;
  auto weight = [&](int i, uint32_t& count) -> uint64_t {
    const float z = clean(r.z[i]);
    const uint32_t k = ordered_bits(z);
    if (k <= kDead || !kept(i, z, k) || (k != top && !over_min(z, r.inv_ref, r.T, p.min_p))) return 0;
    ++count;
    return mass_of(z, r.inv_ref, r.T);
  };
  for (int i = i0; i < i1; ++i) m += weight(i, n);
  total = block_sum(sh, m);
  const uint32_t n_kept = (uint32_t)block_sum(sh, n);
  sh.mass[r.tid] = m;
  __syncthreads();
  if (r.tid == 0) {
    const double want = p.u * (double)total;
    uint64_t c = 0;
    int w = 0, found = -1;
    uint64_t before = 0;
    for (; w < kThreads; ++w) {
      if (sh.mass[w] && (double)(c + sh.mass[w]) > want) {
        found = w, before = c;
        break;
      }
      if (sh.mass[w]) found = w, before = c;
      c += sh.mass[w];
    }
    sh.bin = (uint32_t)found;
    sh.above_mass = before;
  }
  __syncthreads();
  if (r.tid == (int)sh.bin) {
    const double want = p.u * (double)total;
    uint64_t c = sh.above_mass;
    int tok = -1;
    uint32_t d = 0;
    for (int i = i0; i < i1; ++i) {
      const uint64_t x = weight(i, d);
      if (!x) continue;
      tok = i;
      c += x;
      if ((double)c > want) break;
    }
    a.tok[row] = tok;
    if (a.kept) a.kept[row] = (int32_t)n_kept;
    if (a.logp)
      a.logp[row] = (float)(((double)clean(r.z[tok]) - r.inv_ref) / r.T - log((double)total * 0x1p-43));
  }
}

}  // namespace

hipError_t launch_sample(const SampleArgs& a, hipStream_t s) {
  hipLaunchKernelGGL(sample_kernel, dim3(a.rows), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace msd
