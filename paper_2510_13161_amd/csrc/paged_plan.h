// Paged attention: a sequence's key blocks and their split over workgroups.
#pragma once
#include "paged.h"

namespace msd {
namespace {

// 64-key blocks of a sequence: `sink` of the sinks, [w0, n) from the window on,
// `own` (0 or 1) of the rows' own keys.
struct Span {
  int sink, w0, n, own;
  __device__ int total() const { return sink + n - w0 + own; }
};

__device__ __forceinline__ int row_count(const PagedAttnArgs& a, int b) {
  return a.count ? min(max(a.count[b], 0), a.n_slots) : a.n_slots;
}
__device__ __forceinline__ bool seq_fits(const PagedAttnArgs& a, int b) {
  const int64_t L = a.kv.len[b];
  return L >= 0 && L + a.n_slots <= a.kv.capacity;
}
__device__ __forceinline__ Span seq_span(const PagedAttnArgs& a, int b) {
  const int cnt = row_count(a, b);
  if (!seq_fits(a, b) || cnt == 0) return Span{0, 0, 0, 0};
  const int L = a.kv.len[b];
  const int end = a.k_new ? L : L + cnt;
  Span s;
  s.own = a.k_new ? 1 : 0;
  s.n = (end + 63) >> 6;
  s.w0 = a.window > 0 ? min(max(L - a.window + 1, 0) >> 6, s.n) : 0;
  s.sink = min((int)(((int64_t)a.sinks + 63) >> 6), s.w0);
  return s;
}

// Chunks of G blocks, the same G for every sequence and as small as lets all
// chunks fit a.wgs workgroups, from the lengths, which only the device knows: one
// wave tries 64 candidates (multiples of 4, a block for each wave of a
// workgroup) from an equal share up to one chunk a sequence. chunk0[b] (b <=
// batch) = chunks of the sequences before b.
__device__ __forceinline__ int plan_chunks(const PagedAttnArgs& a, int* chunk0, bool flag) {
  const int lane = threadIdx.x & 63;
  int total = 0, most = 0;
  for (int b0 = 0; b0 < a.batch; b0 += 64) {
    const int b = b0 + lane;
    int n = 0;
    if (b < a.batch) {
      n = seq_span(a, b).total();
      chunk0[b] = n;
      if (flag && !seq_fits(a, b)) atomicOr(a.kv.status, 1u);
    }
    int t = n, m = n;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      t += __shfl_xor(t, o);
      m = max(m, __shfl_xor(m, o));
    }
    total += t;
    most = max(most, m);
  }
  wave_lds_sync();
  const int lo = max(4, ((total + a.wgs - 1) / a.wgs + 3) & ~3);
  const int step = (max(4, (most - lo + 62) / 63) + 3) & ~3;
  const int g = lo + lane * step;  // the last is >= most: one chunk a sequence
  int chunks = 0;
  for (int b = 0; b < a.batch; ++b) chunks += (chunk0[b] + g - 1) / g;
  const unsigned long long fit = __ballot(chunks <= a.wgs);
  const int G = lo + step * (fit ? __ffsll((long long)fit) - 1 : 63);
  int before = 0;
  for (int b0 = 0; b0 < a.batch; b0 += 64) {
    const int b = b0 + lane;
    const int n = b < a.batch ? (chunk0[b] + G - 1) / G : 0;
    int x = n;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int y = __shfl_up(x, o);
      if (lane >= o) x += y;
    }
    if (b < a.batch) chunk0[b] = before + x - n;
    before += __shfl(x, 63);
  }
  if (lane == 0) chunk0[a.batch] = before;
  return G;
}

// Query qg of a kv head's group: head gq of the group, slot.
__device__ __forceinline__ void query_of(const PagedAttnArgs& a, int qg, int& gq, int& slot) {
  gq = qg / a.n_slots;
  slot = qg - gq * a.n_slots;
}

}  // namespace
}  // namespace msd
