// Paged attention: a sequence's key blocks and their split over workgroups.
#pragma once
#include "paged.h"

namespace msd {
namespace {

constexpr int kBlock = 32;  // positions of a block: a wave's share of a round
constexpr int kWaves = 8;   // waves of a workgroup

// Blocks of a sequence: `sink` of the sinks, [w0, n) from the window on, `own` of
// the rows' own keys.
struct Span {
  int sink, w0, n, own;
  __device__ int cached() const { return sink + n - w0; }
  __device__ int total() const { return cached() + own; }
  __device__ int first_pos(int i) const { return kBlock * (i < sink ? i : i - sink + w0); }
};

__device__ __forceinline__ int row_count(const PagedAttnArgs& a, int b) {
  return a.count ? min(max(a.count[b], 0), a.n_slots) : a.n_slots;
}
__device__ __forceinline__ bool seq_fits(const PagedAttnArgs& a, int len) {
  return len >= 0 && (int64_t)len + a.n_slots <= a.kv.capacity;
}
__device__ __forceinline__ Span seq_span(const PagedAttnArgs& a, int len, int cnt) {
  if (!seq_fits(a, len) || cnt == 0) return Span{0, 0, 0, 0};
  const int end = a.k_new ? len : len + cnt;
  Span s;
  s.own = a.k_new ? (cnt + kBlock - 1) / kBlock : 0;
  s.n = (end + kBlock - 1) / kBlock;
  s.w0 = a.window > 0 ? min(max(len - a.window + 1, 0) / kBlock, s.n) : 0;
  s.sink = (int)min(((int64_t)a.sinks + kBlock - 1) / kBlock, (int64_t)s.w0);
  return s;
}

// Size of the chunks of a sequence of n blocks: equal, up to whole rounds of a workgroup.
__device__ __forceinline__ int chunk_size(int n, int chunks) {
  return ((n + chunks - 1) / chunks + kWaves - 1) & ~(kWaves - 1);
}

// Chunk counts of the sequences from their lengths, which only the device knows:
// at most G blocks a chunk, the same G for all and as small as lets all chunks
// fit a.wgs workgroups. One wave tries 64 candidates (whole rounds of a workgroup)
// from an equal share up to one chunk a sequence. chunk0[b] (b <= batch) = chunks
// of the sequences before b. (Equal runs of blocks across sequences, which end
// together, lost more: a second sequence costs a workgroup its start once more,
// 8 us. 16 chains at 512 to 8192: 64 us against 56, under a window 30 against 22.)
__device__ __forceinline__ void plan_chunks(const PagedAttnArgs& a, int* chunk0, bool flag) {
  const int lane = threadIdx.x & 63;
  int total = 0, most = 0;
  for (int b0 = 0; b0 < a.batch; b0 += 64) {
    const int b = b0 + lane;
    int n = 0;
    if (b < a.batch) {
      const int len = a.kv.len[b];
      n = seq_span(a, len, row_count(a, b)).total();
      chunk0[b] = n;
      if (flag && !seq_fits(a, len)) atomicOr(a.kv.status, 1u);
    }
    total += __builtin_amdgcn_readlane(wave_scan_add(n), 63);
    most = max(most, wave_max_nonneg(n));
  }
  wave_lds_sync();
  constexpr int R = kWaves - 1;
  const int lo = max(kWaves, ((total + a.wgs - 1) / a.wgs + R) & ~R);
  const int step = (max(kWaves, (most - lo + 62) / 63) + R) & ~R;
  const int g = lo + lane * step;  // the last is >= most: one chunk a sequence
  int chunks = 0;
  if (most < 1 << 21) {
    // ceil(n / g) = floor((n - 1/2) / g) + 1, which lies at least 1 / (2 g) from any
    // integer: the fp32 quotient's error, under n / g * 2^-22, is less than that
    const float inv = 1.0f / (float)g;
#pragma unroll 4
    for (int b = 0; b < a.batch; ++b) {
      const int n = chunk0[b];
      chunks += n > 0 ? (int)(((float)n - 0.5f) * inv) + 1 : 0;
    }
  } else {
    for (int b = 0; b < a.batch; ++b) chunks += (chunk0[b] + g - 1) / g;
  }
  const unsigned long long fit = __ballot(chunks <= a.wgs);
  const int G = lo + step * (fit ? __ffsll((long long)fit) - 1 : 63);
  int before = 0;
  for (int b0 = 0; b0 < a.batch; b0 += 64) {
    const int b = b0 + lane;
    const int n = b < a.batch ? (chunk0[b] + G - 1) / G : 0;
    const int x = wave_scan_add(n);
    if (b < a.batch) chunk0[b] = before + x - n;
    before += __builtin_amdgcn_readlane(x, 63);
  }
  if (lane == 0) chunk0[a.batch] = before;
}

// Query qg of a kv head's group: head gq of the group, slot.
__device__ __forceinline__ void query_of(const PagedAttnArgs& a, int qg, int& gq, int& slot) {
  gq = qg / a.n_slots;
  slot = qg - gq * a.n_slots;
}

// Where 4 (or 8) consecutive output dims of a query from dim d on go: rounded to
// bf16, or as hi + lo words of the output projection's image.
template <int N>
__device__ __forceinline__ void write_output(const PagedAttnArgs& a, int b, int h, int slot, int d, const float (&o)[N]) {
  uint32_t hi[N / 2], lo[N / 2];
#pragma unroll
  for (int i = 0; i < N / 2; ++i) {
    hi[i] = pack_bf16x2(o[2 * i], o[2 * i + 1]);
    lo[i] = pack_bf16x2(o[2 * i] - bf_lo(hi[i]), o[2 * i + 1] - bf_hi(hi[i]));
  }
  uint16_t* dst;
  if (a.out_img) {
    const int m = b * a.n_slots + slot, col = h * a.kv.head_dim + d;
    dst = a.out_img + img_offset(col >> 5, m >> 4, a.MT, 16 * ((col >> 3) & 3) + (m & 15)) + (col & 7);
  } else {
    dst = a.out + b * a.out_seq + slot * a.out_row + h * a.out_head + d;
  }
#pragma unroll
  for (int i = 0; i < N / 4; ++i) reinterpret_cast<u32x2*>(dst)[i] = u32x2{hi[2 * i], hi[2 * i + 1]};
  if (a.out_img) {
#pragma unroll
    for (int i = 0; i < N / 4; ++i) reinterpret_cast<u32x2*>(dst + 512)[i] = u32x2{lo[2 * i], lo[2 * i + 1]};
  }
}

}  // namespace
}  // namespace msd
