// Sampling under temperature, top-k, top-p and min-p from given uniforms.
//
// Tokens are ranked by (logit descending, id ascending), one 64-bit key; every
// filter keeps a prefix of that order, so the kept set is the keys at or above one
// threshold. Masses 2^t, t = (z - max) log2(e) / T, are fp64 values rounded to
// multiples of 2^-43: integer sums, the same in any order, so that
// histograms may be filled with atomics and a run repeats bit for bit (2^20
// tokens of mass one fill 2^63).
//
//  1 top    a workgroup a chunk of 8192 logits: its largest.
//  2 tally  the chunk again (held in registers, 16 a thread): its mass where the row
//           needs the mass of all tokens (unfiltered, or top-p without top-k); for
//           filtered rows a histogram over half octaves of 2^t down to
//           2^-64, of counts and, for top-p without top-k, masses; and the keys of
//           the chunk's highest half octaves, in their order, as many as fit 512.
//  3 draw   a workgroup a row: the histograms added up give the half octave that
//           top-k (else top-p, min-p) cuts. Where the chunks' lists reach
//           down to it, its keys and those above come into LDS; a cut is found by a
//           histogram over 1024 parts of its half octave, the few keys of one
//           part then ranked by counting. Else (flat laws, whose kept sets are a
//           large part of the vocabulary) digit by digit over the row. The draw:
//           masses of 512-id segments, the segment, the id. Unfiltered rows
//           take the chunk from the chunks' masses.
// 144 rows of 152K logits: 87.6 MB, read twice (the second time mostly from the
// memory-side cache).
#include "sample.h"

namespace msd {
namespace {

constexpr int kChunk = 8192, kTally = 512, kEach = kChunk / kTally;
constexpr int kBins = 128;        // half octaves; the last takes all below 2^-63.5
constexpr int kList = 512;        // keys of a chunk's list
constexpr int kDraw = 1024;       // threads of the draw
constexpr int kCands = 8192;      // keys that the draw holds
constexpr int kSeg = 512;         // ids of a segment
constexpr int kSegs = (1 << 20) / kSeg;
constexpr int kMaxChunks = (1 << 20) / kChunk;
constexpr int kDigit = 2048;      // digit values of the search over a row

struct Chunk {
  int32_t list_bin;  // the list holds all its tokens of bins <= list_bin, in order of bins
  int32_t unused;
  uint64_t mass;     // of all its tokens
  uint64_t tokens;   // above -inf
};

// Workspace of a row: [chunks] top keys, Chunk records, counts through each bin
// [kBins], masses of the bins [kBins], lists [kList].
struct Work {
  uint32_t* top;
  Chunk* head;
  uint32_t* cnt;
  uint64_t* mass;
  uint64_t* list;
};
__host__ __device__ inline int chunks_of(int vocab) { return (vocab + kChunk - 1) / kChunk; }
__host__ __device__ inline size_t row_bytes(int C) {
  const size_t b = (size_t)C * (kList * 8 + kBins * 12 + sizeof(Chunk) + 4);
  return (b + 15) / 16 * 16;
}
__device__ __forceinline__ Work work_of(const SampleArgs& a, int row, int C) {
  char* p = static_cast<char*>(a.ws) + row_bytes(C) * row;
  Work w;
  w.list = reinterpret_cast<uint64_t*>(p);
  w.mass = w.list + (size_t)C * kList;
  w.head = reinterpret_cast<Chunk*>(w.mass + (size_t)C * kBins);
  w.cnt = reinterpret_cast<uint32_t*>(w.head + C);
  w.top = w.cnt + (size_t)C * kBins;
  return w;
}

// Half octave of a logit, in fp32: any function does that never rises with z and is
// the same everywhere. x = -2 t (from halves, which do not overflow); its part
// inside the bin is the fraction.
__device__ __forceinline__ float depth_of(float z, float ref, float c4) { return (0.5f * ref - 0.5f * z) * c4; }
__device__ __forceinline__ int bin_of(float x) { return (int)fminf(x, (float)(kBins - 1)); }
__device__ __forceinline__ float c4_of(const Request& q) { return (float)fmin(4.0 * q.c, 3e38); }
// whether the row needs the mass of tokens that no list may hold
__device__ __forceinline__ bool mass_by_bin(const Request& q, int V) { return q.p < 1.0 && q.k >= (uint32_t)V; }

__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, o));
  return v;
}
__device__ __forceinline__ uint64_t wave_sum_u64(uint64_t v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  return v;
}
__device__ __forceinline__ uint64_t wave_scan_u64(uint64_t v) {  // inclusive
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint64_t y = __shfl_up(v, o);
    if (lane >= o) v += y;
  }
  return v;
}

__global__ __launch_bounds__(kTally) void top_kernel(SampleArgs a) {
  __shared__ uint32_t red[kTally / 64];
  const int c = blockIdx.x, row = blockIdx.y, tid = threadIdx.x;
  const float* z = a.logits + (int64_t)row * a.row_stride;
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < kEach; ++j) {
    const int i = c * kChunk + j * kTally + tid;
    if (i < a.vocab) top = max(top, ordered_bits(clean(z[i])));
  }
  top = wave_max_u32(top);
  if ((tid & 63) == 0) red[tid >> 6] = top;
  __syncthreads();
  if (tid == 0) {
    for (int w = 1; w < kTally / 64; ++w) top = max(top, red[w]);
    work_of(a, row, gridDim.x).top[c] = top;
  }
}

__global__ __launch_bounds__(kTally) void tally_kernel(SampleArgs a) {
  __shared__ uint32_t cnt[kBins];
  __shared__ unsigned long long mass[kBins];
  __shared__ uint32_t cursor[kBins];
  __shared__ uint64_t red[kTally / 64];
  __shared__ uint32_t red_n[kTally / 64];
  __shared__ uint32_t last_bin;
  __shared__ int list_bin;
  const int C = gridDim.x, c = blockIdx.x, row = blockIdx.y, tid = threadIdx.x;
  const Work w = work_of(a, row, C);
  const float* z = a.logits + (int64_t)row * a.row_stride;
  float v[kEach];
#pragma unroll
  for (int j = 0; j < kEach; ++j) {
    const int i = c * kChunk + j * kTally + tid;
    v[j] = i < a.vocab ? clean(z[i]) : -INFINITY;
  }
  uint32_t top = 0;
  for (int i = tid & 63; i < C; i += 64) top = max(top, w.top[i]);
  top = wave_max_u32(top);
  if (top <= kDead) return;  // no token
  const float ref = from_ordered_bits(top);
  const Request q = request_of(a, row);
  const float c4 = c4_of(q);
  const bool filtered = q.filtered(), by_bin = mass_by_bin(q, a.vocab);
  if (tid < kBins) cnt[tid] = 0, mass[tid] = 0;
  if (tid == 0) last_bin = 0;
  __syncthreads();
  uint64_t sum = 0;
  uint32_t tokens = 0;
  uint32_t low = 0;  // tokens of the last bin, which most tokens of cold laws share
#pragma unroll
  for (int j = 0; j < kEach; ++j) {
    if (v[j] == -INFINITY) continue;
    ++tokens;
    uint64_t m = 0;
    if (!filtered || by_bin) sum += m = mass_of(exponent_of(v[j], ref, q.c));
    if (!filtered) continue;
    const int b = bin_of(depth_of(v[j], ref, c4));
    if (b == kBins - 1) ++low;
    else atomicAdd(&cnt[b], 1u);
    if (m) atomicAdd(&mass[b], (unsigned long long)m);
  }
  sum = wave_sum_u64(sum);
  tokens = (uint32_t)wave_sum_u64(tokens);
  if (low) atomicAdd(&last_bin, low);
  if ((tid & 63) == 0) red[tid >> 6] = sum, red_n[tid >> 6] = tokens;
  __syncthreads();
  if (tid < 64) {
    // counts through each bin; the deepest bin down to which they fit the list
    const uint32_t c0 = cnt[2 * tid], c1 = tid == 63 ? last_bin : cnt[2 * tid + 1];
    const uint32_t x = (uint32_t)wave_scan_u64(c0 + c1);
    int f = (x - c1 <= kList) + (x <= kList);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) f += __shfl_xor(f, o);
    cursor[2 * tid] = x - c1 - c0;
    cursor[2 * tid + 1] = x - c1;
    cnt[2 * tid] = x - c1;
    cnt[2 * tid + 1] = x;
    if (tid == 0) {
      list_bin = f - 1;
      for (int i = 1; i < kTally / 64; ++i) red[0] += red[i], red_n[0] += red_n[i];
    }
  }
  __syncthreads();
  if (filtered) {
    const int lb = list_bin;
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
      const int b = v[j] == -INFINITY ? kBins : bin_of(depth_of(v[j], ref, c4));
      if (b <= lb) w.list[(size_t)c * kList + atomicAdd(&cursor[b], 1u)] = rank_key(v[j], c * kChunk + j * kTally + tid);
    }
    if (tid < kBins) {
      w.cnt[(size_t)c * kBins + tid] = cnt[tid];
      if (by_bin) w.mass[(size_t)c * kBins + tid] = mass[tid];
    }
  }
  if (tid == 0) w.head[c] = Chunk{list_bin, 0, red[0], red_n[0]};
}

struct Shared {
  uint64_t cand[kCands];       // keys; in the search over a row: digit masses
  uint64_t seg[kSegs];         // segment masses; before, the search among the keys
  uint64_t red[kDraw / 64 + 1];
  uint64_t mass[kBins];        // tokens of the bins above, then of the bin
  uint32_t cnt[kBins];
  uint64_t above_mass, above, key;
  uint32_t n, m, pick;
  int min_list;
  uint32_t from[kMaxChunks + 1];  // candidates of the chunks before
};
static_assert(kCands * 8 >= kDigit * 12, "digit histograms fit the key list");

// inclusive block scan over kDraw threads; total in sh.red[kDraw / 64]
__device__ __forceinline__ uint64_t block_scan(Shared& sh, uint64_t v) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint64_t x = wave_scan_u64(v);
  __syncthreads();
  if (lane == 63) sh.red[wave] = x;
  __syncthreads();
  if (wave == 0) {
    const uint64_t y = lane < kDraw / 64 ? sh.red[lane] : 0;
    const uint64_t s = wave_scan_u64(y);
    if (lane < kDraw / 64) sh.red[lane] = s - y;
    if (lane == kDraw / 64 - 1) sh.red[kDraw / 64] = s;
  }
  __syncthreads();
  return x + sh.red[wave];
}

struct Row {
  const float* z;
  int V;
  float ref;   // the largest logit
  uint32_t top;
  float c4;
  Request q;
  uint64_t threshold;  // smallest kept key
  __device__ uint64_t mass(uint64_t key) const { return mass_of(exponent_of(key_val(key), ref, q.c)); }
  __device__ float depth(uint64_t key) const { return depth_of(key_val(key), ref, c4); }
  __device__ uint64_t weight(int i, bool& kept) const {
    const float x = clean(z[i]);
    kept = false;
    if (x == -INFINITY || rank_key(x, i) < threshold) return 0;
    const double t = exponent_of(x, ref, q.c);
    if (q.min_p > 0.0 && x != ref && exp2_64(t, 0) < q.min_p) return 0;
    kept = true;
    return mass_of(t);
  }
};

// The key at which the kept prefix ends, searched digit by digit (11, 11 and 10
// bits of the ordered logit) over the row's tokens with key >= floor: the n-th
// (by count), or the last whose preceding mass is below `want`. Equal logits are
// cut in id order.
template <bool BY_MASS>
__device__ uint64_t search_row(Shared& sh, const Row& r, uint64_t n, double want, uint64_t floor) {
  uint64_t* mass = sh.cand;
  uint32_t* cnt = reinterpret_cast<uint32_t*>(mass + kDigit);
  const int tid = threadIdx.x;
  uint32_t prefix = 0;
  uint64_t above = 0, above_mass = 0;
  uint32_t equal = 0;
  for (int level = 0; level < 3; ++level) {
    const int shift = level == 0 ? 21 : (level == 1 ? 10 : 0);
    const int bits = level == 2 ? 10 : 11;
    __syncthreads();
    for (int i = tid; i < kDigit; i += kDraw) cnt[i] = 0, mass[i] = 0;
    __syncthreads();
    for (int i = tid; i < r.V; i += kDraw) {
      const float z = clean(r.z[i]);
      const uint32_t k = ordered_bits(z);
      if (k <= kDead || (level && (k >> (shift + bits)) != prefix) || rank_key(z, i) < floor) continue;
      const uint32_t d = (k >> shift) & ((1u << bits) - 1);
      atomicAdd(&cnt[d], 1u);
      if (BY_MASS) {
        const uint64_t m = mass_of(exponent_of(z, r.ref, r.q.c));
        if (m) atomicAdd((unsigned long long*)&mass[d], (unsigned long long)m);
      }
    }
    __syncthreads();
    // scanned from the largest digit: thread t holds digits D - 1 - 2 t and D - 2 - 2 t
    const int D = 1 << bits;
    const int d0 = D - 1 - 2 * tid, d1 = d0 - 1;
    const uint64_t c0 = d0 >= 0 ? cnt[d0] : 0, c1 = d1 >= 0 ? cnt[d1] : 0;
    const uint64_t m0 = d0 >= 0 ? mass[d0] : 0, m1 = d1 >= 0 ? mass[d1] : 0;
    const uint64_t cs = above + block_scan(sh, c0 + c1) - c0 - c1;
    const uint64_t ms = BY_MASS ? above_mass + block_scan(sh, m0 + m1) - m0 - m1 : 0;
    // the last non-empty digit that starts inside
    auto inside = [&](uint64_t cb, uint64_t mb) { return BY_MASS ? (cb == 0 || (double)mb < want) : cb < n; };
    int last = -1;
    if (c0 && inside(cs, ms)) last = 2 * tid;
    if (c1 && inside(cs + c0, ms + m0)) last = 2 * tid + 1;
    if (tid == 0) sh.m = 0;
    __syncthreads();
    if (last >= 0) atomicMax(&sh.m, (uint32_t)last);
    __syncthreads();
    if (last >= 0 && sh.m == (uint32_t)last) {
      sh.pick = D - 1 - last;
      sh.key = cs + (last & 1 ? c0 : 0);
      sh.above_mass = ms + (last & 1 ? m0 : 0);
      sh.n = (uint32_t)(last & 1 ? c1 : c0);
    }
    __syncthreads();
    prefix = (prefix << bits) | sh.pick;
    above = sh.key;
    above_mass = sh.above_mass;
    equal = sh.n;
  }
  // of the `equal` tokens with this logit, the first t ids
  uint32_t t = equal;
  if (BY_MASS) {
    const uint64_t one = mass_of(exponent_of(from_ordered_bits(prefix), r.ref, r.q.c));
    uint32_t lo = 0;  // smallest t >= 1 with above_mass + t * one >= want, at most equal
    while (lo + 1 < t) {
      const uint32_t mid = (lo + t) / 2;
      if ((double)(above_mass + mid * one) < want) lo = mid;
      else t = mid;
    }
  } else if (n - above < equal) {
    t = (uint32_t)(n - above);
  }
  if (t == equal) return (uint64_t)prefix << 32;  // all of them
  // the t-th id: equal logits counted by blocks of kDraw ids
  uint32_t seen = 0;
  for (int i0 = 0; i0 < r.V; i0 += kDraw) {
    const int i = i0 + tid;
    const bool is = i < r.V && ordered_bits(clean(r.z[i])) == prefix;
    const uint64_t x = block_scan(sh, is ? 1 : 0);
    if (is && seen + x == t) sh.key = rank_key(from_ordered_bits(prefix), i);
    seen += (uint32_t)sh.red[kDraw / 64];
    if (seen >= t) break;
  }
  __syncthreads();
  return sh.key;
}

// The same among the candidate keys >= floor of bin `bin`; `above` tokens and
// `above_mass` lie in the bins before. First the part of the bin (1024, a thread
// each) in which the prefix ends, then the keys of that part in order. False:
// more keys in one part than threads (equal logits).
template <bool BY_MASS>
__device__ bool search_bin(Shared& sh, const Row& r, uint32_t N, int bin, uint64_t n, double want, uint64_t above,
                           uint64_t above_mass, uint64_t floor, uint64_t* key_out, uint64_t* kept_mass) {
  const int tid = threadIdx.x;
  uint64_t* mass = sh.seg;                                       // [kDraw]
  uint32_t* cnt = reinterpret_cast<uint32_t*>(sh.seg + kDraw);   // [kDraw]
  auto part_of = [&](uint64_t k) {  // -1: not of the bin
    const float x = r.depth(k);
    return bin_of(x) != bin ? -1 : (int)fminf((x - (float)bin) * kDraw, (float)(kDraw - 1));
  };
  auto inside = [&](uint64_t cb, uint64_t mb) { return BY_MASS ? (cb == 0 || (double)mb < want) : cb < n; };
  __syncthreads();
  mass[tid] = 0;
  cnt[tid] = 0;
  if (tid == 0) sh.m = 0, sh.n = 0;
  __syncthreads();
  for (uint32_t i = tid; i < N; i += kDraw) {
    const uint64_t k = sh.cand[i];
    if (k < floor) continue;
    const int p = part_of(k);
    if (p < 0) continue;
    atomicAdd(&cnt[p], 1u);
    atomicAdd((unsigned long long*)&mass[p], (unsigned long long)r.mass(k));
  }
  __syncthreads();
  {
    const uint64_t c0 = cnt[tid], m0 = mass[tid];
    const uint64_t cb = above + block_scan(sh, c0) - c0;
    const uint64_t mb = above_mass + block_scan(sh, m0) - m0;
    const bool in = c0 && inside(cb, mb);  // a prefix of the parts
    if (in) atomicMax(&sh.m, (uint32_t)tid);
    __syncthreads();
    if (in && sh.m == (uint32_t)tid) sh.above = cb, sh.above_mass = mb, sh.pick = (uint32_t)c0;
    __syncthreads();
  }
  const int part = (int)sh.m;
  const uint32_t m = sh.pick;
  above = sh.above;
  above_mass = sh.above_mass;
  if (m > kDraw) return false;
  uint64_t* mine = sh.seg;
  for (uint32_t i = tid; i < N; i += kDraw) {
    const uint64_t k = sh.cand[i];
    if (k >= floor && part_of(k) == part) mine[atomicAdd(&sh.n, 1u)] = k;
  }
  __syncthreads();
  const uint64_t key = tid < (int)m ? mine[tid] : 0;
  uint32_t rank = 0;
  for (uint32_t i = 0; i < m; ++i) rank += mine[i] > key;
  __syncthreads();
  uint64_t* by_rank = sh.seg;               // masses
  uint64_t* key_by_rank = sh.seg + kDraw;
  if (tid < (int)m) {
    by_rank[rank] = r.mass(key);
    key_by_rank[rank] = key;
  }
  __syncthreads();
  const uint64_t w = tid < (int)m ? by_rank[tid] : 0;
  const uint64_t x = above_mass + block_scan(sh, w);  // mass through rank tid
  // the ranks inside are a prefix: the last of them
  if (tid < (int)m && inside(above + tid, x - w) && (tid + 1 == (int)m || !inside(above + tid + 1, x))) {
    sh.key = key_by_rank[tid];
    sh.above_mass = x;
  }
  __syncthreads();
  *key_out = sh.key;
  *kept_mass = sh.above_mass;
  __syncthreads();
  return true;
}
static_assert(kSegs >= 2 * kDraw, "ranks and their keys fit the segment masses");

__global__ __launch_bounds__(kDraw) void draw_kernel(SampleArgs a, int C) {
  __shared__ Shared sh;
  const int row = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const Work w = work_of(a, row, C);
  Row r;
  r.z = a.logits + (int64_t)row * a.row_stride;
  r.V = a.vocab;
  r.q = request_of(a, row);
  uint32_t top = 0;
  for (int i = lane; i < C; i += 64) top = max(top, w.top[i]);
  r.top = wave_max_u32(top);
  if (r.top <= kDead) {
    if (tid == 0) {
      a.tok[row] = -1;
      if (a.logp) a.logp[row] = -INFINITY;
      if (a.kept) a.kept[row] = 0;
    }
    return;
  }
  r.ref = from_ordered_bits(r.top);
  r.c4 = c4_of(r.q);
  r.threshold = 0;
  const bool filtered = r.q.filtered();
  uint32_t n_kept = 0;
  const int n_seg = (r.V + kSeg - 1) / kSeg;
  int first_seg = 0, last_seg = n_seg;  // segments whose masses are in sh.seg
  uint64_t total = 0, before = 0;       // all kept mass; that of the segments before first_seg
  bool from_list = false;
  uint32_t N = 0;

  if (filtered) {
    const bool by_bin = mass_by_bin(r.q, r.V);
    if (tid < kBins) sh.cnt[tid] = 0, sh.mass[tid] = 0;
    if (tid == 0) sh.min_list = kBins;
    __syncthreads();
    {
      uint32_t n = 0;
      uint64_t m = 0;
      const int b = tid % kBins;
      for (int c = tid / kBins; c < C; c += kDraw / kBins) {
        n += w.cnt[(size_t)c * kBins + b];
        if (by_bin) m += w.mass[(size_t)c * kBins + b];
      }
      if (n) atomicAdd(&sh.cnt[b], n);
      if (m) atomicAdd((unsigned long long*)&sh.mass[b], (unsigned long long)m);
      if (tid < C) atomicMin(&sh.min_list, w.head[tid].list_bin);
    }
    __syncthreads();
    auto mass_prefix = [&]() {  // bins' masses to those through each bin
      if (wave == 0) {
        const uint64_t m0 = sh.mass[2 * lane], m1 = sh.mass[2 * lane + 1];
        const uint64_t x = wave_scan_u64(m0 + m1);
        sh.mass[2 * lane] = x - m1;
        sh.mass[2 * lane + 1] = x;
      }
      __syncthreads();
    };
    if (by_bin) mass_prefix();
    const uint32_t valid = sh.cnt[kBins - 1];
    const bool by_k = r.q.k < valid;
    bool by_p = r.q.p < 1.0;
    auto first_bin = [&](auto before) {  // first bin, of the last at most, that is not `before`
      int lo = 0, hi = kBins - 1;
      while (lo < hi) {
        const int mid = (lo + hi) / 2;
        if (before(mid)) lo = mid + 1;
        else hi = mid;
      }
      return lo;
    };
    auto bin_by_mass = [&](double want) {
      return first_bin([&](int b) { return sh.cnt[b] == 0 || (double)sh.mass[b] < want; });
    };
    // the deepest bin that can hold a kept token; min_p's is one more than its
    // border's, whatever way that rounds
    int deepest = kBins - 1;
    if (r.q.min_p > 0.0) deepest = r.q.min_p < 1.0 ? min(kBins - 1, bin_of((float)(-2.0 * log2(r.q.min_p))) + 1) : 0;
    int k_bin = 0;
    if (by_k) {
      k_bin = first_bin([&](int b) { return sh.cnt[b] < r.q.k; });
      deepest = k_bin;
    } else if (by_p && by_bin) {
      const int b = bin_by_mass(r.q.p * (double)sh.mass[kBins - 1]);
      if (b <= deepest) deepest = b;
      else by_p = false;  // min_p ends before
    } else if (by_p) {
      deepest = kBins - 1;  // top-k that keeps all of a row with few tokens: their masses come from the keys
    }
    N = sh.cnt[deepest];
    from_list = deepest <= sh.min_list && N <= kCands;
    if (from_list) {
      // candidates: the first keys of every chunk's list
      uint32_t n = 0;
      if (tid < C) n = w.cnt[(size_t)tid * kBins + deepest];
      const uint64_t x = block_scan(sh, n);
      if (tid < C) sh.from[tid] = (uint32_t)(x - n);
      if (tid == C) sh.from[C] = (uint32_t)x;
      __syncthreads();
      for (int c = wave; c < C; c += kDraw / 64) {
        const uint32_t at = sh.from[c], m = sh.from[c + 1] - at;
        for (uint32_t i = lane; i < m; i += 64) sh.cand[at + i] = w.list[(size_t)c * kList + i];
      }
      __syncthreads();
    }
    uint64_t all = by_bin ? sh.mass[kBins - 1] : 0;  // mass that top-p is a share of
    if (by_p && !by_bin && from_list) {
      // the bins' masses from the keys
      for (uint32_t i = tid; i < N; i += kDraw) {
        const uint64_t k = sh.cand[i];
        atomicAdd((unsigned long long*)&sh.mass[bin_of(r.depth(k))], (unsigned long long)r.mass(k));
      }
      __syncthreads();
      mass_prefix();
      all = sh.mass[kBins - 1];
    }
    if (by_k) {
      const uint64_t above = k_bin ? sh.cnt[k_bin - 1] : 0, above_mass = k_bin ? sh.mass[k_bin - 1] : 0;
      if (from_list)
        from_list = search_bin<false>(sh, r, N, k_bin, r.q.k, 0.0, above, above_mass, 0, &r.threshold, &all);
      if (!from_list) r.threshold = search_row<false>(sh, r, r.q.k, 0.0, 0);
    }
    if (by_p && !by_bin && !from_list) {
      uint64_t m = 0;
      for (int i = tid; i < r.V; i += kDraw) {
        const float z = clean(r.z[i]);
        if (z != -INFINITY && rank_key(z, i) >= r.threshold) m += mass_of(exponent_of(z, r.ref, r.q.c));
      }
      block_scan(sh, m);
      all = sh.red[kDraw / 64];
      __syncthreads();
    }
    if (by_p) {
      const double want = r.q.p * (double)all;
      if (from_list) {
        const int b = bin_by_mass(want);
        const uint64_t above = b ? sh.cnt[b - 1] : 0, above_mass = b ? sh.mass[b - 1] : 0;
        uint64_t unused;
        from_list = search_bin<true>(sh, r, N, b, 0, want, above, above_mass, r.threshold, &r.threshold, &unused);
      }
      if (!from_list) r.threshold = search_row<true>(sh, r, 0, want, r.threshold);
    }
    __syncthreads();
    for (int i = tid; i < n_seg; i += kDraw) sh.seg[i] = 0;
    __syncthreads();
    if (from_list) {
      uint64_t count = 0;
      for (uint32_t i = tid; i < N; i += kDraw) {
        const uint64_t k = sh.cand[i];
        if (k < r.threshold) continue;
        const float z = key_val(k);
        const double t = exponent_of(z, r.ref, r.q.c);
        if (r.q.min_p > 0.0 && z != r.ref && exp2_64(t, 0) < r.q.min_p) continue;
        ++count;
        atomicAdd((unsigned long long*)&sh.seg[key_id(k) / kSeg], (unsigned long long)mass_of(t));
      }
      block_scan(sh, count);
      n_kept = (uint32_t)sh.red[kDraw / 64];
    }
  } else {
    // the chunk from the chunks' masses (at most 128 of them)
    const uint64_t m = tid < C ? w.head[tid].mass : 0;
    const uint64_t x = block_scan(sh, m);
    total = sh.red[kDraw / 64];
    const double want = r.q.u * (double)total;
    if (m && (double)x > want && !((double)(x - m) > want)) {
      sh.pick = tid;
      sh.above_mass = x - m;
    }
    __syncthreads();
    first_seg = (int)sh.pick * (kChunk / kSeg);
    last_seg = min(n_seg, first_seg + kChunk / kSeg);
    before = sh.above_mass;
    block_scan(sh, tid < C ? w.head[tid].tokens : 0);
    n_kept = (uint32_t)sh.red[kDraw / 64];
    for (int i = tid; i < n_seg; i += kDraw) sh.seg[i] = 0;
    __syncthreads();
  }
  if (!from_list) {
    // segment masses from the row, a wave a segment
    uint64_t count = 0;
    for (int s = first_seg + wave; s < last_seg; s += kDraw / 64) {
      uint64_t m = 0;
#pragma unroll
      for (int j = 0; j < kSeg / 64; ++j) {
        const int i = s * kSeg + j * 64 + lane;
        bool kept = false;
        if (i < r.V) m += r.weight(i, kept);
        count += kept;
      }
      m = wave_sum_u64(m);
      if (lane == 0) sh.seg[s] = m;
    }
    if (filtered) {
      block_scan(sh, count);
      n_kept = (uint32_t)sh.red[kDraw / 64];
    }
  }
  __syncthreads();
  // the segment: thread t holds segments 2 t and 2 t + 1
  {
    const uint64_t s0 = 2 * tid < n_seg ? sh.seg[2 * tid] : 0;
    const uint64_t s1 = 2 * tid + 1 < n_seg ? sh.seg[2 * tid + 1] : 0;
    const uint64_t x = before + block_scan(sh, s0 + s1);
    if (filtered) total = sh.red[kDraw / 64];
    const double want = r.q.u * (double)total;
    const uint64_t b1 = x - s1, b0 = b1 - s0;
    if (s0 && (double)b1 > want && !((double)b0 > want)) sh.pick = 2 * tid, sh.above_mass = b0;
    if (s1 && (double)x > want && !((double)b1 > want)) sh.pick = 2 * tid + 1, sh.above_mass = b1;
  }
  __syncthreads();
  const int seg = (int)sh.pick;
  const uint64_t c0 = sh.above_mass;
  bool kept = false;
  const int id = seg * kSeg + tid;
  const uint64_t m = tid < kSeg && id < r.V ? r.weight(id, kept) : 0;
  const uint64_t x = c0 + block_scan(sh, m);
  const double want = r.q.u * (double)total;
  if (m && (double)x > want && !((double)(x - m) > want)) {
    a.tok[row] = id;
    if (a.kept) a.kept[row] = (int32_t)n_kept;
    if (a.logp)
      a.logp[row] = (float)(exponent_of(clean(r.z[id]), r.ref, r.q.c) * 0.6931471805599453 - log((double)total * 0x1p-43));
  }
}

}  // namespace

size_t sample_row_bytes(int32_t vocab) { return row_bytes(chunks_of(vocab)); }

hipError_t launch_sample(const SampleArgs& a, hipStream_t s) {
  const int C = chunks_of(a.vocab);
  hipLaunchKernelGGL(top_kernel, dim3(C, a.rows), dim3(kTally), 0, s, a);
  hipLaunchKernelGGL(tally_kernel, dim3(C, a.rows), dim3(kTally), 0, s, a);
  hipLaunchKernelGGL(draw_kernel, dim3(a.rows), dim3(kDraw), 0, s, a, C);
  return hipGetLastError();
}

}  // namespace msd
