// Sampling under temperature, top-k, top-p and min-p from given uniforms.
//
// Tokens are ranked by (logit descending, id ascending), one 64-bit key; every
// filter keeps a prefix of that order, so the kept set is the keys at or above one
// threshold. Masses 2^t, t = (z - max) log2(e) / T, are fp64 values rounded to
// multiples of 2^-43: integer sums, the same in any order, so that
// histograms may be filled with atomics and a run repeats bit for bit (2^20
// tokens of mass one fill 2^63).
//
//  1 tally  a workgroup a chunk of 8192 logits, held in registers: the largest; where
//           the row needs the mass of all tokens (unfiltered, or top-p without
//           top-k) the chunk's, against its own largest; for filtered rows the
//           chunk's highest tokens. A histogram over half octaves below its largest, of
//           the threads' largest logits, bounds what fits the chunk's share of 4096 keys;
//           the tokens above that bound are put together (most end here), a histogram of
//           those says how many half octaves fit, and these are listed.
//  2 draw   a workgroup a row, the lists in its registers. A cut is found by a histogram of
//           counts and masses over half octaves below the row's largest, then over
//           1024 parts of one half octave, then by ranking the few keys of one
//           part. It stands if every chunk has listed all it has above it; else
//           (flat laws, whose kept sets are a large part of the vocabulary) it is
//           searched digit by digit over the row. The draw: masses of 512-id
//           segments, the segment, the id. Unfiltered rows take the chunk from the
//           chunks' masses.
// The logits are read once: 144 rows of 152K are 87 MB, 18 us for a kernel that does no
// more than read them (4.9 TB/s). The tally takes 28 us, the fp64 masses, where a row needs
// them, 6 to 16 more: the chunks of a dispatch round are loaded together and worked on
// together, so their times add. (A chunk's loads issued while the one before is worked
// on: 40 us, at half the waves.) The draw is a chain of some 20 barriers: 9 us unfiltered,
// 11 for one filter, 15 for all, 24 for 144 rows of top-1000 with top-p.
#include <algorithm>

#include "paged.h"
#include "sample.h"

namespace msd {
namespace {

constexpr int kTally = 512;       // threads of a chunk
// Logits a thread of a chunk holds: 16 (chunks of 8192), or 8 where all chunks of
// that size are fewer than the compute units (one row of 152K: 19 of 8192 or 38 of 4096).
constexpr int kFew = 8, kMany = 16;
constexpr int kBins = 128;        // half octaves; the last takes all below 2^-63.5
constexpr int kDraw = 1024;       // threads of the draw
constexpr int kCands = 4096;      // keys that the draw holds in registers: all chunks' lists
constexpr int kSeg = 512;         // ids of a segment
constexpr int kSegs = (1 << 20) / kSeg;
constexpr int kMaxChunks = 256;
constexpr int kDigit = 2048;      // digit values of the search over a row

struct Chunk {
  uint32_t top;      // ordered bits of its largest logit, kDead: no token
  int32_t list_bin;  // its list holds all its tokens of half octaves <= list_bin below its largest
  uint32_t n_list;
  uint32_t tokens;   // above -inf
  uint64_t mass;     // of all its tokens, 2^-43 of its largest's
};

// Workspace of a row: lists [chunks][kCands / chunks], Chunk records.
struct Work {
  uint64_t* list;
  Chunk* head;
};
inline int chunks_of(int each, int vocab) { return (vocab + kTally * each - 1) / (kTally * each); }
inline int each_of(int rows, int vocab) {
  return (int64_t)rows * chunks_of(kMany, vocab) < 256 ? kFew : kMany;
}
static_assert(kMaxChunks * kTally * kFew == 1 << 20, "all chunks of the largest vocabulary");
__host__ __device__ inline size_t row_bytes(int C) { return (kCands * 8 + (size_t)C * sizeof(Chunk) + 15) / 16 * 16; }
__device__ __forceinline__ Work work_of(const SampleArgs& a, int row, int C) {
  char* p = static_cast<char*>(a.ws) + row_bytes(C) * row;
  return Work{reinterpret_cast<uint64_t*>(p), reinterpret_cast<Chunk*>(p + kCands * 8)};
}

// Half octave of a logit, in fp32: any function does that never rises with z and is
// the same everywhere. x = -2 t (from halves, which do not overflow); its part
// inside the bin is the fraction.
__device__ __forceinline__ float depth_of(float z, float ref, float c4) { return (0.5f * ref - 0.5f * z) * c4; }
__device__ __forceinline__ int bin_of(float x) { return (int)fminf(x, (float)(kBins - 1)); }
__device__ __forceinline__ float c4_of(const Request& q) { return (float)fmin(q.c / 8, 3e38); }
// whether top-p is a share of the mass of tokens that no list may hold
__device__ __forceinline__ bool share_of_all(const Request& q, int V) { return q.p < 1.0 && q.k >= (uint32_t)V; }

__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, o));
  return v;
}
// Inclusive scan of a wave by lane moves inside the vector unit: rows of 16 shifted
// by 1, 2, 4 and 8, then the last lane of a row added to the next row, and that
// of the lower half to the upper.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint64_t add_moved(uint64_t v) {
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)v, CTRL, ROWS, 0xf, false);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(v >> 32), CTRL, ROWS, 0xf, false);
  return v + (((uint64_t)hi << 32) | lo);
}
__device__ __forceinline__ uint64_t wave_scan_u64(uint64_t v) {
  v = add_moved<0x111, 0xf>(v);  // row_shr 1, 2, 4, 8
  v = add_moved<0x112, 0xf>(v);
  v = add_moved<0x114, 0xf>(v);
  v = add_moved<0x118, 0xf>(v);
  v = add_moved<0x142, 0xa>(v);  // row_bcast 15 into rows 1 and 3
  return add_moved<0x143, 0xc>(v);  // row_bcast 31 into rows 2 and 3
}
__device__ __forceinline__ uint64_t lane_u64(uint64_t v, int lane) {
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, lane);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(v >> 32), lane);
  return ((uint64_t)hi << 32) | lo;
}
__device__ __forceinline__ uint64_t wave_sum_u64(uint64_t v) { return lane_u64(wave_scan_u64(v), 63); }

// Four consecutive logits, bounded, those past the row as -inf. Rows start at any
// fp32 (a 16-byte load takes any 4-byte address).
typedef float float4_any __attribute__((ext_vector_type(4), aligned(4)));
__device__ __forceinline__ void load4(const float* z, int i, int V, float* v) {
  if (i + 4 <= V) {
    const float4_any x = *reinterpret_cast<const float4_any*>(z + i);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = bounded(x[e]);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = i + e < V ? bounded(z[i + e]) : -INFINITY;
  }
}

constexpr int kCopies = 4;     // of the histogram, by lane: tokens of one bin meet less often
constexpr int kPicked = 1024;  // tokens of a chunk that may be listed, at most
template <int EACH>
__global__ __launch_bounds__(kTally, 8) void tally_kernel(SampleArgs a) {
  constexpr int kWaves = kTally / 64;
  __shared__ double parts[32];
  __shared__ uint2 picked[kPicked];  // logit, id
  __shared__ uint32_t cnt[kBins * kCopies];
  __shared__ uint32_t cursor[kBins];
  __shared__ uint64_t red[kWaves];
  __shared__ uint32_t red_n[kWaves], red_top[kWaves], red_in[kWaves];
  __shared__ int limit, list_bin;
  const int C = gridDim.x, c = blockIdx.x, row = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const Work w = work_of(a, row, C);
  const float* z = a.logits + (int64_t)row * a.row_stride;
  const int first = c * (kTally * EACH) + 4 * tid;  // v[j]: id first + kTally * (j & ~3) + (j & 3)
  float v[EACH];
#pragma unroll
  for (int j = 0; j < EACH; j += 4) load4(z, first + j * kTally, a.vocab, v + j);
  const Request q = request_of(a, row);
  for (int i = tid; i < kBins * kCopies; i += kTally) cnt[i] = 0;
  if (tid < 32) parts[tid] = octave_part(tid);
  float most = v[0];
#pragma unroll
  for (int j = 1; j < EACH; ++j) most = fmaxf(most, v[j]);
  uint32_t top = wave_max_u32(ordered_bits(most + 0.0f));
  if (lane == 0) red_top[wave] = top;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kWaves; ++i) top = max(top, red_top[i]);
  if (top <= kDead) {
    if (tid == 0) w.head[c] = Chunk{kDead, kBins - 1, 0, 0, 0};
    return;
  }
  const float ref = from_ordered_bits(top);
  const float c4 = c4_of(q);
  const bool filtered = q.filtered(), need_mass = !filtered || share_of_all(q, a.vocab);
  const uint32_t room = (uint32_t)(kCands / C);
  const int copy = tid % kCopies;
  auto bin = [&](float x) { return bin_of(depth_of(x, ref, c4)); };
  // (a wave) this lane's two bins' counts through each, and how many bins fit the list
  auto bins_that_fit = [&](uint32_t& x0, uint32_t& x1) {
    uint32_t c0 = 0, c1 = 0;
#pragma unroll
    for (int k = 0; k < kCopies; ++k) c0 += cnt[2 * lane * kCopies + k], c1 += cnt[(2 * lane + 1) * kCopies + k];
    x1 = (uint32_t)wave_scan_add((int)(c0 + c1));
    x0 = x1 - c1;
    return (int)__popcll(__ballot(x0 <= room)) + (int)__popcll(__ballot(x1 <= room));
  };
  // First the threads' largest alone: a half octave through which they are more than
  // the list holds cannot be listed, nor any below. Most tokens lie there, and are
  // done with after one comparison.
  if (filtered) {
    if (most > -INFINITY) atomicAdd(&cnt[bin(most) * kCopies + copy], 1u);
    __syncthreads();
    if (wave == 0) {
      uint32_t x0, x1;
      const int f = bins_that_fit(x0, x1);
      if (lane == 0) limit = f;
#pragma unroll
      for (int k = 0; k < 2 * kCopies; ++k) cnt[2 * lane * kCopies + k] = 0;
    }
  }
  uint64_t sum = 0;
  if (need_mass)
#pragma unroll
    for (int j = 0; j < EACH; ++j)
      if (v[j] != -INFINITY) sum += mass_of(parts, exponent_of(v[j], ref, q.c));
  uint32_t tokens = 0;  // of the wave
#pragma unroll
  for (int j = 0; j < EACH; ++j) tokens += (uint32_t)__popcll(__ballot(v[j] != -INFINITY));
  if (need_mass) sum = wave_sum_u64(sum);
  if (lane == 0) red[wave] = sum, red_n[wave] = tokens;
  __syncthreads();
  const int end = filtered ? limit : 0;
  // below any logit of a half octave before `end`: one half octave deeper, and the rounding of that
  float border = ref - 2.0f * (float)(end + 1) / c4;
  border = end == kBins ? -INFINITY : border - fabsf(border) * 0x1p-22f;
  uint32_t in = 0;
  if (filtered) {
#pragma unroll
    for (int j = 0; j < EACH; ++j) in += (uint32_t)__popcll(__ballot(v[j] >= border && v[j] != -INFINITY));
    if (lane == 0) red_in[wave] = in;
  }
  __syncthreads();
  uint32_t n_in = 0, at = 0;
  if (filtered) {
#pragma unroll
    for (int i = 0; i < kWaves; ++i) n_in += red_in[i], at += i < wave ? red_in[i] : 0;
  }
  const bool few = n_in <= kPicked;  // else (lists that hold most of a short row) all are looked at again
  if (few && n_in) {
#pragma unroll
    for (int j = 0; j < EACH; ++j) {
      const bool is = v[j] >= border && v[j] != -INFINITY;
      const uint64_t mask = __ballot(is);
      const uint32_t before = __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0u));
      if (is) picked[at + before] = make_uint2(__float_as_uint(v[j]), (uint32_t)(first + kTally * (j & ~3) + (j & 3)));
      at += (uint32_t)__popcll(mask);
    }
  }
  __syncthreads();
  // each token that may be listed to f(logit, id, half octave)
  auto each_in = [&](auto f) {
    if (few) {
#pragma unroll
      for (int i = 0; i < kPicked / kTally; ++i)
        if (i * kTally + tid < (int)n_in) {
          const uint2 x = picked[i * kTally + tid];
          f(__uint_as_float(x.x), (int)x.y, bin(__uint_as_float(x.x)));
        }
    } else {
#pragma unroll
      for (int j = 0; j < EACH; ++j)
        if (v[j] >= border && v[j] != -INFINITY) f(v[j], first + kTally * (j & ~3) + (j & 3), bin(v[j]));
    }
  };
  if (filtered)
    each_in([&](float, int, int b) {
      if (b < end) atomicAdd(&cnt[b * kCopies + copy], 1u);
    });
  __syncthreads();
  if (wave == 0) {
    // counts through each bin; the deepest bin down to which they fit the list
    uint32_t x0, x1;
    const int f = min(bins_that_fit(x0, x1), end);
    const uint32_t before = (uint32_t)__shfl_up((int)x1, 1);
    cursor[2 * lane] = lane ? before : 0u;
    cursor[2 * lane + 1] = x0;
    // tokens through the last bin that fits, bin f - 1 (lane (f - 1) / 2's second or first)
    const uint32_t n_list = f ? (uint32_t)__builtin_amdgcn_readlane((int)(f & 1 ? x0 : x1), (f - 1) >> 1) : 0u;
    if (lane == 0) {
      list_bin = f - 1;
      uint64_t s = red[0], n = red_n[0];
      for (int i = 1; i < kWaves; ++i) s += red[i], n += red_n[i];
      w.head[c] = Chunk{top, f - 1, n_list, (uint32_t)n, s};
    }
  }
  if (!filtered) return;
  __syncthreads();
  const int lb = list_bin;
  each_in([&](float x, int id, int b) {
    if (b <= lb) w.list[(size_t)c * room + atomicAdd(&cursor[b], 1u)] = rank_key(x + 0.0f, id);
  });
}

constexpr int kHeld = kCands / kDraw;  // keys of a thread

struct Shared {
  uint64_t seg[kSegs];         // segment masses; in the searches, their own tables
  uint64_t more[kDraw];        // their other tables
  uint64_t red[2][kDraw / 64];
  uint64_t mass[kBins];        // of the keys through each bin
  uint32_t cnt[kBins];         // keys through each bin
  uint64_t above_mass, above, key;
  uint32_t top[kDraw / 64];
  uint32_t n, m, pick;
  uint32_t n_list[kMaxChunks];
  uint32_t rank[kDraw];
  double parts[32];
};
static_assert(kBins * kCopies <= kDraw, "a thread for each bin of the copies");
static_assert(kSegs >= kDigit && 2 * kDraw >= kDigit, "masses and counts of the digits");

// Inclusive scan over the block, and the block's sum. One barrier: wave sums go to
// one of two places in turn, so that a wave that is a scan ahead overwrites none.
struct Scan {
  uint64_t (*red)[kDraw / 64];
  int turn = 0;
  uint64_t sum = 0;
  __device__ __forceinline__ uint64_t operator()(uint64_t v) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint64_t x = wave_scan_u64(v);
    if (lane == 63) red[turn][wave] = x;
    __syncthreads();
    const uint64_t y = wave_scan_u64(lane < kDraw / 64 ? red[turn][lane] : 0);
    turn ^= 1;
    sum = lane_u64(y, 63);
    return x + (wave ? lane_u64(y, wave - 1) : 0);
  }
};

struct Row {
  const float* z;
  int V;
  float ref;   // the largest logit
  uint32_t top;
  float c4;
  Request q;
  const double* parts; // of an octave
  uint64_t threshold;  // smallest kept key
  __device__ uint64_t mass_at(float x) const { return mass_of(parts, exponent_of(x, ref, q.c)); }
  __device__ uint64_t mass(uint64_t key) const { return mass_at(key_val(key)); }
  __device__ float depth(uint64_t key) const { return depth_of(key_val(key), ref, c4); }
  __device__ uint64_t weight(int i, bool& kept) const {
    const float x = clean(z[i]);
    kept = false;
    if (x == -INFINITY || rank_key(x, i) < threshold) return 0;
    const double t = exponent_of(x, ref, q.c);
    if (q.min_p > 0.0 && x != ref && exp2_64(parts, t) < q.min_p) return 0;
    kept = true;
    return mass_of(parts, t);
  }
};

// The key at which the kept prefix ends, searched digit by digit (11, 11 and 10
// bits of the ordered logit) over the row's tokens with key >= floor: the n-th
// (by count), or the last whose preceding mass is below `want`. Equal logits are
// cut in id order.
template <bool BY_MASS>
__device__ uint64_t search_row(Shared& sh, Scan& scan, const Row& r, uint64_t n, double want, uint64_t floor) {
  uint64_t* mass = sh.seg;
  uint32_t* cnt = reinterpret_cast<uint32_t*>(sh.more);
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
        const uint64_t m = r.mass_at(z);
        if (m) atomicAdd((unsigned long long*)&mass[d], (unsigned long long)m);
      }
    }
    __syncthreads();
    // scanned from the largest digit: thread t holds digits D - 1 - 2 t and D - 2 - 2 t
    const int D = 1 << bits;
    const int d0 = D - 1 - 2 * tid, d1 = d0 - 1;
    const uint64_t c0 = d0 >= 0 ? cnt[d0] : 0, c1 = d1 >= 0 ? cnt[d1] : 0;
    const uint64_t m0 = d0 >= 0 ? mass[d0] : 0, m1 = d1 >= 0 ? mass[d1] : 0;
    const uint64_t cs = above + scan(c0 + c1) - c0 - c1;
    const uint64_t ms = BY_MASS ? above_mass + scan(m0 + m1) - m0 - m1 : 0;
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
    const uint64_t one = r.mass_at(from_ordered_bits(prefix));
    uint32_t lo = 0;  // smallest t >= 1 with above_mass + t * one >= want, at most equal
    while (lo + 1 < t) {
      const uint32_t mid = (lo + t) / 2;
      if ((double)(above_mass + mid * one) < want) lo = mid;
      else t = mid;
    }
  } else if (n - above < equal) {
    t = (uint32_t)(n - above);
  }
  if (t == equal) return max((uint64_t)prefix << 32, floor);  // all of them
  // the t-th id: equal logits counted by blocks of kDraw ids
  uint32_t seen = 0;
  for (int i0 = 0; i0 < r.V; i0 += kDraw) {
    const int i = i0 + tid;
    const bool is = i < r.V && ordered_bits(clean(r.z[i])) == prefix;
    const uint64_t x = scan(is ? 1 : 0);
    if (is && seen + x == t) sh.key = rank_key(from_ordered_bits(prefix), i);
    seen += (uint32_t)scan.sum;
    if (seen >= t) break;
  }
  __syncthreads();
  return sh.key;
}

// The same among the listed keys >= floor (a thread holds kHeld of them, 0: none) of
// bin `bin`, which has `size`; `above` tokens and `above_mass` lie in the bins before.
// More than kRanked keys are first narrowed to the part of the bin (1024, a thread
// each) in which the prefix ends; the keys that remain are ranked by counting.
// False: more of those than threads (equal logits).
constexpr uint32_t kRanked = 256;
template <bool BY_MASS>
__device__ __forceinline__ bool search_bin(Shared& sh, Scan& scan, const Row& r, const uint64_t (&held)[kHeld], int bin,
                                           uint32_t size, uint64_t n, double want, uint64_t above, uint64_t above_mass,
                                           uint64_t floor, uint64_t* key_out) {
  const int tid = threadIdx.x;
  uint64_t* mass = sh.more;                             // [kDraw]
  uint32_t* cnt = reinterpret_cast<uint32_t*>(sh.seg);  // [kDraw]
  auto part_of = [&](uint64_t k) {  // -1: not of the bin
    if (k < floor || k == 0) return -1;
    const float x = r.depth(k);
    return bin_of(x) != bin ? -1 : (int)fminf((x - (float)bin) * kDraw, (float)(kDraw - 1));
  };
  auto inside = [&](uint64_t cb, uint64_t mb) { return BY_MASS ? (cb == 0 || (double)mb < want) : cb < n; };
  int part = -2;  // any
  __syncthreads();
  if (tid == 0) sh.m = 0, sh.n = 0;
  if (size > kRanked) {
    cnt[tid] = 0;
    if (BY_MASS) mass[tid] = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
      const int p = part_of(held[i]);
      if (p < 0) continue;
      atomicAdd(&cnt[p], 1u);
      if (BY_MASS) atomicAdd((unsigned long long*)&mass[p], (unsigned long long)r.mass(held[i]));
    }
    __syncthreads();
    const uint64_t c0 = cnt[tid], m0 = BY_MASS ? mass[tid] : 0;
    const uint64_t cb = above + scan(c0) - c0;
    const uint64_t mb = BY_MASS ? above_mass + scan(m0) - m0 : 0;
    const bool in = c0 && inside(cb, mb);  // a prefix of the parts
    if (in) atomicMax(&sh.m, (uint32_t)tid);
    __syncthreads();
    if (in && sh.m == (uint32_t)tid) sh.above = cb, sh.above_mass = mb, sh.pick = (uint32_t)c0;
    __syncthreads();
    part = (int)sh.m;
    above = sh.above;
    above_mass = sh.above_mass;
    if (sh.pick > kDraw) return false;
  } else {
    __syncthreads();
  }
  uint64_t* mine = sh.seg;
  sh.rank[tid] = 0;
#pragma unroll
  for (int i = 0; i < kHeld; ++i) {
    const int p = part_of(held[i]);
    if (p >= 0 && (part < 0 || p == part)) mine[atomicAdd(&sh.n, 1u)] = held[i];
  }
  __syncthreads();
  const uint32_t m = sh.n;
  const uint64_t key = tid < (int)m ? mine[tid] : 0;
  {
    // a wave 64 of the keys against its part of all: as many parts as waves are left
    const int wave = tid >> 6, groups = max(((int)m + 63) >> 6, 1), parts = kDraw / 64 / groups;
    const int x = wave % groups * 64 + (tid & 63), part = wave / groups;
    const uint64_t k = x < (int)m ? mine[x] : ~0ull;
    const int each = ((int)m + parts - 1) / parts, end = min((int)m, (part + 1) * each);
    uint32_t above_k = 0;
#pragma unroll 8
    for (int i = part * each; i < end; ++i) above_k += mine[i] > k;
    if (above_k && part < parts) atomicAdd(&sh.rank[x], above_k);
  }
  __syncthreads();
  const uint32_t rank = sh.rank[tid];
  if (!BY_MASS) {  // the token of rank n - 1, or the last
    const uint64_t last = n - above < m ? n - above : m;
    if (tid < (int)m && rank == last - 1) sh.key = key;
    __syncthreads();
    *key_out = sh.key;
    __syncthreads();
    return true;
  }
  uint64_t* by_rank = sh.more;              // masses
  uint64_t* key_by_rank = sh.seg + kDraw;
  if (tid < (int)m) {
    by_rank[rank] = r.mass(key);
    key_by_rank[rank] = key;
  }
  __syncthreads();
  const uint64_t w = tid < (int)m ? by_rank[tid] : 0;
  const uint64_t x = above_mass + scan(w);  // mass through rank tid
  // the ranks inside are a prefix: the last of them
  if (tid < (int)m && inside(above + tid, x - w) && (tid + 1 == (int)m || !inside(above + tid + 1, x)))
    sh.key = key_by_rank[tid];
  __syncthreads();
  *key_out = sh.key;
  __syncthreads();
  return true;
}
static_assert(kSegs >= 2 * kDraw, "ranks and their keys fit the segment masses");

__global__ __launch_bounds__(kDraw) void draw_kernel(SampleArgs a, int C, int chunk) {
  __shared__ Shared sh;
  Scan scan{sh.red};
  const int row = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const Work w = work_of(a, row, C);
  Row r;
  r.z = a.logits + (int64_t)row * a.row_stride;
  r.V = a.vocab;
  r.q = request_of(a, row);
  r.parts = sh.parts;
  if (tid < 32) sh.parts[tid] = octave_part(tid);
  const Chunk head = tid < C ? w.head[tid] : Chunk{kDead, kBins - 1, 0, 0, 0};
  {
    const uint32_t top = wave_max_u32(head.top);
    if (lane == 0) sh.top[wave] = top;
    __syncthreads();
    r.top = sh.top[0];
#pragma unroll
    for (int i = 1; i < kDraw / 64; ++i) r.top = max(r.top, sh.top[i]);
  }
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
  uint64_t total = 0;                   // all kept mass
  double part = r.q.u;                  // share of the segments' mass at which the draw lies
  const float ref = r.ref;
  bool from_list = false;

  // the chunks' masses against the row's largest
  const double down = head.top > kDead ? exponent_of(from_ordered_bits(head.top), r.ref, r.q.c) : 0.0;
  const uint64_t chunk_mass = head.mass ? (uint64_t)((double)head.mass * exp2_64(sh.parts, down) + 0.5) : 0;
  const uint64_t counts = (scan((uint64_t)head.n_list << 32 | head.tokens), scan.sum);  // both under 2^21
  const uint32_t valid = (uint32_t)counts, N = (uint32_t)(counts >> 32);  // tokens above -inf, listed ones

  uint64_t held[kHeld];  // listed keys of this thread, 0: none
  if (filtered) {
    const bool of_all = share_of_all(r.q, r.V), by_k = r.q.k < valid;
    bool by_p = r.q.p < 1.0;
    uint64_t all = 0;  // mass that top-p is a share of
    if (of_all) scan(chunk_mass), all = scan.sum;
    if (tid < C) sh.n_list[tid] = head.n_list;
    __syncthreads();
    const uint32_t room = (uint32_t)(kCands / C);
    const float inv_room = 1.0f / (float)room;
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
      const uint32_t at = i * kDraw + tid, c = (uint32_t)(((float)at + 0.5f) * inv_room);  // at / room: exact under 2^13
      held[i] = c < (uint32_t)C && at - c * room < sh.n_list[c] ? w.list[at] : 0;
    }
    // counts, or counts and masses, of the keys >= floor through each bin
    auto tally = [&](bool with_mass, uint64_t floor) {
      __syncthreads();
      uint64_t* mass = sh.more;                             // copies of the histogram, by lane
      uint32_t* cnt = reinterpret_cast<uint32_t*>(sh.seg);
      if (tid < kBins * kCopies) cnt[tid] = 0, mass[tid] = 0;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kHeld; ++i) {
        if (held[i] < floor || held[i] == 0) continue;
        const int b = bin_of(r.depth(held[i])) * kCopies + tid % kCopies;
        atomicAdd(&cnt[b], 1u);
        if (with_mass) {
          const uint64_t g = r.mass(held[i]);
          if (g) atomicAdd((unsigned long long*)&mass[b], (unsigned long long)g);
        }
      }
      __syncthreads();
      if (wave == 0) {
        uint32_t c0 = 0, c1 = 0;
        uint64_t m0 = 0, m1 = 0;
#pragma unroll
        for (int i = 0; i < kCopies; ++i) {
          c0 += cnt[2 * lane * kCopies + i];
          c1 += cnt[(2 * lane + 1) * kCopies + i];
          m0 += mass[2 * lane * kCopies + i];
          m1 += mass[(2 * lane + 1) * kCopies + i];
        }
        const uint32_t cx = (uint32_t)wave_scan_u64(c0 + c1);
        const uint64_t mx = wave_scan_u64(m0 + m1);
        sh.cnt[2 * lane] = cx - c1;
        sh.cnt[2 * lane + 1] = cx;
        sh.mass[2 * lane] = mx - m1;
        sh.mass[2 * lane + 1] = mx;
      }
      __syncthreads();
    };
    auto first_bin = [&](auto before) {  // first bin, of the last at most, that is not `before`
      int lo = 0, hi = kBins - 1;
      while (lo < hi) {
        const int mid = (lo + hi) / 2;
        if (before(mid)) lo = mid + 1;
        else hi = mid;
      }
      return lo;
    };
    // Whether the lists hold every token at or above a logit: a chunk's list ends at
    // a half octave below its own largest. (Then the counts and masses of the keys
    // down to it are the row's, too.)
    auto complete = [&](float z) {
      const bool ok = head.tokens == head.n_list || ordered_bits(z) > head.top ||
                      bin_of(depth_of(z, from_ordered_bits(head.top), r.c4)) <= head.list_bin;
      return __syncthreads_and(ok) != 0;
    };
    const bool whole = N == valid;  // every token is listed
    // mass of the row's tokens at or above the threshold, from the row
    auto row_mass = [&]() {
      uint64_t m = 0;
      for (int i = tid; i < r.V; i += kDraw) {
        const float z = clean(r.z[i]);
        if (z != -INFINITY && rank_key(z, i) >= r.threshold) m += r.mass_at(z);
      }
      scan(m);
      return scan.sum;
    };
    from_list = true;
    if (by_k) {
      from_list = r.q.k <= N;
      if (from_list) {
        tally(false, 0);
        const int b = first_bin([&](int i) { return sh.cnt[i] < r.q.k; });
        const uint64_t above = b ? sh.cnt[b - 1] : 0;
        from_list = search_bin<false>(sh, scan, r, held, b, (uint32_t)(sh.cnt[b] - above), r.q.k, 0.0, above, 0, 0, &r.threshold) &&
                    complete(key_val(r.threshold));
      }
      if (!from_list) {
        r.threshold = search_row<false>(sh, scan, r, r.q.k, 0.0, 0);
        if (by_p) all = row_mass();
      }
    } else if (by_p && !of_all && !whole) {  // top-k that keeps all of a row with few tokens
      from_list = false;
      all = row_mass();
    }
    if (from_list && (by_p || (!by_k && r.q.min_p > 0.0))) {
      tally(true, r.threshold);
      if (!of_all) all = sh.mass[kBins - 1];
    }
    const double want = r.q.p * (double)all;
    // min_p alone: its border, taken half an octave deeper, whatever way that rounds
    bool by_min = false;
    if (!by_k && r.q.min_p > 0.0 && from_list) {
      const double depth = r.q.min_p < 1.0 ? -2.0 * log2(r.q.min_p) + 1.0 : 1.0;
      const int b = bin_of((float)depth);
      by_min = !by_p || (b < kBins - 1 && (double)sh.mass[b] < want);
      if (by_min) {
        const float z = (float)((double)r.ref - depth * 16 / r.q.c);
        by_min = whole || (z > -INFINITY && complete(z));
        if (by_min) by_p = false;  // top-p, if it is on, cuts deeper than min_p
      }
    }
    if (!by_k && !by_p && !by_min) from_list = whole;  // nothing is cut
    if (by_p) {
      if (from_list) from_list = (double)sh.mass[kBins - 1] >= want;  // else it ends below the lists
      if (from_list) {
        const int b = first_bin([&](int i) { return sh.cnt[i] == 0 || (double)sh.mass[i] < want; });
        const uint64_t above = b ? sh.cnt[b - 1] : 0, above_mass = b ? sh.mass[b - 1] : 0;
        uint64_t key = 0;
        from_list = search_bin<true>(sh, scan, r, held, b, (uint32_t)(sh.cnt[b] - above), 0, want, above, above_mass,
                                     r.threshold, &key) &&
                    (by_k || complete(key_val(key)));
        if (from_list) r.threshold = key;
      }
      if (!from_list) r.threshold = search_row<true>(sh, scan, r, 0, want, r.threshold);
    }
    __syncthreads();
    for (int i = tid; i < n_seg; i += kDraw) sh.seg[i] = 0;
    __syncthreads();
    if (from_list) {
      uint64_t count = 0;
#pragma unroll
      for (int i = 0; i < kHeld; ++i) {
        const uint64_t k = held[i];
        if (k < r.threshold || k == 0) continue;
        const float z = key_val(k);
        const double t = exponent_of(z, r.ref, r.q.c);
        if (r.q.min_p > 0.0 && z != r.ref && exp2_64(sh.parts, t) < r.q.min_p) continue;
        ++count;
        atomicAdd((unsigned long long*)&sh.seg[key_id(k) / kSeg], (unsigned long long)mass_of(sh.parts, t));
      }
      scan(count);
      n_kept = (uint32_t)scan.sum;
    }
  } else {
    // the chunk from the chunks' masses, then the draw inside it, against its own
    // largest logit, at the share of its mass that is left
    const uint64_t m = chunk_mass, x = scan(m);
    total = scan.sum;
    const double want = r.q.u * (double)total;
    if (m && (double)x > want && !((double)(x - m) > want)) {
      sh.pick = tid;
      sh.above_mass = x - m;
      sh.above = m;
      sh.n = head.top;
    }
    __syncthreads();
    first_seg = (int)sh.pick * (chunk / kSeg);
    last_seg = min(n_seg, first_seg + chunk / kSeg);
    part = fmin(fmax((want - (double)sh.above_mass) / (double)sh.above, 0.0), 1.0 - 0x1p-52);
    r.ref = from_ordered_bits(sh.n);
    n_kept = valid;
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
      scan(count);
      n_kept = (uint32_t)scan.sum;
    }
  }
  __syncthreads();
  // the segment: thread t holds segments 2 t and 2 t + 1
  double want;
  {
    const uint64_t s0 = 2 * tid < n_seg ? sh.seg[2 * tid] : 0;
    const uint64_t s1 = 2 * tid + 1 < n_seg ? sh.seg[2 * tid + 1] : 0;
    const uint64_t x = scan(s0 + s1);
    if (filtered) total = scan.sum;
    want = part * (double)scan.sum;
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
  const uint64_t x = c0 + scan(m);
  if (m && (double)x > want && !((double)(x - m) > want)) {
    a.tok[row] = id;
    if (a.kept) a.kept[row] = (int32_t)n_kept;
    if (a.logp)
      a.logp[row] = (float)(exponent_of(clean(r.z[id]), ref, r.q.c) * (0.6931471805599453 / 32) - log((double)total * 0x1p-43));
  }
}

}  // namespace

// Of the smaller chunks, whichever a call takes: never falls when an argument grows.
size_t sample_ws_bytes(int32_t rows, int32_t vocab) { return row_bytes(chunks_of(kFew, vocab)) * rows; }

hipError_t launch_sample(const SampleArgs& a, hipStream_t s) {
  const int each = each_of(a.rows, a.vocab), C = chunks_of(each, a.vocab);
  if (each == kFew) {
    hipLaunchKernelGGL(tally_kernel<kFew>, dim3(C, a.rows), dim3(kTally), 0, s, a);
  } else {
    hipLaunchKernelGGL(tally_kernel<kMany>, dim3(C, a.rows), dim3(kTally), 0, s, a);
  }
  hipLaunchKernelGGL(draw_kernel, dim3(a.rows), dim3(kDraw), 0, s, a, C, kTally * each);
  return hipGetLastError();
}

}  // namespace msd
