// Attention of a block's rows over the paged cache.
//
// A sequence's keys are walked in blocks of 32 positions: those of the sinks, those
// from the first row's window on, and one block of the rows' own keys where
// they come beside the cache; blocks outside the window are not read. A
// workgroup owns a chunk of consecutive blocks of one (sequence, kv head) and
// up to 3 tiles of 16 queries (query head of the kv head's group, slot), its 4
// waves a block each in turn:
//   S^T[key][query] = K Q^T   MFMA 16x16x32 bf16. 8-bit codes become bf16 in
//                             registers, multiplied by their block's scale in
//                             the same instruction: exact, as a code has 4
//                             significant bits and the scale is a power of two.
//                             Queries are bf16, or, where they are rotated
//                             here, a bf16 hi + lo pair (16 significant bits);
//   P = exp2(S - m)           online softmax in fp32; the running maximum of a
//                             query moves only when a score passes it by 2^8,
//                             and no lanes talk on a block that moves none: sums
//                             stay per lane until the end;
//   O += P V                  P as a bf16 hi + lo pair against exact values, staged
//                             row-wise in the wave's LDS and read back by the
//                             transposing LDS read. Rounding P to one bf16 would
//                             cost as much as the output's own rounding.
// A wave loads its next block as soon as the scores have read the keys of the current
// one, into the same registers. The block's own keys go first, while the first
// cached block is on its way.
// The waves are joined in LDS; a chunk that is its sequence's only one writes
// the output, others leave (max, sum, output) in the workspace and a second
// kernel joins them in chunk order. No atomics on values: a run repeats bit for
// bit.
//
// Values that no query sees are zeroed as they are staged, so NaN in stale
// rows, past the window or past the length meets no product. A non-finite value that
// only some of the wave's queries see would reach the others as 0 * NaN: where a
// wave ends with a non-finite output, it walks its blocks again with such
// values taken out of the products and added to the queries that see them.
#pragma once
#include "paged_plan.h"

namespace msd {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
typedef short v4i16 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) v4i16 lds_v4i16;

template <int HD>
struct Lds {
  static constexpr int kVS = HD + 4;  // bf16 per staged row, conflict-free strides
  static constexpr int kOS = HD + 4;  // floats per row of a wave's output
  static constexpr int kRegion = kBlock * kVS * 2 > 16 * kOS * 4 ? kBlock * kVS * 2 : 16 * kOS * 4;
};

__device__ __forceinline__ bool finite_bf16(uint32_t b) { return (b & 0x7F80u) != 0x7F80u; }
// a pair of bf16, non-finite ones as zero
__device__ __forceinline__ uint32_t finite_pair(uint32_t w) {
  return (finite_bf16(w) ? w & 0xFFFFu : 0u) | (finite_bf16(w >> 16) ? w & 0xFFFF0000u : 0u);
}

// 8 codes as bf16, times a power of two
__device__ __forceinline__ bf16x8 widen8(uint32_t w0, uint32_t w1, float scale) {
  u32x4 r;
  r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, scale, false));
  r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, scale, true));
  r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, scale, false));
  r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, scale, true));
  return __builtin_bit_cast(bf16x8, r);
}

// Operand place of the 8-dim group c of a row: k-step and lane group. bf16
// rows: 8 dims a lane and k-step. 8-bit rows: a lane's 16-byte load holds the 8
// dims of two k-steps.
template <bool FP8>
__device__ __forceinline__ void operand_place(int c, int& kk, int& g) {
  if (FP8) {
    kk = 2 * (c >> 3) + (c & 1);
    g = (c & 7) >> 1;
  } else {
    kk = c >> 2;
    g = c & 3;
  }
}
template <bool FP8>
__device__ __forceinline__ int operand_group(int kk, int g) {  // its inverse
  return FP8 ? 8 * (kk >> 1) + 2 * g + (kk & 1) : 4 * kk + g;
}

template <int HD, bool FP8, int QPW, bool ROT>
struct Core {
  static constexpr int KSTEPS = HD / 32;
  static constexpr int DSUB = HD / 16;
  static constexpr int QPARTS = ROT ? 2 : 1;
  static constexpr int KW = FP8 ? HD / 64 : HD / 32;       // 16-byte loads of a key row per lane
  static constexpr int EB = FP8 ? 1 : 2;                   // bytes of a cached element
  static constexpr int LPR = HD * EB / 16;                 // lanes of a value row
  static constexpr int VIT = LPR / 2;                      // 16-byte value loads of a block per lane
  static constexpr int KPI = 64 / LPR;                     // value rows of an iteration
  using L = Lds<HD>;

  const PagedAttnArgs a;
  const int* depth;     // LDS copies of the block's topology
  const uint64_t* ancs;
  const uint16_t* q_sh;
  uint16_t* vs;      // this wave's staged rows [kBlock][kVS]
  int lane, r16, g;
  int b, kvh, Len, end, pmax, cnt;
  int pq[QPW];       // position of this lane's query of each tile
  uint64_t anc[QPW];
  float s2;

  float mrun[QPW], lrun[QPW];
  floatx4 o[QPW][DSUB];

  // the wave's next cached block: keys, values, scales; which of its two 16-key tiles
  // have a page
  u32x4 xk[2][KW], xv[VIT];
  int xscale;        // lane t < 2: key scale of tile t; 2 + t: value scale
  int xvalid;        // bit t: tile t lies in a page (uniform)
  int x0;            // first position

  // lane t < 2: page of tile t of the block at k0, -2 past the sequence's end
  __device__ __forceinline__ int page_lane(int k0) const {
    const int pos = k0 + 16 * (lane & 1);
    return pos < end ? a.kv.page_table[(size_t)b * a.kv.max_pages + (pos >> a.kv.page_shift)] : -2;
  }

  __device__ __forceinline__ void load(int k0, int pages) {
    x0 = k0;
    xvalid = 0;
    const int mask = (1 << a.kv.page_shift) - 1;
    const char* kp[2];
    const char* vp[2];
    const uint8_t* sp[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      int pg = __builtin_amdgcn_readlane(pages, t);
      const bool ok = pg >= 0 && pg < a.kv.n_pages;
      if (pg != -2 && !ok && lane == 0) atomicOr(a.kv.status, 8u);
      xvalid |= ok ? 1 << t : 0;
      pg = ok ? pg : 0;
      const size_t plane = ((size_t)a.layer * a.kv.n_pages + pg) * a.kv.heads + kvh;
      const int off = (k0 + 16 * t) & mask;
      const size_t row = (plane << a.kv.page_shift) + off;
      kp[t] = static_cast<const char*>(a.kv.k) + row * (HD * EB);
      vp[t] = static_cast<const char*>(a.kv.v) + row * (HD * EB);
      if (FP8) sp[t] = reinterpret_cast<const uint8_t*>((plane << (a.kv.page_shift - 4)) + (off >> 4));
    }
    const uint32_t klane = r16 * (HD * EB) + 16 * g;
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int w = 0; w < KW; ++w) xk[j][w] = *reinterpret_cast<const u32x4*>(kp[j] + (klane + 64 * w));
#pragma unroll
    for (int it = 0; it < VIT; ++it)  // an iteration's rows lie in one tile: 16 % KPI = 0
      xv[it] = *reinterpret_cast<const u32x4*>(vp[it * KPI / 16] + (it * KPI % 16 * (HD * EB) + (uint32_t)lane * 16));
    if (FP8) {
      const uint8_t* sc = lane & 2 ? a.kv.v_scale : a.kv.k_scale;
      xscale = sc[reinterpret_cast<size_t>(lane & 1 ? sp[1] : sp[0])];
    }
  }

  __device__ __forceinline__ float block_scale(int i) const {
    return FP8 ? scale_value((uint32_t)__builtin_amdgcn_readlane(xscale, i)) : 1.0f;
  }

  // whether every query sees all of the block
  __device__ __forceinline__ bool is_open() const {
    return xvalid == 3 && x0 + kBlock <= Len &&
           (a.window <= 0 || pmax - x0 < a.window || x0 + kBlock <= a.sinks);
  }
  __device__ __forceinline__ bool sees(int t, int pos, int j) const {
    return ((xvalid >> j) & 1) && pos < end && pos <= pq[t] &&
           (a.window <= 0 || pq[t] - pos < a.window || pos < a.sinks);
  }

  // values of the cached block into the wave's LDS; rows that no query sees as zero
  __device__ __forceinline__ void stage(bool open) {
#pragma unroll
    for (int it = 0; it < VIT; ++it) {
      const int key = it * KPI + lane / LPR;
      const int t = it * KPI / 16;
      u32x4 w = xv[it];
      if (!open) {
        const int pos = x0 + key;
        const bool live = ((xvalid >> t) & 1) && pos < end &&
                          (a.window <= 0 || Len - pos < a.window || pos < a.sinks);
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = live ? w[i] : 0u;
      }
      uint16_t* dst = vs + key * L::kVS;
      if constexpr (FP8) {
        const float f = block_scale(2 + t);
        dst += (lane % LPR) * 16;
        *reinterpret_cast<bf16x8*>(dst) = widen8(w[0], w[1], f);
        *reinterpret_cast<bf16x8*>(dst + 8) = widen8(w[2], w[3], f);
      } else {
        *reinterpret_cast<u32x4*>(dst + (lane % LPR) * 8) = w;
      }
    }
  }

  __device__ __forceinline__ void clear(floatx4 (&sc)[QPW][2]) const {
#pragma unroll
    for (int t = 0; t < QPW; ++t)
#pragma unroll
      for (int j = 0; j < 2; ++j) sc[t][j] = floatx4{0.f, 0.f, 0.f, 0.f};
  }

  // sc[t][j] += K Q^T of every tile; frag(j, kk): K operand of the 16 keys j
  template <class F>
  __device__ __forceinline__ void scores(floatx4 (&sc)[QPW][2], F frag) {
#pragma unroll
    for (int kk = 0; kk < KSTEPS; ++kk) {
      const bf16x8 k0 = frag(0, kk), k1 = frag(1, kk);
#pragma unroll
      for (int t = 0; t < QPW; ++t)
#pragma unroll
        for (int p = 0; p < QPARTS; ++p) {
          const bf16x8 qf = *reinterpret_cast<const bf16x8*>(
              q_sh + (((t * KSTEPS + kk) * QPARTS + p) * 64 + lane) * 8);
          sc[t][0] = mfma16x16x32(k0, qf, sc[t][0]);
          sc[t][1] = mfma16x16x32(k1, qf, sc[t][1]);
        }
    }
  }

  // masked scores (base-2 units over s2, -inf where unseen) to the running
  // softmax and output
  template <bool CAREFUL>
  __device__ __forceinline__ void accumulate(floatx4 (&sc)[QPW][2]) {
    u32x4 ph[QPW], pl[QPW];
#pragma unroll
    for (int t = 0; t < QPW; ++t) {
      float mx = sc[t][0][0];
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) mx = fmaxf(mx, sc[t][j][r]);
      mx *= s2;  // s2 >= 0
      if (__ballot(mx > mrun[t] + 8.0f)) {
        mx = fmaxf(mx, __shfl_xor(mx, 16));
        mx = fmaxf(mx, __shfl_xor(mx, 32));
        const float mnew = fmaxf(mrun[t], mx);
        const float alpha = mrun[t] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(mrun[t] - mnew);
        lrun[t] *= alpha;
        mrun[t] = mnew;
        // o[t][ds][r] belongs to query 4 g + r, whose factor lane 4 g + r holds
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float ar = __shfl(alpha, 4 * g + r);
#pragma unroll
          for (int ds = 0; ds < DSUB; ++ds) o[t][ds][r] *= ar;
        }
      }
      const float mref = mrun[t] == -INFINITY ? 0.0f : mrun[t];
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          sc[t][j][r] = __builtin_amdgcn_exp2f(fmaf(sc[t][j][r], s2, -mref));
          lrun[t] += sc[t][j][r];
        }
      // P in the k order of the V operand: keys 4 g + r of the two 16-key tiles
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const float p0 = sc[t][x >> 1][2 * (x & 1)];
        const float p1 = sc[t][x >> 1][2 * (x & 1) + 1];
        ph[t][x] = pack_bf16x2(p0, p1);
        pl[t][x] = pack_bf16x2(p0 - bf_lo(ph[t][x]), p1 - bf_hi(ph[t][x]));
      }
    }
#pragma unroll
    for (int ds = 0; ds < DSUB; ++ds) {
      // transposing LDS reads: lane takes dim 16 ds + lane % 16 of keys 4 g + e
      // and 16 + 4 g + e (e < 4), the k order of P
      const uint16_t* p0 = vs + (4 * g + (r16 >> 2)) * L::kVS + 16 * ds + 4 * (r16 & 3);
      const v4i16 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16*)p0);
      const v4i16 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16*)(p0 + 16 * L::kVS));
      u32x4 w = __builtin_bit_cast(u32x4, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
      if (CAREFUL) {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = finite_pair(w[i]);
      }
      const bf16x8 vb = __builtin_bit_cast(bf16x8, w);
#pragma unroll
      for (int t = 0; t < QPW; ++t) {
        o[t][ds] = mfma16x16x32(__builtin_bit_cast(bf16x8, ph[t]), vb, o[t][ds]);
        o[t][ds] = mfma16x16x32(__builtin_bit_cast(bf16x8, pl[t]), vb, o[t][ds]);
      }
    }
    if (CAREFUL) {
      // the non-finite values, one key after the other, to the queries that
      // give it weight: query 4 g + r's weight of key 16 j + 4 gk + rk sits in lane
      // 16 gk + 4 g + r
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int rk = 0; rk < 4; ++rk)
          for (int gk = 0; gk < 4; ++gk) {
            const uint16_t* row = vs + (16 * j + 4 * gk + rk) * L::kVS + r16;
            bool any = false;
#pragma unroll
            for (int ds = 0; ds < DSUB; ++ds) any |= !finite_bf16(row[16 * ds]);
            if (!__ballot(any)) continue;
#pragma unroll
            for (int t = 0; t < QPW; ++t)
#pragma unroll
              for (int r = 0; r < 4; ++r) {
                const float p = __shfl(sc[t][j][rk], 16 * gk + 4 * g + r);
#pragma unroll
                for (int ds = 0; ds < DSUB; ++ds) {
                  const uint16_t v = row[16 * ds];
                  if (!finite_bf16(v) && p > 0.0f) o[t][ds][r] += bf2f(v);
                }
              }
          }
    }
  }

  __device__ __forceinline__ void reset() {
#pragma unroll
    for (int t = 0; t < QPW; ++t) {
      mrun[t] = -INFINITY;
      lrun[t] = 0.0f;
#pragma unroll
      for (int ds = 0; ds < DSUB; ++ds) o[t][ds] = floatx4{0.f, 0.f, 0.f, 0.f};
    }
  }

  // Blocks i0, i0 + kWaves, ... < i1 of the span. begin() issues the first
  // cached block's loads and looks up the pages of the second (in `pages`).
  __device__ __forceinline__ void begin(const Span& s, int i0, int i1, int& pages) {
    const int ic = min(i1, s.cached());
    pages = -2;
    if (i0 >= ic) return;
    const int k0 = s.first_pos(i0);
    const int first = page_lane(k0);
    if (i0 + kWaves < ic) pages = page_lane(s.first_pos(i0 + kWaves));
    load(k0, first);
  }

  template <bool CAREFUL>
  __device__ __forceinline__ void walk(const Span& s, int i0, int i1, int pages) {
    const int ic = min(i1, s.cached());
    // own blocks of this wave: indices from s.cached() on, congruent to i0
    for (int i = ic > i0 ? i0 + (ic - i0 + kWaves - 1) / kWaves * kWaves : i0; i < i1; i += kWaves)
      if (i >= s.cached()) own_block<CAREFUL>((i - s.cached()) * kBlock);
    for (int i = i0; i < ic; i += kWaves) {
      const bool open = is_open();
      // the wave's LDS reads of its previous block are done: one wave's LDS
      // accesses complete in order
      wave_lds_sync();
      stage(open);
      const float ks0 = block_scale(0), ks1 = block_scale(1);
      floatx4 sc[QPW][2];
      clear(sc);
      scores(sc, [&](int j, int kk) {
        if constexpr (FP8) return widen8(xk[j][kk >> 1][2 * (kk & 1)], xk[j][kk >> 1][2 * (kk & 1) + 1], j ? ks1 : ks0);
        else return __builtin_bit_cast(bf16x8, xk[j][kk]);
      });
      if (!open) {
#pragma unroll
        for (int t = 0; t < QPW; ++t)
#pragma unroll
          for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r)
              sc[t][j][r] = sees(t, x0 + 16 * j + 4 * g + r, j) ? sc[t][j][r] : -INFINITY;
      }
      if (i + kWaves < ic) {
        load(s.first_pos(i + kWaves), pages);
        if (i + 2 * kWaves < ic) pages = page_lane(s.first_pos(i + 2 * kWaves));
      }
      wave_lds_sync();
      accumulate<CAREFUL>(sc);
    }
  }

  // One row-wise copy in the wave's LDS of the rows' own keys (part 0: rounded to
  // bf16, 1: what that left) or values (part 2), slots first .. first + kBlock - 1;
  // slots past the count zero.
  __device__ __forceinline__ void stage_own(int first, int part) {
    const int64_t seq = b * a.new_seq + kvh * a.new_head;
    const int rows = min(cnt - first, kBlock) * (HD / 8);
    wave_lds_sync();
#pragma unroll 2
    for (int x = lane; x < rows; x += 64) {
      const int key = first + x / (HD / 8), c = x % (HD / 8);
      bf16x8 w;
      if (part == 2) {
        w = load16(a.v_new + seq + key * a.new_row + 8 * c);
      } else {
        float v[8];
        load_rotated8(a.k_new + seq + key * a.new_row, c, a.rope, (int64_t)Len + depth[key], v);
        bf16x8 hi, lo;
        split_vals(v, hi, lo);
        w = part == 0 ? hi : lo;
      }
      *reinterpret_cast<bf16x8*>(vs + (key - first) * L::kVS + 8 * c) = w;
    }
    for (int x = rows + lane; x < kBlock * (HD / 8); x += 64)
      *reinterpret_cast<bf16x8*>(vs + x / (HD / 8) * L::kVS + 8 * (x % (HD / 8))) = zero_bf16x8();
    wave_lds_sync();
  }

  // the rows' own keys; rotated ones enter as hi + lo, like the queries
  template <bool CAREFUL>
  __device__ __forceinline__ void own_block(int first) {
    floatx4 sc[QPW][2];
    clear(sc);
#pragma unroll 1
    for (int p = 0; p < QPARTS; ++p) {
      stage_own(first, p);
      scores(sc, [&](int j, int kk) {
        return *reinterpret_cast<const bf16x8*>(vs + (16 * j + r16) * L::kVS + 8 * operand_group<FP8>(kk, g));
      });
    }
    stage_own(first, 2);
#pragma unroll
    for (int t = 0; t < QPW; ++t)
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int slot = first + 16 * j + 4 * g + r;
          const int pos = Len + depth[slot];
          const bool vis = slot < cnt && ((anc[t] >> slot) & 1ull) &&
                           (a.window <= 0 || pq[t] - pos < a.window || pos < a.sinks);
          sc[t][j][r] = vis ? sc[t][j][r] : -INFINITY;
        }
    accumulate<CAREFUL>(sc);
  }

  __device__ __forceinline__ bool all_finite() const {
    bool ok = true;
#pragma unroll
    for (int t = 0; t < QPW; ++t)
#pragma unroll
      for (int ds = 0; ds < DSUB; ++ds)
#pragma unroll
        for (int r = 0; r < 4; ++r) ok &= __builtin_isfinite(o[t][ds][r]);
    return __ballot(!ok) == 0;
  }
};

template <int HD, bool FP8, int QPW, bool ROT>
__global__ __launch_bounds__(64 * kWaves, 2) void paged_attn_kernel(PagedAttnArgs a, Topo topo) {
  using C = Core<HD, FP8, QPW, ROT>;
  using L = Lds<HD>;
  constexpr int kThreads = 64 * kWaves;
  __shared__ __attribute__((aligned(16))) unsigned char region[kWaves][L::kRegion];
  __shared__ __attribute__((aligned(16))) uint16_t q_sh[QPW * C::KSTEPS * C::QPARTS * 512];
  __shared__ float ml_sh[kWaves][16][2];
  __shared__ int chunk0[kPagedPlanBatch + 1];
  __shared__ int G_sh;
  __shared__ int depth[kMaxSlots];
  __shared__ uint64_t ancs[kMaxSlots];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int G = a.n_heads / a.kv.heads;
  const int Qn = G * a.n_slots, QT = (Qn + 15) >> 4;

  // kv heads first: the hardware deals workgroups to the 8 XCDs in turn, so the
  // query groups of a chunk that re-read its keys meet in one L2 where the kv
  // heads are a multiple of 8
  int id = blockIdx.x;
  const int kvh = id % a.kv.heads;
  id /= a.kv.heads;
  const int qgi = id % a.groups;
  const int unit = id / a.groups;
  int b, c = 0, nch = 1;
  Span s;
  int i0 = 0, i1;
  if (wave == 1) {
    depth[lane] = topo.depth[lane];
    ancs[lane] = topo.anc[lane];
  }
  if (a.wgs > 0) {
    if (wave == 0) {
      const int g = plan_chunks(a, chunk0, blockIdx.x == 0);
      if (lane == 0) G_sh = g;
    }
    __syncthreads();
    if (blockIdx.x == 0)
      for (int i = tid; i <= a.batch; i += kThreads) a.plan[i] = chunk0[i];
    if (unit >= chunk0[a.batch]) return;
    int lo = 0, hi = a.batch;  // chunk0[lo] <= unit < chunk0[hi]
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (chunk0[mid] <= unit) lo = mid;
      else hi = mid;
    }
    b = lo;
    c = unit - chunk0[b];
    nch = chunk0[b + 1] - chunk0[b];
  } else {
    b = unit;
  }
  const int len = a.kv.len[b], cnt = row_count(a, b);
  s = seq_span(a, len, cnt);
  i1 = s.total();
  if (a.wgs > 0) {
    i0 = c * G_sh;
    i1 = min(i1, i0 + G_sh);
  } else {
    if (kvh == 0 && qgi == 0 && tid == 0 && !seq_fits(a, len)) atomicOr(a.kv.status, 1u);
    if (i1 == 0) return;
    __syncthreads();
  }

  C w{a, depth, ancs, q_sh, reinterpret_cast<uint16_t*>(region[wave])};
  w.lane = lane;
  w.r16 = lane & 15;
  w.g = lane >> 4;
  w.b = b;
  w.kvh = kvh;
  w.Len = len;
  w.cnt = cnt;
  w.end = a.k_new ? len : len + cnt;
  w.pmax = len + topo.max_depth;
  int pages;
  w.begin(s, i0 + wave, i1, pages);
  // a negative scale turns the queries' sign, so that the largest score is the largest product
  w.s2 = fabsf(a.scale) * kLog2e;
  const int qt0 = qgi * QPW, ntile = min(QPW, QT - qt0);
#pragma unroll
  for (int t = 0; t < QPW; ++t) {
    const int qg = (qt0 + t) * 16 + w.r16;
    int gq, slot;
    query_of(a, min(qg, Qn - 1), gq, slot);
    w.pq[t] = len + depth[slot];
    w.anc[t] = ancs[slot];
  }
  // query tiles, rotated, in operand order; padding queries and slots past the count are zero
  for (int i = tid; i < QPW * 16 * (HD / 8); i += kThreads) {
    const int cg = i % (HD / 8), q = i / (HD / 8);
    const int t = q >> 4, qg = (qt0 + t) * 16 + (q & 15);
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (qg < Qn) {
      int gq, slot;
      query_of(a, qg, gq, slot);
      if (slot < cnt)
        load_rotated8(a.q + b * a.q_seq + slot * a.q_row + (kvh * G + gq) * a.q_head, cg, a.rope,
                      (int64_t)len + depth[slot], v);
    }
    if (a.scale < 0.0f) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = -v[e];
    }
    int kk, g;
    operand_place<FP8>(cg, kk, g);
    bf16x8 hi, lo;
    split_vals(v, hi, lo);
    uint16_t* dst = q_sh + (((t * C::KSTEPS + kk) * C::QPARTS) * 64 + 16 * g + (q & 15)) * 8;
    *reinterpret_cast<bf16x8*>(dst) = hi;
    if (ROT) *reinterpret_cast<bf16x8*>(dst + 512) = lo;
  }
  __syncthreads();
  w.reset();
  w.template walk<false>(s, i0 + wave, i1, pages);
  if (!w.all_finite()) {
    w.reset();
    w.begin(s, i0 + wave, i1, pages);
    w.template walk<true>(s, i0 + wave, i1, pages);
  }

  // join the waves, tile by tile
  const size_t slot0 = ((size_t)unit * a.kv.heads + kvh) * a.groups + qgi;  // partial of this workgroup
#pragma unroll
  for (int t = 0; t < QPW; ++t) {
    if (t >= ntile) break;
    float* os = reinterpret_cast<float*>(region[wave]);
    float ls = w.lrun[t];
    ls += __shfl_xor(ls, 16);
    ls += __shfl_xor(ls, 32);
    __syncthreads();
#pragma unroll
    for (int ds = 0; ds < C::DSUB; ++ds)
#pragma unroll
      for (int r = 0; r < 4; ++r) os[(4 * w.g + r) * L::kOS + ds * 16 + w.r16] = w.o[t][ds][r];
    if (w.g == 0) {
      ml_sh[wave][w.r16][0] = w.mrun[t];
      ml_sh[wave][w.r16][1] = ls;
    }
    __syncthreads();
    for (int x = tid; x < 16 * (HD / 4); x += kThreads) {
      const int qloc = x / (HD / 4), c4 = x % (HD / 4);
      const int qg = (qt0 + t) * 16 + qloc;
      float M = -INFINITY;
#pragma unroll
      for (int v = 0; v < kWaves; ++v) M = fmaxf(M, ml_sh[v][qloc][0]);
      float S = 0.0f;
      floatx4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int v = 0; v < kWaves; ++v) {
        const float mw = ml_sh[v][qloc][0];
        if (mw == -INFINITY) continue;
        const float f = __builtin_amdgcn_exp2f(mw - M);
        S += ml_sh[v][qloc][1] * f;
        acc += f * *reinterpret_cast<const floatx4*>(reinterpret_cast<const float*>(region[v]) + qloc * L::kOS + 4 * c4);
      }
      if (nch > 1) {
        *reinterpret_cast<floatx4*>(a.part_o + ((slot0 * QPW + t) * 16 + qloc) * HD + 4 * c4) = acc;
        if (c4 == 0) *reinterpret_cast<float2*>(a.part_ml + ((slot0 * QPW + t) * 16 + qloc) * 2) = make_float2(M, S);
      } else if (qg < Qn) {
        int gq, slot;
        query_of(a, qg, gq, slot);
        if (slot >= cnt) continue;
        const float inv = S != 0.0f ? 1.0f / S : 0.0f;
        const u32x2 y = {pack_bf16x2(acc[0] * inv, acc[1] * inv), pack_bf16x2(acc[2] * inv, acc[3] * inv)};
        *reinterpret_cast<u32x2*>(a.out + b * a.out_seq + slot * a.out_row + (kvh * G + gq) * a.out_head + 4 * c4) = y;
      }
    }
  }
}

template <int HD, bool FP8, int QPW>
void launch_core(const PagedAttnArgs& a, const Topo& topo, dim3 grid, hipStream_t s) {
  if (a.rope.table) hipLaunchKernelGGL((paged_attn_kernel<HD, FP8, QPW, true>), grid, dim3(64 * kWaves), 0, s, a, topo);
  else hipLaunchKernelGGL((paged_attn_kernel<HD, FP8, QPW, false>), grid, dim3(64 * kWaves), 0, s, a, topo);
}
template <int HD, bool FP8>
void launch_tiles(const PagedAttnArgs& a, const Topo& topo, dim3 grid, hipStream_t s) {
  switch (a.q_per_wg) {
    case 1: return launch_core<HD, FP8, 1>(a, topo, grid, s);
    case 2: return launch_core<HD, FP8, 2>(a, topo, grid, s);
    default: return launch_core<HD, FP8, 3>(a, topo, grid, s);
  }
}

}  // namespace
}  // namespace msd
