// Attention of a block's rows over the paged cache.
//
// A sequence's keys are walked in blocks of 32 positions: those of the sinks, those
// from the first row's window on, and one block of the rows' own keys where
// they come beside the cache; blocks outside the window are not read. A
// workgroup owns a chunk of consecutive blocks of one (sequence, kv head) and
// up to 3 tiles of 16 queries (query head of the kv head's group, slot), its 8
// waves (two a SIMD) a block each in turn:
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
// The waves are joined in LDS; a chunk that is its sequence's only one writes the
// output, others leave (max, sum, output) in the workspace and a second kernel
// joins them in order. No atomics on values: a call repeats bit for bit.
//
// Values that no query sees are zeroed as they are staged, so NaN in stale
// rows, past the window or past the length meets no product. A non-finite value that
// only some of the wave's queries see would reach the others as 0 * NaN: where a
// wave ends with a non-finite output, the workgroup does its chunk again query by
// query, with only the keys that a query sees.
//
// What bounds it: the bytes of the seen keys and values where they are many (65.5K
// positions, 32 kv heads, 8 bits: 537 MB in 98 us, 5.5 TB/s; 16 single tokens at 512 to
// 8192: 167 MB in 38 to 42 us, 4.2 TB/s with chunks a quarter uneven); a round of
// 8 blocks takes a workgroup of 3 tiles 2.7 to 3.1 us, bytes, exponentials and products alike. Few
// bytes: a chain of latencies, as stamped in a copy: launch, plan 2.2 us, page numbers
// 2, queries and first keys 4, joining the waves 1.3 to 2.5, the second kernel 4 to 5.
// 32 positions a block, not 64: half the registers of a load, so two waves a SIMD
// (16 chains 77 -> 62 us). A chunk's own reads are 16 bytes a lane from the rows of its
// pages; keys go to the products without LDS, values through it, for their transpose.
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
  static constexpr bool kTight = QPW == 1 && HD == 64;  // two workgroups a compute unit
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

  // where tile t of the block at k0 lies: its first row and its scale
  __device__ __forceinline__ bool locate(int k0, int pages, int t, size_t& row, size_t& scale) const {
    int pg = __builtin_amdgcn_readlane(pages, t);
    const bool ok = pg >= 0 && pg < a.kv.n_pages;
    if (pg != -2 && !ok && lane == 0) atomicOr(a.kv.status, 8u);
    pg = ok ? pg : 0;
    const size_t plane = ((size_t)a.layer * a.kv.n_pages + pg) * a.kv.heads + kvh;
    const int off = (k0 + 16 * t) & ((1 << a.kv.page_shift) - 1);
    row = (plane << a.kv.page_shift) + off;
    scale = row >> 4;  // scales are [..][page / 16]: the plane's and the tile's
    return ok;
  }
  __device__ __forceinline__ void load_keys(int k0, int pages) {
    x0 = k0;
    xvalid = 0;
    size_t sc[2];
    const uint32_t at = r16 * (HD * EB) + 16 * g;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      size_t row;
      xvalid |= locate(k0, pages, t, row, sc[t]) ? 1 << t : 0;
      const char* p = static_cast<const char*>(a.kv.k) + row * (HD * EB);
#pragma unroll
      for (int w = 0; w < KW; ++w) xk[t][w] = *reinterpret_cast<const u32x4*>(p + (at + 64 * w));
    }
    if (FP8) xscale = (lane & 2 ? a.kv.v_scale : a.kv.k_scale)[lane & 1 ? sc[1] : sc[0]];
  }
  __device__ __forceinline__ void load_values(int k0, int pages) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      size_t row, sc;
      (void)locate(k0, pages, t, row, sc);
      const char* p = static_cast<const char*>(a.kv.v) + row * (HD * EB);
#pragma unroll
      for (int it = 0; it < VIT / 2; ++it)
        xv[t * (VIT / 2) + it] = *reinterpret_cast<const u32x4*>(p + ((uint32_t)lane * 16 + 1024 * it));
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
  __device__ __forceinline__ bool sees(int t, int pos, int valid, int j) const {
    return ((valid >> j) & 1) && pos < end && pos <= pq[t] &&
           (a.window <= 0 || pq[t] - pos < a.window || pos < a.sinks);
  }

  // values of the block at k0 into the wave's LDS (vs0, vs1: its tiles' scales); rows
  // that no query sees as zero
  __device__ __forceinline__ void stage(bool open, int k0, int valid, float vs0, float vs1) {
#pragma unroll
    for (int it = 0; it < VIT; ++it) {
      const int key = it * KPI + lane / LPR;
      const int t = it / (VIT / 2);
      u32x4 w = xv[it];
      if (!open) {
        const int pos = k0 + key;
        const bool live = ((valid >> t) & 1) && pos < end &&
                          (a.window <= 0 || Len - pos < a.window || pos < a.sinks);
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = live ? w[i] : 0u;
      }
      uint16_t* dst = vs + key * L::kVS;
      if constexpr (FP8) {
        const float f = t ? vs1 : vs0;
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

  // masked scores (base-2 units over s2, -inf where unseen) to weights in the running
  // softmax, in sc and as bf16 hi and lo operands
  __device__ __forceinline__ void soften(floatx4 (&sc)[QPW][2], u32x4 (&ph)[QPW], u32x4 (&pl)[QPW]) {
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
  }

  // O += P V over the staged values
  __device__ __forceinline__ void gather(const u32x4 (&ph)[QPW], const u32x4 (&pl)[QPW]) {
#pragma unroll
    for (int ds = 0; ds < DSUB; ++ds) {
      // transposing LDS reads: lane takes dim 16 ds + lane % 16 of keys 4 g + e
      // and 16 + 4 g + e (e < 4), the k order of P
      const uint16_t* p0 = vs + (4 * g + (r16 >> 2)) * L::kVS + 16 * ds + 4 * (r16 & 3);
      const v4i16 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16*)p0);
      const v4i16 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16*)(p0 + 16 * L::kVS));
      const bf16x8 vb = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
      for (int t = 0; t < QPW; ++t) {
        o[t][ds] = mfma16x16x32(__builtin_bit_cast(bf16x8, ph[t]), vb, o[t][ds]);
        o[t][ds] = mfma16x16x32(__builtin_bit_cast(bf16x8, pl[t]), vb, o[t][ds]);
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
    load_keys(k0, first);
    load_values(k0, first);
  }

  __device__ __forceinline__ void walk(const Span& s, int i0, int i1, int pages) {
    const int ic = min(i1, s.cached());
    floatx4 sc[QPW][2];
    u32x4 ph[QPW], pl[QPW];
    if (!kTight) own_blocks(s, i0, ic, i1, sc, ph, pl);
    // keys of the next block are loaded when the scores have read these, values when
    // these are staged: either is on its way for most of a round
    for (int i = i0; i < ic; i += kWaves) {
      const bool open = is_open(), more = i + kWaves < ic;
      const int k0 = x0, valid = xvalid;
      const float ks0 = block_scale(0), ks1 = block_scale(1), vs0 = block_scale(2), vs1 = block_scale(3);
      clear(sc);
      scores(sc, [&](int j, int kk) {
        if constexpr (FP8) return widen8(xk[j][kk >> 1][2 * (kk & 1)], xk[j][kk >> 1][2 * (kk & 1) + 1], j ? ks1 : ks0);
        else return __builtin_bit_cast(bf16x8, xk[j][kk]);
      });
      if (more) load_keys(s.first_pos(i + kWaves), pages);
      if (!open) {
#pragma unroll
        for (int t = 0; t < QPW; ++t)
#pragma unroll
          for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r)
              sc[t][j][r] = sees(t, k0 + 16 * j + 4 * g + r, valid, j) ? sc[t][j][r] : -INFINITY;
      }
      soften(sc, ph, pl);
      // the wave's LDS reads of its previous block are done: one wave's LDS
      // accesses complete in order
      wave_lds_sync();
      stage(open, k0, valid, vs0, vs1);
      if (more) {
        load_values(x0, pages);
        if (i + 2 * kWaves < ic) pages = page_lane(s.first_pos(i + 2 * kWaves));
      }
      wave_lds_sync();
      gather(ph, pl);
    }
    if (kTight) own_blocks(s, i0, ic, i1, sc, ph, pl);
  }

  // Own blocks of this wave: indices from s.cached() on, congruent to i0. Before the
  // cached blocks, whose first loads are on their way; with 128 registers a wave
  // (kTight) after them, when those loads' registers are free.
  __device__ __forceinline__ void own_blocks(const Span& s, int i0, int ic, int i1, floatx4 (&sc)[QPW][2],
                                             u32x4 (&ph)[QPW], u32x4 (&pl)[QPW]) {
    for (int i = ic > i0 ? i0 + (ic - i0 + kWaves - 1) / kWaves * kWaves : i0; i < i1; i += kWaves)
      if (i >= s.cached()) {
        own_scores(sc, (i - s.cached()) * kBlock);
        soften(sc, ph, pl);
        gather(ph, pl);
      }
  }

  // One row-wise copy in the wave's LDS of the rows' own keys (part 0: rounded to
  // bf16, 1: what that left) or values (part 2), slots first .. first + kBlock - 1;
  // slots past the count zero.
  __device__ __forceinline__ void stage_own(int first, int part) {
    const int64_t seq = b * a.new_seq + kvh * a.new_head;
    const int rows = min(cnt - first, kBlock) * (HD / 8);
    wave_lds_sync();
#pragma unroll 1
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
  __device__ __forceinline__ void own_scores(floatx4 (&sc)[QPW][2], int first) {
    clear(sc);
    const int parts = a.rope.table ? 2 : 1;
#pragma unroll 1
    for (int p = 0; p < parts; ++p) {
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

// The workgroup's chunk once more, a query a wave at a time, in plain steps: two lanes
// a key for the scores, then a lane the dims lane + 64 i of the keys that the query
// sees. Only for chunks that hold infinities or NaN.
template <int HD, bool FP8, int QPW, bool ROT>
__device__ __forceinline__ void walk_apart(const Core<HD, FP8, QPW, ROT>& w, const Span& s, int i0, int i1, int qt0,
                                           int ntile, bool partial, size_t slot0) {
  using C = Core<HD, FP8, QPW, ROT>;
  const PagedAttnArgs& a = w.a;
  const int lane = w.lane, key = lane & 31, half = lane >> 5;
  const int G = a.n_heads / a.kv.heads, Qn = G * a.n_slots;
  const int64_t seq = w.b * a.new_seq + w.kvh * a.new_head;
  auto row_of = [&](int pos) -> int64_t {  // row of the pages, -1: no page
    const int pg = a.kv.page_table[(size_t)w.b * a.kv.max_pages + (pos >> a.kv.page_shift)];
    if (pg < 0 || pg >= a.kv.n_pages) return -1;
    const int64_t plane = ((int64_t)a.layer * a.kv.n_pages + pg) * a.kv.heads + w.kvh;
    return (plane << a.kv.page_shift) + (pos & ((1 << a.kv.page_shift) - 1));
  };
#pragma unroll 1
  for (int q = threadIdx.x >> 6; q < ntile * 16; q += kWaves) {
    const int qg = qt0 * 16 + q;
    if (qg >= Qn) break;
    int gq, slot;
    query_of(a, qg, gq, slot);
    if (slot >= w.cnt) continue;
    const int P = w.Len + w.depth[slot];
    const uint64_t anc = w.ancs[slot];
    float m = -INFINITY, sum = 0.0f, o[HD / 64];
#pragma unroll
    for (int i = 0; i < HD / 64; ++i) o[i] = 0.0f;
#pragma unroll 1
    for (int i = i0; i < i1; ++i) {
      const bool own = i >= s.cached();
      const int k0 = own ? (i - s.cached()) * kBlock : s.first_pos(i);
      const int at = k0 + key;  // slot or position
      const int pos = own ? w.Len + w.depth[min(at, kMaxSlots - 1)] : at;
      bool vis = own ? at < w.cnt && ((anc >> (at & 63)) & 1ull) : at < w.end && at <= P;
      vis = vis && (a.window <= 0 || P - pos < a.window || pos < a.sinks);
      const int64_t row = vis && !own ? row_of(at) : 0;
      vis = vis && row >= 0;
      float acc = 0.0f;
      if (vis) {
#pragma unroll 1
        for (int c = half * (HD / 16); c < (half + 1) * (HD / 16); ++c) {
          float k[8];
          if (own) {
            load_rotated8(a.k_new + seq + at * a.new_row, c, a.rope, pos, k);
          } else if constexpr (FP8) {
            const u32x2 x = *reinterpret_cast<const u32x2*>(static_cast<const uint8_t*>(a.kv.k) + row * HD + 8 * c);
            const float f = scale_value(a.kv.k_scale[row >> 4]);
            float lo[4], hi[4];
            decode4(x[0], lo);
            decode4(x[1], hi);
#pragma unroll
            for (int e = 0; e < 4; ++e) k[e] = lo[e] * f, k[4 + e] = hi[e] * f;
          } else {
            load8(static_cast<const uint16_t*>(a.kv.k) + row * HD + 8 * c, k);
          }
          int kk, g;
          operand_place<FP8>(c, kk, g);
          const uint16_t* qp = w.q_sh + ((((q >> 4) * C::KSTEPS + kk) * C::QPARTS) * 64 + 16 * g + (q & 15)) * 8;
#pragma unroll
          for (int e = 0; e < 8; ++e) acc += (bf2f(qp[e]) + (ROT ? bf2f(qp[512 + e]) : 0.0f)) * k[e];
        }
      }
      acc += __shfl_xor(acc, 32);
      const float sc = vis ? acc * w.s2 : -INFINITY;
      const float mn = fmaxf(m, wave_max(sc));
      const float ref = mn == -INFINITY ? 0.0f : mn;
      const float alpha = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m - ref);
      const float p = vis ? __builtin_amdgcn_exp2f(sc - ref) : 0.0f;
      sum = sum * alpha + wave_sum(half ? 0.0f : p);
      m = mn;
#pragma unroll
      for (int e = 0; e < HD / 64; ++e) o[e] *= alpha;
      const uint32_t seen = (uint32_t)__ballot(vis);
#pragma unroll 1
      for (int k = 0; k < kBlock; ++k) {
        const float pk = __shfl(p, k);
        if (!((seen >> k) & 1u) || pk == 0.0f) continue;
        const int64_t r = own ? 0 : row_of(k0 + k);
#pragma unroll
        for (int e = 0; e < HD / 64; ++e) {
          const int d = lane + 64 * e;
          float v;
          if (own) v = bf2f(a.v_new[seq + (k0 + k) * a.new_row + d]);
          else if constexpr (FP8)
            v = __builtin_amdgcn_cvt_pk_f32_fp8((int)static_cast<const uint8_t*>(a.kv.v)[r * HD + d], false)[0] *
                scale_value(a.kv.v_scale[r >> 4]);
          else v = bf2f(static_cast<const uint16_t*>(a.kv.v)[r * HD + d]);
          o[e] += pk * v;
        }
      }
    }
    const size_t part = (slot0 * QPW + (q >> 4)) * 16 + (q & 15);
    if (partial && lane == 0) *reinterpret_cast<float2*>(a.part_ml + part * 2) = make_float2(m, sum);
    const float inv = sum != 0.0f ? 1.0f / sum : 0.0f;
#pragma unroll
    for (int e = 0; e < HD / 64; ++e) {
      const int d = lane + 64 * e;
      if (partial) a.part_o[part * HD + d] = o[e];
    }
    if (!partial) {  // 4 dims a lane, from the lanes that hold them
#pragma unroll
      for (int e = 0; e < HD / 64; ++e) {
        float y[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) y[k] = __shfl(o[e], (4 * lane + k) & 63) * inv;
        if (lane < 16) write_output(a, w.b, w.kvh * G + gq, slot, 64 * e + 4 * lane, y);
      }
    }
  }
}

template <int HD, bool FP8, int QPW, bool ROT>
__global__ __launch_bounds__(64 * kWaves, (Core<HD, FP8, QPW, ROT>::kTight) ? 4 : 2) void paged_attn_kernel(
    PagedAttnArgs a, Topo topo) {
  using C = Core<HD, FP8, QPW, ROT>;
  using L = Lds<HD>;
  constexpr int kThreads = 64 * kWaves;
  __shared__ __attribute__((aligned(16))) unsigned char region[kWaves][L::kRegion];
  __shared__ __attribute__((aligned(16))) uint16_t q_sh[QPW * C::KSTEPS * C::QPARTS * 512];
  __shared__ float ml_sh[kWaves][16][2];
  __shared__ int chunk0[kPagedPlanBatch + 1];
  __shared__ int depth[kMaxSlots];
  __shared__ uint64_t ancs[kMaxSlots];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int G = a.n_heads / a.kv.heads;
  const int Qn = G * a.n_slots, QT = (Qn + 15) >> 4;

  // kv heads first: the hardware deals workgroups to the 8 XCDs in turn, so the
  // query groups of a chunk that re-read its keys meet in one L2 where the kv heads
  // are a multiple of 8
  int id = blockIdx.x;
  const int kvh = id % a.kv.heads;
  id /= a.kv.heads;
  const int qgi = id % a.groups;
  const int unit = id / a.groups;
  const int qt0 = qgi * QPW, ntile = min(QPW, QT - qt0);
  if (wave == 1) {
    depth[lane] = topo.depth[lane];
    ancs[lane] = topo.anc[lane];
  }
  if (a.wgs > 0 && wave == 0) plan_chunks(a, chunk0, blockIdx.x == 0);
  __syncthreads();
  int b = unit, c = 0, nch = 1;
  if (a.wgs > 0) {
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
  }
  const int len = a.kv.len[b], cnt = row_count(a, b);
  const Span s = seq_span(a, len, cnt);
  if (a.wgs == 0 && kvh == 0 && qgi == 0 && tid == 0 && !seq_fits(a, len)) atomicOr(a.kv.status, 1u);
  if (s.total() == 0) return;
  const int size = chunk_size(s.total(), nch);
  const int i0 = min(c * size, s.total());  // rounding up may leave the last chunks less, or nothing
  const int i1 = min(s.total(), i0 + size);

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
    int kk, g;
    operand_place<FP8>(cg, kk, g);
    uint16_t* dst = q_sh + (((t * C::KSTEPS + kk) * C::QPARTS) * 64 + 16 * g + (q & 15)) * 8;
    if (ROT && a.q_img) {  // already hi and lo, 8 dims a lane and k-step
      bf16x8 hi = zero_bf16x8(), lo = hi;
      if (qg < Qn) {
        const uint16_t* src = a.q_img + (((size_t)b * a.kv.heads + kvh) * QT + qt0 + t) * (size_t)(C::KSTEPS * 1024) +
                              (cg >> 2) * 1024 + (16 * (cg & 3) + (q & 15)) * 8;
        hi = load16(src);
        lo = load16(src + 512);
      }
      *reinterpret_cast<bf16x8*>(dst) = hi;
      *reinterpret_cast<bf16x8*>(dst + 512) = lo;
      continue;
    }
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
    bf16x8 hi, lo;
    split_vals(v, hi, lo);
    *reinterpret_cast<bf16x8*>(dst) = hi;
    if (ROT) *reinterpret_cast<bf16x8*>(dst + 512) = lo;
  }
  __syncthreads();
  w.reset();
  w.walk(s, i0 + wave, i1, pages);
  const size_t slot0 = ((size_t)unit * a.kv.heads + kvh) * a.groups + qgi;  // place of the partial result
  if (__syncthreads_or(!w.all_finite())) {
    walk_apart(w, s, i0, i1, qt0, ntile, nch > 1, slot0);
    return;
  }

  // join the waves, tile by tile
#pragma unroll
  for (int t = 0; t < QPW; ++t) {
    if (t >= ntile) break;
    float* os = reinterpret_cast<float*>(region[wave]);
    float ls = w.lrun[t];
    ls += __shfl_xor(ls, 16);
    ls += __shfl_xor(ls, 32);
    if (t) __syncthreads();
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
        const float y[4] = {acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv};
        write_output(a, b, kvh * G + gq, slot, 4 * c4, y);
      }
    }
  }
}

template <int HD, bool FP8, int QPW>
void launch_core(const PagedAttnArgs& a, const Topo& topo, dim3 grid, hipStream_t s) {
  if (a.rope.table || a.q_img) hipLaunchKernelGGL((paged_attn_kernel<HD, FP8, QPW, true>), grid, dim3(64 * kWaves), 0, s, a, topo);
  else hipLaunchKernelGGL((paged_attn_kernel<HD, FP8, QPW, false>), grid, dim3(64 * kWaves), 0, s, a, topo);
}
template <int HD, bool FP8>
void launch_tiles(const PagedAttnArgs& a, const Topo& topo, dim3 grid, hipStream_t s) {
  if (a.q_per_wg == 1) return launch_core<HD, FP8, 1>(a, topo, grid, s);
  if (a.q_per_wg == 2) return launch_core<HD, FP8, 2>(a, topo, grid, s);
  if constexpr (paged_max_tiles(FP8, HD) == 3) launch_core<HD, FP8, 3>(a, topo, grid, s);
}

}  // namespace
}  // namespace msd
